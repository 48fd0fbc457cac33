"""GPU: causal attention over packed sequences with grouped heads, against the definition in 64 bits element by element."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _inputs(lens, H, Hkv, dh, dtype, gain=1.0, seed=0):
    from synth import to_bf16_round
    rng = np.random.default_rng(sum(lens) * 131 + H * 17 + Hkv + dh + seed)
    qkv = rng.standard_normal((sum(lens), (H + 2 * Hkv) * dh)).astype(np.float32)
    qkv[:, :(H + Hkv) * dh] *= gain
    dO = rng.standard_normal((sum(lens), H * dh)).astype(np.float32)
    return (to_bf16_round(qkv), to_bf16_round(dO)) if dtype == "bf16" else (qkv, dO)


def _check(lens, dtype, H, Hkv, dh, gain=1.0, **more):
    import packedlib as pl
    print(f"packed attention {dtype} lens={lens} H={H} Hkv={Hkv} dh={dh} gain={gain} {more}", flush=True)
    qkv, dO = _inputs(lens, H, Hkv, dh, dtype, gain)
    u = 2.0 ** -8 if dtype == "bf16" else 1e-5              # fp32: sums of up to a few thousand terms in 32 bits
    o, lse, d, ob, db = pl.attention(lens, H, Hkv, dh, qkv, dO, u)
    got = pl.run_attention(lens, dtype, H, Hkv, dh, qkv, dO, **more)
    err = np.abs(got[0].double().cpu().numpy() - o)
    assert np.all(err <= ob + 1e-30), ("o", float((err / (ob + 1e-30)).max()))
    # products of up to 128 terms and sums of exponentials in 32 bits: relative to the scores' size
    assert np.abs(got[1].double().cpu().numpy() - lse).max() <= 2e-5 * (1 + np.abs(lse).max())
    # where the reference and its bound vanish (one row: dQ, dK), dP - delta is what the rounding of O leaves of two equal sums
    err = np.abs(got[2].double().cpu().numpy() - d)
    at = np.unravel_index(np.argmax(err / (db + 1e-30)), err.shape)
    assert np.all(err <= db + 1e-30), ("dqkv", at, float(err[at]), float(db[at]))
    print("  worst error / bound", float((err / (db + 1e-30)).max()), flush=True)


LENS = [1, 45, 0, 17, 33, 64, 65, 130]


@pytest.mark.parametrize("H,Hkv", [(1, 1), (4, 2), (6, 2), (8, 2), (5, 1), (7, 1), (8, 8), (16, 2), (13, 1), (9, 3), (32, 1), (33, 1), (64, 1)])
@pytest.mark.parametrize("dh", [64, 128])
def test_groups(H, Hkv, dh):
    _check(LENS, "bf16", H, Hkv, dh)


@pytest.mark.parametrize("dtype,H,Hkv,dh", [("fp32", 4, 2, 32), ("fp32", 3, 1, 64), ("fp32", 2, 2, 128), ("fp32", 8, 1, 32), ("bf16", 4, 1, 32), ("bf16", 6, 6, 32)])
@pytest.mark.parametrize("lens", [LENS, [1], [32], [33, 31], [200, 0, 1]])
def test_fp32_arithmetic(dtype, H, Hkv, dh, lens):
    _check(lens, dtype, H, Hkv, dh)


# one row; ends of tiles of 32 and 64 keys and of blocks of 64, 128 and 256 rows, alone and behind one another
@pytest.mark.parametrize("lens", [[1], [2], [1, 1, 1], [31], [32], [63], [64, 64], [127, 1, 128], [129], [255], [256, 257], [321, 320], [0, 0, 5, 0]])
@pytest.mark.parametrize("H,Hkv,dh", [(4, 1, 64), (3, 3, 64), (6, 2, 128), (8, 2, 128)])
def test_ends_of_tiles_and_blocks(lens, H, Hkv, dh):
    _check(lens, "bf16", H, Hkv, dh)


# blocks of keys whose tiles are shared by several workgroups; many heads, so that a wavefront has 32 query rows instead of 16
@pytest.mark.parametrize("lens,H,Hkv,dh", [([1500], 4, 1, 64), ([900, 40], 6, 2, 128), ([1111, 700], 5, 1, 128), ([1024], 2, 2, 64),
                                           ([700, 650, 30, 512], 48, 8, 64), ([600, 555, 800], 40, 10, 128), ([2048], 7, 1, 64)])
def test_long_and_many(lens, H, Hkv, dh):
    _check(lens, "bf16", H, Hkv, dh)


@pytest.mark.parametrize("dtype,H,Hkv,dh", [("bf16", 4, 2, 64), ("bf16", 3, 1, 128), ("fp32", 2, 1, 32)])
def test_a_thousand_sequences(dtype, H, Hkv, dh):
    _check([1, 2, 0, 3, 1] * 250, dtype, H, Hkv, dh)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(4, 1), (3, 1)])
def test_scores_whose_maximum_keeps_rising(dh, H, Hkv):
    """Scores of +-50: the softmax's reference exponent is raised many times and by more than the range it tolerates."""
    _check([300, 33, 170], "bf16", H, Hkv, dh, gain=4.0)


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("bf16", 32), ("fp32", 32), ("fp32", 64)])
def test_strides_and_rows_behind_the_last_sequence(dtype, dh):
    """Columns behind the heads and rows behind the batch hold NaN where they are read from, and keep what they held where they are not written."""
    _check([70, 3, 131], dtype, 6, 2, dh, extra_rows=40, pad=24, pad_o=8)


@pytest.mark.parametrize("dtype,H,Hkv,dh", [("bf16", 4, 2, 64), ("bf16", 6, 2, 128), ("bf16", 4, 1, 32), ("fp32", 4, 2, 32), ("fp32", 2, 1, 64)])
def test_sequences_do_not_see_each_other(dtype, H, Hkv, dh):
    """Every other sequence NaN: the rest has the bits that it has alone."""
    import torch
    import packedlib as pl
    lens = [50, 64, 7, 129, 300, 31]
    print(f"packed attention beside NaN {dtype} H={H} Hkv={Hkv} dh={dh}", flush=True)
    qkv, dO = _inputs(lens, H, Hkv, dh, dtype)
    off = pl.offsets(lens)
    for bad in range(2):
        x, g = qkv.copy(), dO.copy()
        for i in range(bad, len(lens), 2):
            x[off[i]:off[i + 1]] = np.nan
            g[off[i]:off[i + 1]] = np.nan
        o, lse, d = pl.run_attention(lens, dtype, H, Hkv, dh, x, g)
        for i in range(1 - bad, len(lens), 2):
            r = slice(off[i], off[i + 1])
            a = pl.run_attention([lens[i]], dtype, H, Hkv, dh, qkv[r], dO[r])
            assert torch.isfinite(d[r]).all()
            assert torch.equal(o[r], a[0]) and torch.equal(lse[:, r], a[1])
            # blocks of keys may be cut differently: their sums are then in another order
            assert torch.equal(d[r][:, :H * dh], a[2][:, :H * dh])


@pytest.mark.parametrize("dtype,H,Hkv,dh", [("bf16", 4, 2, 64), ("bf16", 3, 1, 64), ("bf16", 48, 8, 64), ("bf16", 8, 2, 128), ("bf16", 5, 1, 128), ("bf16", 32, 8, 128),
                                            ("fp32", 4, 2, 32), ("bf16", 4, 1, 32)])
@pytest.mark.parametrize("value", [-np.inf, -1e30])
def test_whole_tiles_of_keys_that_count_for_nothing(dtype, H, Hkv, dh, value):
    """The first 70 keys of a sequence, and others, far below the rest: rows that see another one have the values of a batch in which these keys
    and their values are not there.  Bounds as above: the sums' order and the roundings of P are others."""
    import packedlib as pl
    lens, first, n = [20, 400, 5], 20, 400
    print(f"packed attention, keys that count for nothing {dtype} H={H} Hkv={Hkv} dh={dh} {value}", flush=True)
    qkv, dO = _inputs(lens, H, Hkv, dh, dtype)
    x = qkv.reshape(-1, H + 2 * Hkv, dh).copy()
    x[:, :H, 5] = np.abs(x[:, :H, 5]) + 0.25
    if dtype == "bf16":
        from synth import to_bf16_round
        x = to_bf16_round(x)
    gone = list(range(70)) + list(range(128, 160)) + [200]
    x[[first + k for k in gone], H:H + Hkv, 5] = value
    o, lse, _ = pl.run_attention(lens, dtype, H, Hkv, dh, x.reshape(len(x), -1), dO)
    keep = [k for k in range(n) if k not in gone]
    u, G = 2.0 ** -8 if dtype == "bf16" else 1e-5, H // Hkv
    got, got_lse = o.double().cpu().numpy().reshape(-1, H, dh)[first:first + n], lse.double().cpu().numpy()[:, first:first + n]
    q = x[first:first + n].astype(np.float64)
    for h in range(H):
        s = np.where(np.array(keep)[None, :] > np.arange(70, n)[:, None], -np.inf, q[70:, h] @ q[keep, H + h // G].T / np.sqrt(dh))
        m = s.max(1, keepdims=True)
        e = np.exp(s - m)
        p = e / e.sum(1, keepdims=True)
        v = q[keep, H + Hkv + h // G]
        assert np.all(np.abs(got[70:, h] - p @ v) <= u * (np.abs(p @ v) + p @ np.abs(v))), h
        assert np.abs(got_lse[h, 70:] - (m + np.log(e.sum(1, keepdims=True)))[:, 0]).max() <= 1e-3


@pytest.mark.parametrize("H,Hkv,dh", [(4, 2, 64), (3, 1, 64), (8, 2, 128), (5, 1, 128)])
def test_gradients_of_keys_at_minus_infinity(H, Hkv, dh):
    """A key whose scores are all -inf takes part in nothing: the gradients are those of a key far below every other.  The forward pass
    rescales at other tiles then, which changes the rounding of probabilities, their gradients and the outputs to bf16: 2^-8 each."""
    import torch
    import packedlib as pl
    lens = [50, 333, 64, 1, 129]
    qkv, dO = _inputs(lens, H, Hkv, dh, "bf16")
    off = pl.offsets(lens)
    x = qkv.reshape(-1, H + 2 * Hkv, dh)
    x[:, :H, 5] = np.abs(x[:, :H, 5]) + 0.25
    keys = [int(r) for a, n in zip(off, lens) if n > 4 for r in (a + 1, a + n // 2, a + n - 1)]

    def run(value):
        y = x.copy()
        y[keys, H:H + Hkv, 5] = value
        return pl.run_attention(lens, "bf16", H, Hkv, dh, y.reshape(len(y), -1), dO)
    low, far = run(-np.inf), run(-1e30)
    for name, a, b in (("o", low[0], far[0]), ("lse", low[1], far[1]), ("dk, dv", low[2][:, H * dh:], far[2][:, H * dh:])):
        assert torch.isfinite(a).all(), name
        a, b = a.double(), b.double()
        assert ((a - b).norm() <= 3 * 2.0 ** -8 * b.norm()).item(), name


@pytest.mark.parametrize("lens,H,Hkv,dh", [([34, 2, 3, 27], 8, 4, 64), ([17] * 4, 12, 12, 64), ([8, 1, 208, 14], 8, 2, 128), ([300, 9, 40], 10, 2, 128), ([60] * 5, 33, 1, 64),
                                           ([1500, 40], 8, 2, 64), ([700, 650, 30, 512], 48, 8, 64), ([600, 555, 800], 40, 10, 128)])
def test_short_rows_keep_their_precision(lens, H, Hkv, dh):
    """dQ of the first sixteen rows of every sequence, and dQ and dK of short batches, are as far off as two roundings make them.

    dS is rounded to bf16 and the result is, each an independent error of the same size relative to the norm, which is that of the definition's result
    rounded once: together sqrt(2) of it.  P, of which dS is made, and delta are held to 32 bits here; half a rounding of delta in O would add 0.7 to 1 of
    it in rows of few keys.  6 % for the sample: the few hundred roundings of dS that count."""
    import torch
    import packedlib as pl
    print(f"precision lens={lens} H={H} Hkv={Hkv} dh={dh}", flush=True)
    qkv, dO = _inputs(lens, H, Hkv, dh, "bf16")
    d = pl.attention(lens, H, Hkv, dh, qkv, dO, 0.0)[2]
    once = torch.from_numpy(d).to(torch.bfloat16).double().numpy()
    got = pl.run_attention(lens, "bf16", H, Hkv, dh, qkv, dO)[2].double().cpu().numpy()
    first = np.concatenate([a + np.arange(min(n, 16)) for a, n in zip(pl.offsets(lens), lens)])
    parts = {"dq": (first, slice(0, H * dh))}
    if max(lens) <= 300:
        parts |= {"all dq": (slice(None), slice(0, H * dh)), "dk": (slice(None), slice(H * dh, (H + Hkv) * dh))}
    for name, at in parts.items():
        a, b = (np.linalg.norm(x[at] - d[at]) for x in (got, once))
        assert a <= 1.5 * b, (name, a / b)


@pytest.mark.parametrize("dtype,H,Hkv,dh", [("bf16", 4, 2, 64), ("bf16", 5, 1, 128), ("fp32", 4, 2, 32)])
def test_gradients_against_differences(dtype, H, Hkv, dh):
    """Directional differences of the forward pass's own log-sum-exp and output in fp32-readable steps: the gradient of sum(w * o) along a random
    direction against (f(x + t v) - f(x - t v)) / 2 t of the definition in 64 bits, from the kernel's gradient."""
    import packedlib as pl
    lens = [40, 1, 77]
    qkv, dO = _inputs(lens, H, Hkv, dh, dtype)
    v = np.random.default_rng(5).standard_normal(qkv.shape)
    t = 1e-5
    f = [float((pl.attention(lens, H, Hkv, dh, qkv.astype(np.float64) + s * t * v, dO, 0.0)[0] * dO).sum()) for s in (1, -1)]
    got = pl.run_attention(lens, dtype, H, Hkv, dh, qkv, dO)[2].double().cpu().numpy()
    bound = pl.attention(lens, H, Hkv, dh, qkv, dO, 2.0 ** -8 if dtype == "bf16" else 1e-5)[4]
    assert abs((f[0] - f[1]) / (2 * t) - (got * v).sum()) <= np.sqrt((bound * v) ** 2).sum() * 0.1 + 1e-4


def test_same_bits_again_and_on_another_stream():
    import torch
    import packedlib as pl
    lens, H, Hkv, dh = [900, 33, 257], 6, 2, 64
    qkv, dO = _inputs(lens, H, Hkv, dh, "bf16")
    first = pl.run_attention(lens, "bf16", H, Hkv, dh, qkv, dO)
    s = torch.cuda.Stream()
    again = pl.run_attention(lens, "bf16", H, Hkv, dh, qkv, dO, stream=s.cuda_stream)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_two_streams_at_once():
    """Two batches on two streams, buffers of their own: neither changes the other's bits."""
    import torch
    import paper_2506_06472_amd as tio
    import packedlib as pl
    cases = [([900, 33, 257], "bf16", 6, 2, 64), ([400, 31, 700], "bf16", 8, 2, 128)]
    alone, states = [], []
    for lens, dtype, H, Hkv, dh in cases:
        qkv, dO = _inputs(lens, H, Hkv, dh, dtype)
        alone.append(pl.run_attention(lens, dtype, H, Hkv, dh, qkv, dO))
        p, dev = pl.packing(lens, dtype, H, Hkv, dh)
        q, g = (torch.from_numpy(a).cuda().bfloat16() for a in (qkv, dO))
        states.append((p, dev, q, g, torch.zeros_like(g), torch.zeros_like(q), torch.zeros((H, sum(lens)), device="cuda"),
                       torch.zeros(tio.tio_op_attention_packed_work(p), device="cuda", dtype=torch.uint8), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(5):
        for p, dev, q, g, o, d, lse, work, s in states:
            tio.tio_op_attention_packed(s.cuda_stream, p, dev.data_ptr(), q.data_ptr(), q.stride(0), o.data_ptr(), o.stride(0), lse.data_ptr())
            tio.tio_op_attention_packed_bwd(s.cuda_stream, p, dev.data_ptr(), q.data_ptr(), q.stride(0), o.data_ptr(), g.data_ptr(), o.stride(0),
                                            lse.data_ptr(), work.data_ptr(), d.data_ptr())
    torch.cuda.synchronize()
    for want, (_, _, _, _, o, d, lse, _, _) in zip(alone, states):
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1]) and torch.equal(d, want[2])


@pytest.mark.parametrize("dtype,H,Hkv,dh", [("bf16", 6, 2, 64), ("bf16", 8, 2, 128), ("fp32", 4, 2, 32)])
def test_captured_and_replayed(dtype, H, Hkv, dh):
    """Forward and backward in a graph, replayed on new inputs with eager work in between: the eager bits every time."""
    import torch
    import paper_2506_06472_amd as tio
    import packedlib as pl
    lens = [700, 1, 65, 128]
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    p, dev = packed = pl.packing(lens, dtype, H, Hkv, dh)
    qkv, dO = (torch.zeros((sum(lens), n * dh), device="cuda", dtype=t) for n in (H + 2 * Hkv, H))
    o, dqkv, lse = torch.zeros_like(dO), torch.zeros_like(qkv), torch.zeros((H, sum(lens)), device="cuda")
    work = torch.zeros(tio.tio_op_attention_packed_work(p), device="cuda", dtype=torch.uint8)

    def call(stream):
        tio.tio_op_attention_packed(stream, p, dev.data_ptr(), qkv.data_ptr(), qkv.stride(0), o.data_ptr(), o.stride(0), lse.data_ptr())
        tio.tio_op_attention_packed_bwd(stream, p, dev.data_ptr(), qkv.data_ptr(), qkv.stride(0), o.data_ptr(), dO.data_ptr(), o.stride(0),
                                        lse.data_ptr(), work.data_ptr(), dqkv.data_ptr())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(s.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(torch.cuda.current_stream().cuda_stream)
    for seed in range(3):
        a, b = _inputs(lens, H, Hkv, dh, dtype, seed=seed)
        qkv.copy_(torch.from_numpy(a))
        dO.copy_(torch.from_numpy(b))
        graph.replay()
        torch.cuda.synchronize()
        eager = pl.run_attention(lens, dtype, H, Hkv, dh, a, b, packed=packed)
        for name, x, y in zip(("o", "lse", "dqkv"), (o, lse, dqkv), eager):
            assert torch.equal(x, y), (seed, name)


@pytest.mark.parametrize("H,Hkv,dh", [(4, 2, 64), (3, 1, 64), (33, 1, 64), (8, 2, 128), (5, 1, 128), (4, 4, 128)])
@pytest.mark.parametrize("more", [[], [700]], ids=["short", "beside a long one"])
def test_gradients_of_keys_at_minus_infinity_in_short_sequences(H, Hkv, dh, more):
    """Sequences of fewer than sixteen rows in which a key's scores are all -inf: it takes part in nothing, so dK and dV are the definition's, and so is
    dQ but for the component in which the key is infinite (zero times infinity)."""
    import packedlib as pl
    lens = [5, 40, 9, 2, 15, 0, 3, 16, 17] + more
    print(f"packed attention, infinite keys of short sequences lens={lens} H={H} Hkv={Hkv} dh={dh}", flush=True)
    qkv, dO = _inputs(lens, H, Hkv, dh, "bf16")
    x = qkv.reshape(-1, H + 2 * Hkv, dh)
    x[:, :H, 5] = np.abs(x[:, :H, 5]) + 0.25
    from synth import to_bf16_round
    x = to_bf16_round(x)
    for a, n in zip(pl.offsets(lens), lens):
        if n > 1:
            x[int(a) + max(1, n // 2), H:H + Hkv, 5] = -np.inf
    qkv = x.reshape(len(x), -1)
    with np.errstate(invalid="ignore"):
        o, _, d, ob, db = pl.attention(lens, H, Hkv, dh, qkv, dO, 2.0 ** -8)
    got = [t.double().cpu().numpy() for t in pl.run_attention(lens, "bf16", H, Hkv, dh, qkv, dO)]
    assert np.all(np.abs(got[0] - o) <= ob + 1e-30)
    there = np.ones(d.shape, bool)
    there[:, :H * dh].reshape(len(d), H, dh)[:, :, 5] = False
    assert np.isfinite(d[there]).all() and np.isfinite(db[there]).all() and np.isfinite(got[2][there]).all()
    assert np.all(np.abs(got[2] - d)[there] <= db[there] + 1e-30)


# batches of both sizes of forward blocks, with one set and two of wavefronts; keys in the first seventy rows of the second sequence
LOW_BATCHES = [("bf16", [20, 400, 5], 4, 2, 64), ("bf16", [20, 400, 5], 3, 1, 64), ("bf16", [20, 400, 5], 5, 1, 128), ("bf16", [20, 400, 5], 33, 1, 64),
               ("bf16", [300, 400, 340], 32, 8, 128), ("bf16", [300, 400, 340], 48, 16, 64), ("bf16", [700, 650, 600, 580], 64, 8, 64),
               ("bf16", [500, 400, 340, 600, 700], 32, 8, 128), ("fp32", [20, 400, 5], 4, 2, 32), ("fp32", [20, 400, 5], 2, 1, 64), ("bf16", [20, 400, 5], 4, 1, 32)]


def _low_scores(dtype, lens, H, Hkv, dh, how, power, sign=-1, low=70):
    """The first `low` keys of the second sequence have scores of -1.0625 2^power and less (sign = 1: that and more), each an exact product (and of a size at
    which exp2(score - log-sum-exp), of two rounded numbers, is infinite).  Its rows, the definition's values for them, and the library's for the batch."""
    import packedlib as pl
    print(f"packed attention, low scores {dtype} lens={lens} H={H} Hkv={Hkv} dh={dh} {how} {sign} 2^{power}", flush=True)
    second, n = lens[0], lens[1]
    qkv, dO = _inputs(lens, H, Hkv, dh, dtype)
    x = qkv.reshape(-1, H + 2 * Hkv, dh)
    x[:, :H, 5] = 1.0
    x[second:second + low, H:H + Hkv] = 0.0
    at = {"equal": np.full(low, power), "falling": power + np.arange(low) // 4, "rising": power + (low - np.arange(low)) // 4}[how]
    x[second:second + low, H:H + Hkv, 5] = sign * 1.0625 * np.exp2(np.minimum(at, 120).astype(float))[:, None]
    qkv = x.reshape(len(x), -1)
    rows = slice(second, second + n)
    want = pl.attention([n], H, Hkv, dh, qkv[rows], dO[rows], 2.0 ** -8 if dtype == "bf16" else 1e-5)
    return rows, want, [t.double().cpu().numpy() for t in pl.run_attention(lens, dtype, H, Hkv, dh, qkv, dO)]


@pytest.mark.parametrize("dtype,lens,H,Hkv,dh", LOW_BATCHES)
@pytest.mark.parametrize("how", ["equal", "falling", "rising"])
@pytest.mark.parametrize("power", [23, 40, 100])
def test_rows_that_see_only_very_low_scores(dtype, lens, H, Hkv, dh, how, power):
    """Such rows have the softmax of what they see (all alike; the first, or the latest, of keys far apart), the rows behind them that of the other keys."""
    low = 70
    rows, (o, lse, _, ob, _), got = _low_scores(dtype, lens, H, Hkv, dh, how, power)
    assert np.all(np.abs(got[0][rows] - o) <= ob + 1e-30)
    # of a low row: the scale, the product and the sum with log l, each 2^-24 of it
    err = np.abs(got[1][:, rows] - lse)
    assert np.all(err[:, :low] <= 2.0 ** -21 * np.abs(lse[:, :low])) and err[:, low:].max() <= 2e-5 * (1 + np.abs(lse[:, low:]).max())
    assert np.isfinite(got[0]).all() and np.isfinite(got[1]).all()


@pytest.mark.parametrize("dtype,lens,H,Hkv,dh", LOW_BATCHES)
@pytest.mark.parametrize("how", ["equal", "falling", "rising"])
@pytest.mark.parametrize("power", [23, 40, 100])
def test_rows_that_see_very_high_scores(dtype, lens, H, Hkv, dh, how, power):
    """The rows behind them too have the softmax of these keys alone."""
    rows, (o, lse, _, ob, _), got = _low_scores(dtype, lens, H, Hkv, dh, how, power, 1)
    assert np.all(np.abs(got[0][rows] - o) <= ob + 1e-30)
    assert np.all(np.abs(got[1][:, rows] - lse) <= 2.0 ** -21 * np.abs(lse))
    assert np.isfinite(got[0]).all() and np.isfinite(got[1]).all()


@pytest.mark.parametrize("dtype,lens,H,Hkv,dh", LOW_BATCHES)
@pytest.mark.parametrize("how", ["equal", "falling", "rising"])
@pytest.mark.parametrize("power", [23, 40, 100])
@pytest.mark.parametrize("low", [9, 70])
def test_gradients_beside_rows_of_very_low_scores(dtype, lens, H, Hkv, dh, how, power, low):
    """Gradients of the rows and keys behind them are the definition's: neither those keys nor the rows that see only them count there, in the blocks that
    they share with them either."""
    rows, (_, _, d, _, db), got = _low_scores(dtype, lens, H, Hkv, dh, how, power, low=low)
    assert np.all(np.abs(got[2][rows] - d)[low:] <= db[low:] + 1e-30)
    assert np.isfinite(got[2][:rows.start]).all() and np.isfinite(got[2][rows.stop:]).all()


# (rows of a forward block, keys of a backward block, whether blocks of keys are cut) of each batch: the kernels of large batches
@pytest.mark.parametrize("lens,H,Hkv,dh,want", [
    ([900, 11], 66, 2, 64, (64, 128, True)), ([900, 800, 14], 64, 16, 64, (64, 128, True)), ([1100, 9, 64], 64, 4, 64, (64, 128, True)),
    ([800, 780, 300, 31, 1, 7], 64, 64, 64, (128, 128, False)), ([1000, 900, 9], 64, 32, 64, (128, 128, False)),
    ([700, 690, 640, 513, 0, 9], 48, 8, 64, (128, 128, True)), ([700, 650, 600, 580, 12], 64, 8, 64, (128, 128, True)),
    ([1500, 13], 40, 8, 128, (64, 256, True)), ([1500, 200, 9, 1], 32, 8, 128, (64, 256, True)), ([1500, 9], 32, 32, 128, (64, 256, False)),
    ([1200, 9], 64, 8, 128, (128, 256, True)), ([1300, 3], 64, 2, 128, (128, 256, True)), ([1400, 11], 66, 2, 128, (128, 256, True)),
    ([1000, 700, 0, 300, 15], 64, 64, 128, (128, 64, False))])
def test_blocks_of_large_batches(lens, H, Hkv, dh, want):
    """Values, and the precision of the first sixteen rows' dQ (see test_short_rows_keep_their_precision), where two groups of sixteen keys or query rows
    belong to a wavefront: groups of heads that divide a tile and groups that do not, blocks of keys in one piece and in several."""
    import torch
    import packedlib as pl
    fwd, keys, cut = pl.blocks(lens, H, Hkv, dh)
    assert (fwd, keys, cut > 0) == want
    print(f"packed attention in blocks of {fwd} rows and {keys} keys, {cut} cut: lens={lens} H={H} Hkv={Hkv} dh={dh}", flush=True)
    qkv, dO = _inputs(lens, H, Hkv, dh, "bf16")
    o, lse, d, ob, db = pl.attention_on("cuda", lens, H, Hkv, dh, qkv, dO, 2.0 ** -8)
    got = [t.double().cpu().numpy() for t in pl.run_attention(lens, "bf16", H, Hkv, dh, qkv, dO)]
    err = np.abs(got[0] - o)
    assert np.all(err <= ob + 1e-30), ("o", float((err / (ob + 1e-30)).max()))
    assert np.abs(got[1] - lse).max() <= 2e-5 * (1 + np.abs(lse).max())
    err = np.abs(got[2] - d)
    assert np.all(err <= db + 1e-30), ("dqkv", float((err / (db + 1e-30)).max()))
    first = np.concatenate([a + np.arange(min(n, 16)) for a, n in zip(pl.offsets(lens), lens)])
    once = torch.from_numpy(d).to(torch.bfloat16).double().numpy()
    a, b = (np.linalg.norm(x[first, :H * dh] - d[first, :H * dh]) for x in (got[2], once))
    assert a <= 1.5 * b, a / b


@pytest.mark.parametrize("dtype,H,Hkv,dh", [("bf16", 4, 2, 64), ("bf16", 8, 8, 64), ("bf16", 5, 1, 128), ("fp32", 4, 2, 32)])
@pytest.mark.parametrize("part", ["q", "k", "v"])
def test_gradients_of_each_part_against_differences(dtype, H, Hkv, dh, part):
    """sum(w * o) of the definition in 64 bits, a step either way in one of q, k and v, against the kernel's gradient along that direction.  The direction
    is near the gradient's own, so that the derivative is large beside what the element-wise bounds allow: a gradient that is zero, half as large or
    of the other sign does not pass.  Differences in 64 bits with a step of 1e-3 of norm 1: their error is of the step's square, 1e-6 of the third
    derivative, which is of the derivative's size."""
    import packedlib as pl
    lens = [40, 1, 77]
    qkv, dO = _inputs(lens, H, Hkv, dh, dtype)
    _, _, d, _, db = pl.attention(lens, H, Hkv, dh, qkv, dO, 2.0 ** -8 if dtype == "bf16" else 1e-5)
    first = {"q": 0, "k": H, "v": H + Hkv}[part]
    cols = slice(first * dh, (first + (H if part == "q" else Hkv)) * dh)
    v = np.zeros_like(d)
    v[:, cols] = d[:, cols] * np.random.default_rng(7).uniform(0.5, 1.5, d[:, cols].shape)
    v /= np.linalg.norm(v)
    t = 1e-3
    f = [float((pl.attention(lens, H, Hkv, dh, qkv.astype(np.float64) + s * t * v, dO, 0.0)[0] * dO).sum()) for s in (1, -1)]
    slope, limit = (f[0] - f[1]) / (2 * t), float((db * np.abs(v)).sum())
    assert limit < slope / 2.5
    got = pl.run_attention(lens, dtype, H, Hkv, dh, qkv, dO)[2].double().cpu().numpy()
    assert abs(slope - (got * v).sum()) <= limit + 1e-5 * slope


@pytest.mark.parametrize("dtype,H,Hkv,dh,ld", [("bf16", 4, 2, 64, 1 << 20), ("bf16", 5, 1, 128, 1 << 20), ("fp32", 4, 2, 64, 1 << 19), ("bf16", 4, 2, 32, 1 << 20)])
def test_rows_beyond_4_gib(dtype, H, Hkv, dh, ld):
    """Buffers whose later sequences lie past 32-bit offsets: the bits of rows side by side."""
    import torch
    import packedlib as pl
    lens = [511] * 5 + [31, 257]                           # (511 + 512) 2^21 bytes: the longest that a stride of 2^20 bf16 elements allows
    print(f"packed attention in rows of {ld} elements {dtype} H={H} Hkv={Hkv} dh={dh}", flush=True)
    qkv, dO = _inputs(lens, H, Hkv, dh, dtype)
    assert sum(lens[:-1]) * ld * (2 if dtype == "bf16" else 4) > 1 << 32
    near = pl.run_attention(lens, dtype, H, Hkv, dh, qkv, dO)
    far = pl.run_attention(lens, dtype, H, Hkv, dh, qkv, dO, pad=ld - (H + 2 * Hkv) * dh, pad_o=ld - H * dh)
    assert all(torch.equal(a, b) for a, b in zip(near, far))
    del far
    torch.cuda.empty_cache()
