"""GPU: the paired preference loss on packed logits, and its gradient, against the definition in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _definition(lens, logits, labels, ref, beta, s, total):
    """seq, losses, loss, dlogits"""
    V = logits.shape[1]
    x = logits.astype(np.float64)
    with np.errstate(all="ignore"):
        m = x.max(1, keepdims=True)
        lse = (m + np.log(np.exp(x - m).sum(1, keepdims=True)))[:, 0]
    ok = (labels >= 0) & (labels < V)
    rows = np.arange(len(x))
    lp = np.where(ok, x[rows, np.where(ok, labels, 0)] - np.where(ok, lse, 0), 0.0)
    off = np.concatenate([[0], np.cumsum(lens)])
    seq = np.array([lp[a:b].sum() for a, b in zip(off, off[1:])])
    h = seq - ref.astype(np.float64)
    z = np.float64(np.float32(beta)) * (h[0::2] - h[1::2])
    s = np.float64(np.float32(s))
    ls = lambda t: np.minimum(t, 0) - np.log1p(np.exp(-np.abs(t)))
    losses = -(1 - s) * ls(z) - s * ls(-z)
    w = -np.float64(np.float32(beta)) / total * ((1 - s) * np.exp(ls(-z)) - s * np.exp(ls(z)))
    w = np.repeat(np.stack([w, -w], 1).reshape(-1), lens) * ok
    p = np.exp(x - lse[:, None], where=ok[:, None], out=np.zeros_like(x))
    d = -w[:, None] * p
    d[rows[ok], labels[ok]] += w[ok]
    return seq, losses, losses.sum() / total, d, w, p


def _run(lens, dtype, logits, labels, ref, beta, s, V, grad="apart", extra_rows=2, pad=0, total=0, stream=None):
    import torch
    import paper_2506_06472_amd as tio
    import packedlib as pl
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    p, dev = pl.packing(lens)
    c = 8 if dtype == "bf16" else 4
    up = (V + c - 1) // c * c
    rows = int(np.sum(lens))
    x = torch.full((rows + extra_rows, up + pad), float("nan"), device="cuda", dtype=t)
    x[:rows, :V] = torch.from_numpy(logits).cuda().to(t)
    d = x if grad == "in place" else torch.full_like(x, 7.0)
    before = x.clone()
    y = torch.from_numpy(labels.astype(np.int32)).cuda()
    r = torch.from_numpy(ref.astype(np.float32)).cuda()
    need = tio.tio_op_preference_loss_work(p)
    work = torch.full((need + 64,), 255, device="cuda", dtype=torch.uint8)
    seq, losses, loss = (torch.full((n + 4,), 7.0, device="cuda") for n in (len(lens), len(lens) // 2, 1))
    torch.cuda.synchronize()
    tio.tio_op_preference_loss(stream or 0, dtype, p, dev.data_ptr(), V, x.data_ptr(), x.stride(0), y.data_ptr(), r.data_ptr(), beta, s, seq.data_ptr(),
                               losses.data_ptr(), loss.data_ptr(), work.data_ptr(), d.data_ptr() if grad else 0, total)
    torch.cuda.synchronize()
    assert (work[need:] == 255).all() and (seq[len(lens):] == 7).all() and (losses[len(lens) // 2:] == 7).all() and (loss[1:] == 7).all()
    same = lambda a, b: torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0))
    if grad == "in place":
        assert same(x[rows:], before[rows:]) and same(x[:, up:], before[:, up:])
    else:
        assert same(x, before) and (d[rows:] == 7.0).all() and (d[:, up:] == 7.0).all()
    if grad:
        assert (d[:rows, V:up] == 0).all()
    else:
        assert (d == 7.0).all()
    return seq[:len(lens)], losses[:len(lens) // 2], loss[:1], d[:rows, :V]


def _inputs(lens, V, dtype, masked, seed=0, scale=2.0):
    from synth import to_bf16_round
    rng = np.random.default_rng(sum(lens) + V + seed)
    rows = sum(lens)
    x = (rng.standard_normal((rows, V)) * scale).astype(np.float32)
    y = rng.integers(0, V, rows)
    x[np.arange(rows), y] += 4.0
    if dtype == "bf16":
        x = to_bf16_round(x)
    y = np.where(rng.random(rows) < masked, -100, y)
    lp = np.log(V) * np.array(lens)
    return x, y, (-0.6 * lp + rng.standard_normal(len(lens)) * 5).astype(np.float32)


def _check(lens, V, dtype, masked=0.3, beta=0.1, s=0.0, total=0, grad="apart", **more):
    print(f"preference {dtype} lens={lens} V={V} beta={beta} smoothing={s} {grad} {more}", flush=True)
    x, y, ref = _inputs(lens, V, dtype, masked, **{k: more.pop(k) for k in ("scale", "seed") if k in more})
    seq, losses, loss, d, w, p = _definition(lens, x, y, ref, beta, s, total or len(lens) // 2)
    got = _run(lens, dtype, x, y, ref, beta, s, V, grad, total=total, **more)
    # of a row's log-sum-exp: exponentials (two roundings and 2^-23 of the exponent, which p weights down to log V), a sum of up to 64 terms in a
    # thread and a tree, and the logarithm: less than 2^-16; of a sequence's sum as much for each row, and its own rounding
    row = 2.0 ** -17 * (1 + np.abs(x).max(initial=0.0) / 30)
    of_seq = row * np.array(lens)
    assert np.all(np.abs(got[0].double().cpu().numpy() - seq) <= of_seq + 2.0 ** -24 * np.abs(seq))
    of_z = beta * of_seq.reshape(-1, 2).sum(1)
    # a loss of z in 32 bits: z's rounding, 2^-24 |z|, which the loss passes on with a factor of at most 1; and relative to the loss, whose terms all have
    # one sign, the exponential (2 ulp, 2^-22, which log1p passes on with at most 1), log1p (2 ulp, 2^-22), and at 2^-24 each log1p + z, 1 - s, a product,
    # the sum: 2^-22 + 2^-22 + 4 2^-24 < 2^-20.  Where the rows' part is zero (two empty sequences) nothing else would count these.
    h = seq - ref.astype(np.float64)
    of_loss = 2.0 ** -24 * np.abs(beta * (h[0::2] - h[1::2])) + 2.0 ** -20 * np.abs(losses)
    assert np.all(np.abs(got[1].double().cpu().numpy() - losses) <= of_z + of_loss + 1e-12)
    assert abs(got[2].item() - loss) <= of_z.mean() + 2.0 ** -20 * abs(loss)
    if grad:
        half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
        rel = np.repeat(np.repeat(of_z, 2), lens)[:, None] + 4 * row             # of the weight and of the probabilities
        onehot = np.zeros_like(p)
        ok = (y >= 0) & (y < V)
        onehot[np.arange(len(y))[ok], y[ok]] = 1
        lim = half * np.abs(d) + rel * np.abs(w)[:, None] * (p + onehot) + 2.0 ** -126
        err = np.abs(got[3].double().cpu().numpy() - d)
        assert np.all(err <= lim), float((err / lim).max())
        assert (got[3][~ok] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 500, 1024, 1025, 2047, 2056, 8191, 8200, 16391])
def test_vocabularies(dtype, V):
    _check([5, 9, 0, 3], V, dtype)


@pytest.mark.parametrize("dtype,V", [("bf16", 50257), ("bf16", 32000), ("bf16", 70001), ("fp32", 50257)])
def test_large_vocabularies(dtype, V):
    _check([9, 17, 1, 2], V, dtype, s=0.1)


@pytest.mark.parametrize("lens", [[1, 1], [0, 0], [0, 5], [7, 0, 300, 2], [1000, 513], list(range(64)), [3, 3] * 70])
@pytest.mark.parametrize("masked", [0.0, 0.5, 1.0])
def test_lengths_and_prompts(lens, masked):
    _check(lens, 300, "bf16", masked)


@pytest.mark.parametrize("lens,V", [([20] * 16, 300), ([20] * 18, 300), ([1024, 1024], 40), ([1024, 1025], 40), ([2000, 10, 1000, 1086], 40),
                                    ([2000, 10, 1000, 1087], 40), ([500, 525, 512, 511], 2049), ([500, 525, 512, 512], 2049), ([0, 0, 0, 1, 4095, 0], 16)])
@pytest.mark.parametrize("grad", [None, "apart", "in place"])
def test_batches_of_every_size(lens, V, grad):
    """At the numbers of pairs, rows, rows to a pair and chunks where the launches change."""
    _check(lens, V, "bf16", grad=grad, s=0.1, pad=8)


@pytest.mark.parametrize("beta,s", [(0.01, 0.0), (0.5, 0.2), (2.0, 1.0), (5.0, 0.5)])
def test_betas_and_smoothing(beta, s):
    _check([40, 33, 8, 50], 777, "fp32", beta=beta, s=s)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("grad", [None, "apart", "in place"])
@pytest.mark.parametrize("pad", [0, 16])
def test_forms(dtype, grad, pad):
    """Loss alone, gradients in a buffer of their own and over the logits; rows wider than the vocabulary; a part of a larger batch."""
    _check([33, 20, 5, 60], 1003, dtype, grad=grad, pad=pad, total=5)


def test_masked_vocabulary_and_unknown_labels():
    """Logits of -inf have probability and gradient zero; labels past the vocabulary count as a prompt's."""
    lens, V = [6, 4], 900
    x, y, ref = _inputs(lens, V, "fp32", 0.0)
    x[:, ::3] = -np.inf
    x[np.arange(10), y] = 1.0
    x[2, :] = -np.inf
    x[2, y[2]] = -3.0                                      # one possible token: log p = 0
    y[4], y[7] = V, 2 ** 31 - 1
    for dtype in ("bf16", "fp32"):
        if dtype == "bf16":
            from synth import to_bf16_round
            fine = np.isfinite(x)
            x = np.where(fine, to_bf16_round(np.where(fine, x, 0)), x)
        seq, losses, loss, d, w, p = _definition(lens, x, y, ref, 0.1, 0.0, 1)
        got = _run(lens, dtype, x, y, ref, 0.1, 0.0, V)
        assert np.allclose(got[0].cpu().numpy(), seq, rtol=1e-5, atol=1e-4) and np.allclose(got[1].cpu().numpy(), losses, rtol=1e-4)
        g = got[3].double().cpu().numpy()
        assert np.all(np.abs(g - d) <= 2.0 ** -8 * np.abs(d) + 1e-4 * np.abs(w)[:, None] * (p + 1e-3))
        assert np.all(g[:, ::3][x[:, ::3] == -np.inf] == 0) and np.all(g[[4, 7]] == 0)


def test_nothing_possible_and_nan_stay_in_their_pair():
    """A row of -inf, and one with a NaN, make their own pair's sums and gradients NaN and nobody else's."""
    lens, V = [3, 2, 4, 4], 100
    x, y, ref = _inputs(lens, V, "fp32", 0.0)
    x[1] = -np.inf
    got = [t.cpu().numpy() for t in _run(lens, "fp32", x, y, ref, 0.1, 0.0, V)]
    assert np.isnan(got[0][0]) and np.isfinite(got[0][1:]).all() and np.isnan(got[1][0]) and np.isfinite(got[1][1]) and np.isnan(got[2][0])
    assert np.isnan(got[3][:5]).any() and np.isfinite(got[3][5:]).all()
    x[1], x[1, 50] = 0.0, np.nan
    got = [t.cpu().numpy() for t in _run(lens, "fp32", x, y, ref, 0.1, 0.0, V)]
    assert np.isnan(got[0][0]) and np.isfinite(got[0][1:]).all() and np.isfinite(got[3][5:]).all()


def test_gradient_against_differences():
    lens, V = [12, 9, 30, 1], 64
    x, y, ref = _inputs(lens, V, "fp32", 0.2)
    v = np.random.default_rng(1).standard_normal(x.shape)
    t = 1e-5
    f = [_definition(lens, x.astype(np.float64) + a * t * v, y, ref, 0.3, 0.1, 2)[2] for a in (1, -1)]
    d = _run(lens, "fp32", x, y, ref, 0.3, 0.1, V)[3].double().cpu().numpy()
    assert abs((f[0] - f[1]) / (2 * t) - (d * v).sum()) <= 1e-5 * np.abs(d * v).sum() + 1e-8


def test_very_large_logits():
    """A common offset of 1e4 in every logit: probabilities do not lose what the offset costs (fp32)."""
    lens, V = [10, 12], 400
    x, y, ref = _inputs(lens, V, "fp32", 0.0)
    x = np.round(x * 8) / 8                                # exact with the offset too
    a = _run(lens, "fp32", x.astype(np.float32), y, ref, 0.1, 0.0, V)
    b = _run(lens, "fp32", (x + 10240.0).astype(np.float32), y, ref, 0.1, 0.0, V)
    for p, q in zip(a, b):
        assert ((p - q).abs() <= 1e-5 * q.abs() + 1e-8).all()


@pytest.mark.parametrize("lens", [[70, 65, 3, 128], [70, 65, 3, 128] * 5], ids=["few", "many"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_captured_and_replayed(dtype, lens):
    import torch
    import paper_2506_06472_amd as tio
    import packedlib as pl
    V, n = 3000, len(lens)
    p, dev = pl.packing(lens)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.zeros((sum(lens), V), device="cuda", dtype=t)
    d = torch.zeros_like(x)
    y = torch.zeros(sum(lens), device="cuda", dtype=torch.int32)
    r, seq = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    losses, loss = torch.zeros(n // 2, device="cuda"), torch.zeros(1, device="cuda")
    work = torch.zeros(tio.tio_op_preference_loss_work(p), device="cuda", dtype=torch.uint8)

    def call(stream):
        tio.tio_op_preference_loss(stream, dtype, p, dev.data_ptr(), V, x.data_ptr(), V, y.data_ptr(), r.data_ptr(), 0.1, 0.0, seq.data_ptr(),
                                   losses.data_ptr(), loss.data_ptr(), work.data_ptr(), d.data_ptr())
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(s.cuda_stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(torch.cuda.current_stream().cuda_stream)
    for seed in range(3):
        a, b, c = _inputs(lens, V, dtype, 0.3, seed=seed)
        x.copy_(torch.from_numpy(a))
        y.copy_(torch.from_numpy(b.astype(np.int32)))
        r.copy_(torch.from_numpy(c))
        graph.replay()
        torch.cuda.synchronize()
        eager = _run(lens, dtype, a, b, c, 0.1, 0.0, V)
        for name, u, v in zip(("seq", "losses", "loss", "dlogits"), (seq, losses, loss, d), eager):
            assert torch.equal(u, v), (seed, name)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V,masked", [(300, slice(100, 251)), (64, slice(0, 64)), (9000, slice(0, 8200)), (50257, slice(300, 50257))])
@pytest.mark.parametrize("lens", [[4, 5, 3, 2], [4, 5, 3, 2] * 5], ids=["few", "many"])
def test_logits_of_the_types_lowest_and_largest_value(dtype, V, masked, lens):
    """Tokens taken out with the type's lowest value, all of a row's too, and the largest value, which times log2(e) are beyond 32 bits."""
    import torch
    print(f"preference, lowest and largest values {dtype} V={V} masked={masked} {len(lens)} sequences", flush=True)
    x, y, ref = _inputs(lens, V, dtype, 0.0)
    low = np.float32(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    x[:, masked] = low
    x[1] = low                                             # every token as likely as every other
    x[2] = low
    x[2, :3] = [1.0, 2.0, 3.0]
    y[2] = 1
    x[5, :] = 0.0                                          # one token certain
    x[5, 7] = -low
    y[5] = 7
    x[6, :] = low                                          # the same beside the lowest
    x[6, 9] = -low
    y[6] = 9
    x[10, :] = 0.5 * low                                   # the row's largest is near the end of the range, and not alone
    x[10, ::2] = 0.75 * low
    y[10] = 11
    at = np.arange(len(y))
    assert x.shape[1] == V and (np.isfinite(x)).all()
    keep = np.isin(at, (1, 2, 5, 6, 10))
    x[~keep, y[~keep]] = 2.0                               # the label is possible
    # the definition of logits less their row's largest, which is the same: of -3.4e38 + log V 64 bits lose log V
    shifted = x.astype(np.float64) - x.max(1, keepdims=True).astype(np.float64)
    seq, losses, loss, d, w, p = _definition(lens, shifted, y, ref, 0.1, 0.1, len(lens) // 2)
    assert np.isfinite(seq).all() and np.isfinite(d).all()
    got = [t.double().cpu().numpy() for t in _run(lens, dtype, x, y, ref, 0.1, 0.1, V)]
    # the bounds of _check, where no row's largest logit is more than a few apart from those that count
    row = 2.0 ** -17 * 2
    of_seq = row * np.array(lens)
    assert np.all(np.abs(got[0] - seq) <= of_seq + 2.0 ** -24 * np.abs(seq))
    of_z = 0.1 * of_seq.reshape(-1, 2).sum(1)
    h = seq - ref.astype(np.float64)
    of_loss = 2.0 ** -24 * np.abs(0.1 * (h[0::2] - h[1::2])) + 2.0 ** -20 * np.abs(losses)
    assert np.all(np.abs(got[1] - losses) <= of_z + of_loss + 1e-12)
    assert abs(got[2][0] - loss) <= of_z.mean() + 2.0 ** -20 * abs(loss)
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    onehot = np.zeros_like(p)
    onehot[at, y] = 1
    lim = half * np.abs(d) + (np.repeat(np.repeat(of_z, 2), lens)[:, None] + 4 * row) * np.abs(w)[:, None] * (p + onehot) + 2.0 ** -126
    assert np.all(np.abs(got[3] - d) <= lim)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_label_of_the_types_lowest_value(dtype):
    """The label of a preferred answer's row is as good as impossible: its pair's loss is -beta times the lowest value, nobody else's."""
    import torch
    lens, V = [2, 3, 2, 2], 100
    x, y, ref = _inputs(lens, V, dtype, 0.0)
    low = torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min
    x[1, y[1]] = low
    seq, losses, loss, d, _, _ = _definition(lens, x, y, ref, 0.1, 0.0, 2)
    got = [t.double().cpu().numpy() for t in _run(lens, dtype, x, y, ref, 0.1, 0.0, V)]
    for g, want in zip(got, (seq, losses, np.array([loss]), d)):
        assert np.isfinite(g).all() and np.all(np.abs(g - want) <= 2.0 ** -8 * np.abs(want) + 1e-4)


@pytest.mark.parametrize("dtype,lens,V", [("bf16", [40000, 30000, 5, 3], 40), ("fp32", [65535, 1, 65536, 2], 17), ("bf16", [1, 2] * 6000, 24)])
@pytest.mark.parametrize("grad", ["apart", "in place"])
def test_more_rows_than_a_launch_of_the_gradient(dtype, lens, V, grad):
    """Rows past 65535, whose gradient takes several launches, and thousands of pairs."""
    _check(lens, V, dtype, grad=grad, s=0.1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("lens", [[40, 33, 5, 20], [1200, 700, 300, 200, 3, 1]], ids=["few", "many"])
def test_rows_beyond_4_gib(dtype, lens):
    """Strides that take the later rows past 32-bit offsets: the bits of rows side by side."""
    import torch
    V, rows = 4100, sum(lens)
    x, y, ref = _inputs(lens, V, dtype, 0.3)
    near = _run(lens, dtype, x, y, ref, 0.1, 0.1, V)
    ld = (5 << 30) // (rows * (2 if dtype == "bf16" else 4)) // 8 * 8
    far = _run(lens, dtype, x, y, ref, 0.1, 0.1, V, pad=ld - (V + 7) // 8 * 8)
    assert all(torch.equal(a, b) for a, b in zip(near, far))
    del far
    torch.cuda.empty_cache()
