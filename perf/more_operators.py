"""The operators of a decoder layer trained in 8-bit floating point, as cases that can be timed and checked.

  linear     a linear layer on 8-bit operands, y = x w^T with dx = dy w and dw = dy^T x: blocks of 128 neighbours along the
             contraction (of the weight 128 x 128) share a power of two, each element keeps eight bits (e4m3, gradients e4m3 or
             e5m2); sums in 32 bits;
  product    its forward product alone for a few rows, with a weight that was laid out once;
  values     a matrix stored in 8 bits, as it is and transposed, and read back;
  residual   what stands between two blocks of a layer: norm of a block's output, dropout, gate, scaled residual sum, norm in front of the
             next block; forward, or forward and backward;
  dropout    alone, with the residual it is added to; the mask comes from a counter (Philox-4x32, 10 rounds) and is never stored;
  rope       rotary positions with several axes (time, height, width) on the query and key heads of packed rows.

`run` computes them with plain torch operations in 32 bits (angles in 64), or (`own`) through the library.  Widths are those of the
repository's workloads (tiny GPT and Llama in fp32; GPT-2 small, Llama 7B and 30B in bf16).
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = 128                                            # neighbours along the contraction that share a power of two
TOP = {"e4m3": 8, "e5m2": 15}                          # the largest value is 1.75 times two to this
MANTISSA = {"e4m3": 3, "e5m2": 2}
LOWEST = {"e4m3": -6, "e5m2": -14}                     # exponent of the smallest normal number
MIN_EXP = -110                                         # smallest power of a block: all values are normal numbers of 32 bits


def _linear(name, dtype, rows, K, N, grad="e4m3"):
    return dict(name=name, kind="linear", dtype=dtype, rows=rows, K=K, N=N, grad=grad)


def _product(name, dtype, rows, K, N):
    return dict(name=name, kind="product", dtype=dtype, rows=rows, K=K, N=N)


def _values(name, dtype, rows, cols, form="e4m3", tiles=False):
    return dict(name=name, kind="values", dtype=dtype, rows=rows, cols=cols, form=form, tiles=tiles)


def _residual(name, dtype, rows, d, rms, post=True, gate="shared", p=0.0, train=True):
    return dict(name=name, kind="residual", dtype=dtype, rows=rows, d=d, rms=rms, post=post, gate=gate, p=p, train=train)


def _dropout(name, dtype, rows, cols, p, resid):
    return dict(name=name, kind="dropout", dtype=dtype, rows=rows, cols=cols, p=p, resid=resid)


def _rope(name, dtype, rows, H, Hkv, dh, sections, own_ladder=False, inverse=False, far=0):
    return dict(name=name, kind="rope", dtype=dtype, rows=rows, H=H, Hkv=Hkv, dh=dh, sections=sections, own_ladder=own_ladder, inverse=inverse, far=far)


def listed():
    return [
        # the gate matrix of Llama 7B on a batch of 8192 tokens: forward, both gradients, the weight stored anew for the step
        _linear("linear_llama_7b_gate", "bf16", 8192, 4096, 11008),
        # the output projection of GPT-2 small's attention on the same batch: few tiles, a long contraction in the weight gradient
        _linear("linear_gpt2_small_proj", "bf16", 8192, 768, 768, "e5m2"),
        # sizes that are no multiple of a block anywhere, fp32 results, gradients with the wider range
        _linear("linear_ragged_fp32", "fp32", 1021, 352, 515, "e5m2"),
        # one answer's next tokens through the head of Llama 7B: the weight's bytes are what counts
        _product("product_few_rows", "bf16", 4, 4096, 32000),
        # a weight of Llama 30B stored for a step, as it is and transposed, and read back
        _values("values_llama_30b_weight", "bf16", 6656, 6656, "e4m3", True),
        # between attention and MLP of Llama 7B with norms on both sides of a block, a gate and dropout
        _residual("residual_llama_7b", "bf16", 8192, 4096, True, p=0.1),
        # the tiny GPT's: the smallest call, layer norms, no norm behind the block
        _residual("residual_tiny", "fp32", 128, 128, False, post=False, gate="none", p=0.1),
        # Llama 30B's width, an odd number of rows, a gate for every row (a projection of the token's own)
        _residual("residual_row_gates", "bf16", 1021, 6656, True, gate="rows"),
        # the embedding's dropout on a batch at Llama 7B's width
        _dropout("dropout_llama_7b", "bf16", 8192, 4096, 0.1, False),
        # the tiny GPT's residual dropout
        _dropout("dropout_tiny", "fp32", 128, 128, 0.1, True),
        # text and images in packed rows at Llama 7B's width with eight key heads, three axes
        _rope("rope_llama_7b_images", "bf16", 8192, 32, 8, 128, "16 24 24"),
        # the gradient of one odd batch at the tiny Llama's heads, far positions, rotation of a part of each head
        _rope("rope_tiny_far", "fp32", 129, 4, 4, 32, "6 4", True, True, 1 << 20),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "product", "values", "residual", "residual", "dropout", "rope"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])

    def size(lo, hi):
        n = _log_uniform(rng, lo, hi)
        return n if rng.random() < 0.5 else max(8, n // 8 * 8)
    if kind == "linear":
        while True:
            S, K, N = size(1, 8192), size(16, 11008), size(16, 11008)
            if S * K * N <= 8192 * 4096 * 11008 // (1 if dtype == "bf16" else 4):
                break
        c = _linear("", dtype, S, K, N, rng.choice(["e4m3", "e4m3", "e5m2"]))
    elif kind == "product":
        while True:
            S, K, N = _log_uniform(rng, 1, 128), size(64, 11008), size(64, 32000)
            if K * N <= 4096 * 32000:
                break
        c = _product("", dtype, S, K, N)
    elif kind == "values":
        while True:
            R, C = size(1, 8192), size(1, 11008)
            if R * C <= 6656 * 6656:
                break
        c = _values("", dtype, R, C, rng.choice(["e4m3", "e5m2"]), rng.random() < 0.5)
    elif kind == "residual":
        while True:
            R, d = _log_uniform(rng, 1, 8192), size(8, 8192)
            if R * d <= 8192 * 4096 // (1 if dtype == "bf16" else 2):
                break
        c = _residual("", dtype, R, d, rng.random() < 0.6, rng.random() < 0.7, rng.choice(["none", "shared", "rows"]), rng.choice([0.0, 0.1, 0.5]),
                      rng.random() < 0.75)
    elif kind == "dropout":
        while True:
            R, C = _log_uniform(rng, 1, 8192), size(1, 11008)
            if R * C <= 8192 * 4096 // (1 if dtype == "bf16" else 2):
                break
        c = _dropout("", dtype, R, C, rng.choice([0.05, 0.1, 0.5]), rng.random() < 0.5)
    else:
        dh, axes = rng.choice([32, 64, 128]), rng.choice([1, 2, 3])
        while True:
            R, Hkv, G = _log_uniform(rng, 1, 8192), _log_uniform(rng, 1, 12), rng.choice([1, 2, 4, 7])
            if R * Hkv * (G + 2) * dh <= 8192 * 48 * 128 // (1 if dtype == "bf16" else 2):
                break
        left, sections = dh // 2, []
        for a in range(axes):
            sections.append(left // (axes - a) if rng.random() < 0.7 else rng.randint(1, left - (axes - a - 1)))
            left -= sections[-1]
        c = _rope("", dtype, R, Hkv * G, Hkv, dh, " ".join(map(str, sections)), rng.random() < 0.5, rng.random() < 0.5, rng.choice([0, 0, 1 << 20]))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _up8(n):
    return (n + 7) // 8 * 8


def _matrix(g, rows, cols, dtype, std=1.0, odd_columns=0.0):
    """Normal values in rows padded to eight elements; `odd_columns`: in a few columns so many times as large."""
    out = torch.zeros((rows, _up8(cols)), device=DEV, dtype=TYPES[dtype])
    v = torch.randn((rows, cols), device=DEV, generator=g) * std
    if odd_columns:
        v[:, torch.randint(0, cols, (max(1, cols // 500),), device=DEV, generator=g)] *= odd_columns
    out[:, :cols] = v.to(out.dtype)
    return out


def _linear_inputs(c, seed):
    """The input a norm's output with a few large columns, the weight, and the gradient of the output, in which rows differ in size."""
    g = _gen(seed)
    x = _matrix(g, c["rows"], c["K"], c["dtype"], 1.0, 30.0)
    w = _matrix(g, c["N"], c["K"], c["dtype"], 0.02)
    if c["kind"] == "product":
        return x, w
    dy = _matrix(g, c["rows"], c["N"], c["dtype"], 1e-3)
    dy *= torch.exp(torch.randn((c["rows"], 1), device=DEV, generator=g)).to(dy.dtype)
    return x, w, dy


def _residual_inputs(c, seed):
    g = _gen(seed)
    R, d, dt = c["rows"], c["d"], c["dtype"]
    t = {"branch": _matrix(g, R, d, dt, 0.5, 8.0), "x": _matrix(g, R, d, dt, 2.0, 4.0)}
    if c["gate"] != "none":
        t["gate"] = (0.5 + 0.1 * _matrix(g, R if c["gate"] == "rows" else 1, d, dt)).to(TYPES[dt])
    names = (["post_gain", "gain"] if c["post"] else ["gain"])
    for n in names:
        t[n] = (1.0 + 0.1 * _matrix(g, 1, d, dt)).to(TYPES[dt])
        if not c["rms"]:
            t[n.replace("gain", "bias")] = _matrix(g, 1, d, dt, 0.1)
    if c["train"]:
        t["dy"], t["dh"] = _matrix(g, R, d, dt, 1e-2), _matrix(g, R, d, dt, 1e-2)
    return t


RESID_SCALE, BRANCH_SCALE, EPS = 0.9375, 0.5, 1e-5


def _seed_of(seed):
    """The key and the place in its sequence that a program hands to dropout at one of its steps."""
    return (seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 63), (seed % 7) * (1 << 33) + seed


def _dropout_inputs(c, seed):
    g = _gen(seed)
    x = _matrix(g, c["rows"], c["cols"], c["dtype"])
    return x, _matrix(g, c["rows"], c["cols"], c["dtype"]) if c["resid"] else None


def _rope_inputs(c, seed):
    """Rows of sequences in which text (the same position on every axis) and images (a grid on the last two) take turns."""
    g = _gen(seed)
    rows, axes = c["rows"], len(c["sections"].split())
    width = (c["H"] + 2 * c["Hkv"]) * c["dh"]
    x = _matrix(g, rows, width, c["dtype"])
    i = torch.arange(rows, device=DEV)
    span = 96 + seed % 64
    at, inside = i // (2 * span), i % (2 * span)
    image = inside >= span
    start = c["far"] + (seed % 1000) * (c["far"] > 0) + at * (span + 16)
    pos = torch.empty((rows, axes), device=DEV, dtype=torch.int64)
    for a in range(axes):
        grid = 0 if axes > 1 and a == 0 else (inside - span) // 12 if a < axes - 1 else (inside - span) % 12
        pos[:, a] = start + torch.where(image, torch.full_like(i, span) + grid, inside)
    return x, pos.to(torch.int32)


# ------------------------------------------------------------------ the plain forms
def _powers(top, form):
    """Exponent of each block from its largest magnitude (fp32): the smallest with all of the block within the type's range."""
    bits = top.view(torch.int32)
    e = (bits >> 23) - 127 - TOP[form] + ((bits & 0x7fffff) > 0x600000).to(torch.int32)
    return e.clamp(min=MIN_EXP)


def _two_to(e):
    return ((e + 127) << 23).view(torch.float32)


def _eight_bits(v, form):
    """The nearest values of the 8-bit type, ties to even; |v| is within its range."""
    e = ((v.abs().view(torch.int32) >> 23) - 127).clamp(min=LOWEST[form]) - MANTISSA[form]
    return torch.round(v * _two_to(-e)) * _two_to(e)


def _stored(x, form, tiles=False):
    """[rows, cols] in 32 bits -> the values that it stands for, in blocks along the columns."""
    rows, n = x.shape
    full = (n + BLOCK - 1) // BLOCK * BLOCK
    b = torch.nn.functional.pad(x, (0, full - n))
    if tiles:
        up = (rows + BLOCK - 1) // BLOCK * BLOCK
        b = torch.nn.functional.pad(b, (0, 0, 0, up - rows)).view(up // BLOCK, BLOCK, full // BLOCK, BLOCK)
        top = b.abs().amax((1, 3), keepdim=True)
    else:
        b = b.view(rows, full // BLOCK, BLOCK)
        top = b.abs().amax(2, keepdim=True)
    e = _powers(top, form)
    v = _eight_bits(b * _two_to(-e), form) * _two_to(e)
    v = torch.where(torch.isfinite(top), v, torch.full_like(v, math.nan))
    return v.reshape(-1, full)[:rows, :n]


def _uniform16(rows, cols, seed, offset):
    """Sixteen bits for each element: Philox-4x32 with ten rounds, one counter for eight neighbours of a row."""
    groups = (cols + 7) // 8
    i = torch.arange(rows * groups, device=DEV, dtype=torch.int64)
    low = 0xffffffff
    c0, c1 = i & low, i >> 32
    c2, c3 = torch.full_like(i, offset & low), torch.full_like(i, offset >> 32 & low)
    k0, k1 = seed & low, seed >> 32 & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57            # mod 2^64; the high half is cut out of it
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack((c0, c1, c2, c3), 1)
    halves = torch.stack((words & 0xffff, words >> 16), 2).to(torch.int32)
    return halves.reshape(rows, groups * 8)[:, :cols]


def _mask(rows, cols, p, seed, offset):
    """Zero where an element is dropped, elsewhere what makes up for those that are."""
    t = round(p * 65536)
    return (_uniform16(rows, cols, seed, offset) >= t).float() * (65536.0 / (65536 - t))


def _plain_linear(s, c):
    x, w, dy = s["x"][:, :c["K"]].float(), s["w"][:, :c["K"]].float(), s["dy"][:, :c["N"]].float()
    dt = s["x"].dtype
    wq = _stored(w, "e4m3", True)
    y = (_stored(x, "e4m3") @ wq.t()).to(dt)
    dx = (_stored(dy, c["grad"]) @ wq).to(dt)
    dw = _stored(dy.t().contiguous(), c["grad"]) @ _stored(x.t().contiguous(), "e4m3").t()
    return {"y": y, "dx": dx, "dw": dw.to(dt)}


def _plain_product(s, c):
    y = _stored(s["x"][:, :c["K"]].float(), "e4m3") @ s["kept"].float().t()
    return {"y": y.to(s["x"].dtype)}


def _plain_values(s, c):
    x = s["x"][:, :c["cols"]].float()
    v = _stored(x, c["form"], c["tiles"])
    vt = v.t() if c["tiles"] else _stored(x.t().contiguous(), c["form"])
    return {"x": v.to(s["x"].dtype), "xt": vt.to(s["x"].dtype)}


def _norm(x, rms):
    mean = 0.0 if rms else x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)
    return (x - mean) * rstd, rstd


def _norm_gradient(g, xh, rstd, rms):
    g = g - xh * (g * xh).mean(1, keepdim=True)
    return (g if rms else g - (g).mean(1, keepdim=True)) * rstd


def _plain_residual(s, c):
    R, d, dt = c["rows"], c["d"], s["x"].dtype
    f = {n: t[:, :d].float() for n, t in s.items() if torch.is_tensor(t) and n in
         ("branch", "x", "gate", "post_gain", "post_bias", "gain", "bias", "dy", "dh")}
    gate = BRANCH_SCALE * f["gate"] if "gate" in f else BRANCH_SCALE
    n = f["branch"]
    if c["post"]:
        bh, post_rstd = _norm(n, c["rms"])
        n = bh * f["post_gain"] + f.get("post_bias", 0.0)
    mask = _mask(R, d, c["p"], s["seed"], s["offset"]) if c["p"] else 1.0
    u = n * mask
    y = RESID_SCALE * f["x"] + gate * u
    yh, rstd = _norm(y, c["rms"])
    out = {"y": y.to(dt), "h": (yh * f["gain"] + f.get("bias", 0.0)).to(dt)}
    if not c["train"]:
        return out
    D = f["dy"] + _norm_gradient(f["dh"] * f["gain"], yh, rstd, c["rms"])
    out["dx"] = (RESID_SCALE * D).to(dt)
    out["dgain"] = (f["dh"] * yh).sum(0).to(dt)
    if not c["rms"]:
        out["dbias"] = f["dh"].sum(0).to(dt)
    if "gate" in f:
        dgate = BRANCH_SCALE * u * D
        out["dgate"] = (dgate if c["gate"] == "rows" else dgate.sum(0)).to(dt)
    dn = gate * mask * D
    if c["post"]:
        out["dpost_gain"] = (dn * bh).sum(0).to(dt)
        if not c["rms"]:
            out["dpost_bias"] = dn.sum(0).to(dt)
        dn = _norm_gradient(dn * f["post_gain"], bh, post_rstd, c["rms"])
    out["dbranch"] = dn.to(dt)
    return out


def _plain_dropout(s, c):
    y = s["x"][:, :c["cols"]].float() * _mask(c["rows"], c["cols"], c["p"], s["seed"], s["offset"])
    if c["resid"]:
        y = y + s["resid"][:, :c["cols"]].float()
    return {"y": y.to(s["x"].dtype)}


def _pairs(c):
    """(axis, exponent of theta) for each rotated pair of a head"""
    out = []
    for a, n in enumerate(int(v) for v in c["sections"].split()):
        for j in range(n):
            out.append((a, -j / n if c["own_ladder"] else -2.0 * len(out) / c["dh"]))
    return out


THETA = 10000.0


def _plain_rope(s, c):
    rows, heads, dh = c["rows"], c["H"] + c["Hkv"], c["dh"]
    pairs = _pairs(c)
    n = len(pairs)
    frequency = THETA ** torch.tensor([e for _, e in pairs], device=DEV, dtype=torch.float64)
    angle = s["pos"][:, [a for a, _ in pairs]].double() * frequency
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if c["inverse"]:
        sin = -sin
    x = s["x"][:, :heads * dh].float().reshape(rows, heads, dh // 2, 2)
    y = x.clone()
    a, b = x[:, :, :n, 0], x[:, :, :n, 1]
    y[:, :, :n, 0] = a * cos - b * sin
    y[:, :, :n, 1] = a * sin + b * cos
    return {"y": y.view(rows, heads * dh).to(s["x"].dtype)}


# ------------------------------------------------------------------ the library's calls
def _bytes(n):
    return torch.empty(n, device=DEV, dtype=torch.uint8)


def _prepare_own(s, c):
    """The buffers that a program keeps from step to step."""
    import paper_2506_06472_amd as tio
    kind = c["kind"]
    if kind in ("linear", "product"):
        S, K, N = c["rows"], c["K"], c["N"]
        s["xq"], s["wq"] = _bytes(tio.tio_fp8_bytes(S, K)), _bytes(tio.tio_fp8_bytes(N, K))
        s["y"] = torch.empty((S, _up8(N)), device=DEV, dtype=s["x"].dtype)
        work = tio.tio_op_gemm_fp8_work(S, N, K)
        if kind == "linear":
            s["xt"], s["wt"] = _bytes(tio.tio_fp8_bytes(K, S)), _bytes(tio.tio_fp8_bytes(K, N))
            s["dyq"], s["dyt"] = _bytes(tio.tio_fp8_bytes(S, N)), _bytes(tio.tio_fp8_bytes(N, S))
            s["dx"], s["dw"] = torch.empty_like(s["x"]), torch.empty_like(s["w"])
            work = max(work, tio.tio_op_gemm_fp8_work(S, K, N), tio.tio_op_gemm_fp8_work(N, K, S))
        s["work"] = _bytes(work)
        if kind == "product":
            stream = torch.cuda.current_stream().cuda_stream
            tio.tio_op_fp8_store(stream, c["dtype"], "e4m3", True, N, K, s["w"].data_ptr(), s["w"].stride(0), s["wq"].data_ptr())
            del s["w"]
    elif kind == "values":
        R, C = c["rows"], c["cols"]
        s["q"], s["qt"] = _bytes(tio.tio_fp8_bytes(R, C)), _bytes(tio.tio_fp8_bytes(C, R))
        s["v"] = torch.empty_like(s["x"])
        s["vt"] = torch.empty((C, _up8(R)), device=DEV, dtype=s["x"].dtype)
    elif kind == "residual":
        s["cfg"] = tio.tio_residual_cfg(c["rms"], EPS, RESID_SCALE, BRANCH_SCALE, c["p"], s["seed"], s["offset"])
        s["y"], s["h"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        s["stats"] = torch.empty((c["rows"], 4), device=DEV)
        if c["train"]:
            for n in ("x", "branch", "gate", "post_gain", "post_bias", "gain", "bias"):
                if n in s:
                    s["d" + n] = torch.empty_like(s[n])
            s["work"] = _bytes(tio.tio_op_residual_norm_bwd_work(c["rows"], c["d"]))
    elif kind == "dropout":
        s["y"] = torch.empty_like(s["x"])
    else:
        s["y"] = torch.empty((c["rows"], (c["H"] + c["Hkv"]) * c["dh"]), device=DEV, dtype=s["x"].dtype)


def _own_linear(s, c, tio, stream, at):
    S, K, N, dt, grad = c["rows"], c["K"], c["N"], c["dtype"], c["grad"]
    ldk, ldn, work = s["x"].stride(0), s["dy"].stride(0), at("work")
    tio.tio_op_fp8_store(stream, dt, "e4m3", True, N, K, at("w"), ldk, at("wq"), at("wt"))
    tio.tio_op_fp8_store(stream, dt, "e4m3", False, S, K, at("x"), ldk, at("xq"), at("xt"))
    tio.tio_op_gemm_fp8(stream, dt, S, N, K, "e4m3", at("xq"), "e4m3", at("wq"), at("y"), ldn, work_ptr=work)
    tio.tio_op_fp8_store(stream, dt, grad, False, S, N, at("dy"), ldn, at("dyq"), at("dyt"))
    tio.tio_op_gemm_fp8(stream, dt, S, K, N, grad, at("dyq"), "e4m3", at("wt"), at("dx"), ldk, work_ptr=work)
    tio.tio_op_gemm_fp8(stream, dt, N, K, S, grad, at("dyt"), "e4m3", at("xt"), at("dw"), ldk, work_ptr=work)
    return {"y": s["y"][:, :N], "dx": s["dx"][:, :K], "dw": s["dw"][:, :K]}


def _own_product(s, c, tio, stream, at):
    S, K, N, dt = c["rows"], c["K"], c["N"], c["dtype"]
    tio.tio_op_fp8_store(stream, dt, "e4m3", False, S, K, at("x"), s["x"].stride(0), at("xq"))
    tio.tio_op_gemm_fp8(stream, dt, S, N, K, "e4m3", at("xq"), "e4m3", at("wq"), at("y"), s["y"].stride(0), work_ptr=at("work"))
    return {"y": s["y"][:, :N]}


def _own_values(s, c, tio, stream, at):
    R, C, dt, form = c["rows"], c["cols"], c["dtype"], c["form"]
    tio.tio_op_fp8_store(stream, dt, form, c["tiles"], R, C, at("x"), s["x"].stride(0), at("q"), at("qt"))
    tio.tio_op_fp8_load(stream, dt, form, R, C, at("q"), at("v"), s["v"].stride(0))
    tio.tio_op_fp8_load(stream, dt, form, C, R, at("qt"), at("vt"), s["vt"].stride(0))
    return {"x": s["v"][:, :C], "xt": s["vt"][:, :R]}


def _own_residual(s, c, tio, stream, at):
    R, d, dt, ld = c["rows"], c["d"], c["dtype"], s["x"].stride(0)
    ldg = s["gate"].stride(0) if c["gate"] == "rows" else 0
    tio.tio_op_residual_norm(stream, dt, s["cfg"], R, d, ld, at("branch"), at("x"), at("gate"), ldg, at("post_gain"), at("post_bias"), at("gain"),
                             at("bias"), at("y"), at("h"), at("stats"))
    out = {"y": s["y"][:, :d], "h": s["h"][:, :d]}
    if c["train"]:
        tio.tio_op_residual_norm_bwd_from_x(stream, dt, s["cfg"], R, d, ld, at("branch"), at("x"), at("gate"), ldg, at("post_gain"), at("post_bias"),
                                            at("gain"), at("stats"), at("dy"), at("dh"), at("dx"), at("dbranch"), at("dgate"), at("dpost_gain"),
                                            at("dpost_bias"), at("dgain"), at("dbias"), at("work"))
        for n in ("x", "branch", "gate", "post_gain", "post_bias", "gain", "bias"):
            if n in s:
                t = s["d" + n][:, :d]
                out["d" + n] = t if n in ("x", "branch") or (n == "gate" and ldg) else t[0]
    return out


def _own_dropout(s, c, tio, stream, at):
    ld = s["x"].stride(0)
    tio.tio_op_dropout(stream, c["dtype"], c["rows"], c["cols"], at("x"), ld, at("resid"), ld, at("y"), ld, c["p"], s["seed"], s["offset"])
    return {"y": s["y"][:, :c["cols"]]}


def _own_rope(s, c, tio, stream, at):
    tio.tio_op_rope_axes(stream, c["dtype"], c["rows"], c["H"] + c["Hkv"], c["dh"], at("x"), s["x"].stride(0), at("y"), s["y"].stride(0),
                         at("pos"), s["sections"], THETA, c["own_ladder"], c["inverse"])
    return {"y": s["y"]}


def prepare(case, seed):
    c, kind = case, case["kind"]
    s = {}
    if kind in ("linear", "product"):
        s.update(zip(("x", "w", "dy"), _linear_inputs(c, seed)))
        if kind == "product" and not own:
            s["kept"] = _stored(s.pop("w")[:, :c["K"]].float(), "e4m3", True).bfloat16()       # four significant bits: exact
    elif kind == "values":
        s["x"] = _matrix(_gen(seed), c["rows"], c["cols"], c["dtype"], 0.02, 20.0)
    elif kind == "residual":
        s.update(_residual_inputs(c, seed))
    elif kind == "dropout":
        s["x"], resid = _dropout_inputs(c, seed)
        if resid is not None:
            s["resid"] = resid
    else:
        s["x"], s["pos"] = _rope_inputs(c, seed)
        s["sections"] = [int(v) for v in c["sections"].split()]
    if kind in ("residual", "dropout"):
        s["seed"], s["offset"] = _seed_of(seed)
    if own:
        _prepare_own(s, c)
        s["at"] = {n: t.data_ptr() for n, t in s.items() if torch.is_tensor(t)}              # addresses, 0 for what there is none of
    return case, s


def run(state):
    c, s = state
    if not own:
        return {"linear": _plain_linear, "product": _plain_product, "values": _plain_values, "residual": _plain_residual, "dropout": _plain_dropout,
                "rope": _plain_rope}[c["kind"]](s, c)
    import paper_2506_06472_amd as tio
    addresses = s["at"]
    return {"linear": _own_linear, "product": _own_product, "values": _own_values, "residual": _own_residual, "dropout": _own_dropout,
            "rope": _own_rope}[c["kind"]](s, c, tio, torch.cuda.current_stream().cuda_stream, lambda n: addresses.get(n, 0))


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, kind = case, case["kind"]
    e = 2 if c["dtype"] == "bf16" else 4
    R = c["rows"]
    if kind == "linear":
        K, N = c["K"], c["N"]
        return {"bytes": 2 * (R * K + N * K + R * N) * e, "flops": 6.0 * R * K * N}
    if kind == "product":
        K, N = c["K"], c["N"]
        return {"bytes": R * K * e + N * K + (N + BLOCK - 1) // BLOCK * ((K + BLOCK - 1) // BLOCK) + R * N * e, "flops": 2.0 * R * K * N}
    if kind == "values":
        n = R * c["cols"]
        return {"bytes": 3 * n * e + 4 * n, "flops": 4.0 * n}                      # both forms written, and read back
    if kind == "residual":
        n, d = R * c["d"], c["d"]
        rows_gate = n if c["gate"] == "rows" else 0
        moved = 4 * n + rows_gate
        if c["train"]:
            moved += 6 * n + 2 * rows_gate
        return {"bytes": moved * e + 8 * d * e, "flops": (60.0 if c["train"] else 20.0) * n}
    if kind == "dropout":
        n = R * c["cols"]
        return {"bytes": n * (3 if c["resid"] else 2) * e, "flops": 3.0 * n}
    n = R * (c["H"] + c["Hkv"]) * c["dh"]
    return {"bytes": 2 * n * e + R * 4 * len(c["sections"].split()), "flops": 3.0 * n}


# ------------------------------------------------------------------ the same in 64 bits
def _exact_stored(x, form, tiles=False):
    """x: [rows, cols] in 64 bits, blocks along the columns."""
    eight = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}[form]
    rows, cols = x.shape
    high = BLOCK if tiles else 1
    top = x.abs()
    top = torch.nn.functional.max_pool2d(top[None, None], (high, BLOCK), ceil_mode=True)[0, 0]
    fraction, exponent = torch.frexp(top / 1.75)
    power = exponent.double() - (fraction == 0.5).double() - {"e4m3": 8, "e5m2": 15}[form]       # ceil(log2(top / largest))
    power = torch.where(top == 0, torch.full_like(power, MIN_EXP), power).clamp(min=MIN_EXP)
    unit = torch.exp2(power).repeat_interleave(high, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]
    return (x / unit).float().to(eight).double() * unit


def _exact_linear(c, seed):
    inputs = _linear_inputs(c, seed)
    x, w = (t[:, :c["K"]].double() for t in inputs[:2])
    xq, wq = _exact_stored(x, "e4m3"), _exact_stored(w, "e4m3", True)
    out = {"y": torch.nn.functional.linear(xq, wq)}
    if c["kind"] == "product":
        return out
    del xq
    dy = inputs[2][:, :c["N"]].double()
    out["dx"] = torch.mm(_exact_stored(dy, c["grad"]), wq)
    out["dw"] = torch.nn.functional.linear(_exact_stored(dy.t().contiguous(), c["grad"]), _exact_stored(x.t().contiguous(), "e4m3"))
    return out


def _exact_values(c, seed):
    x = _matrix(_gen(seed), c["rows"], c["cols"], c["dtype"], 0.02, 20.0)[:, :c["cols"]].double()
    return {"x": _exact_stored(x, c["form"], c["tiles"]), "xt": _exact_stored(x.t().contiguous(), c["form"], c["tiles"])}


def _exact_keep(rows, cols, p, seed, offset):
    """Philox with products from halves of sixteen bits."""
    m32 = (1 << 32) - 1

    def product(a, m):                                         # (high, low) words of a 32-bit word times a constant
        al, ah, ml, mh = a & 0xffff, a >> 16, m & 0xffff, m >> 16
        low = al * ml
        mid = ah * ml + (low >> 16)
        mid2 = al * mh + (mid & 0xffff)
        return ah * mh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xffff) << 16) | (low & 0xffff)
    groups = -(-cols // 8)
    number = torch.arange(rows, device=DEV)[:, None] * groups + torch.arange(groups, device=DEV)[None, :]
    ctr = [number % (1 << 32), number // (1 << 32), torch.full_like(number, offset % (1 << 32)), torch.full_like(number, offset // (1 << 32))]
    key = [seed % (1 << 32), seed // (1 << 32)]
    for r in range(10):
        (h0, l0), (h1, l1) = product(ctr[0], 0xD2511F53), product(ctr[2], 0xCD9E8D57)
        bump = [(key[0] + r * 0x9E3779B9) & m32, (key[1] + r * 0xBB67AE85) & m32]
        ctr = [h1 ^ ctr[1] ^ bump[0], l1, h0 ^ ctr[3] ^ bump[1], l0]
    bits = torch.empty((rows, groups, 8), device=DEV, dtype=torch.int64)
    for j in range(8):
        bits[:, :, j] = (ctr[j // 2] >> (16 * (j % 2))) % 65536
    limit = int(round(p * 65536))
    return (bits.flatten(1)[:, :cols] >= limit).double() / (1.0 - limit / 65536)


def _exact_residual(c, seed):
    t = {n: v[:, :c["d"]].double() for n, v in _residual_inputs(c, seed).items()}
    leaves = [n for n in ("x", "branch", "gate", "post_gain", "post_bias", "gain", "bias") if n in t]
    for n in leaves:
        t[n].requires_grad_(c["train"])

    def normed(v, gain, bias):
        if not c["rms"]:
            return torch.nn.functional.layer_norm(v, (c["d"],), t[gain][0], t[bias][0], EPS)
        return v * torch.rsqrt(v.square().mean(1, keepdim=True) + EPS) * t[gain]
    n = normed(t["branch"], "post_gain", "post_bias") if c["post"] else t["branch"]
    if c["p"]:
        n = n * _exact_keep(c["rows"], c["d"], c["p"], *_seed_of(seed))
    y = RESID_SCALE * t["x"] + BRANCH_SCALE * n * t.get("gate", 1.0)
    h = normed(y, "gain", "bias")
    out = {"y": y.detach(), "h": h.detach()}
    if c["train"]:
        grads = torch.autograd.grad((y, h), [t[n] for n in leaves], (t["dy"], t["dh"]))
        for name, g in zip(leaves, grads):
            whole = name in ("x", "branch") or (name == "gate" and c["gate"] == "rows")
            out["d" + name] = g if whole else g[0]
    return out


def _exact_dropout(c, seed):
    x, resid = _dropout_inputs(c, seed)
    y = x[:, :c["cols"]].double() * _exact_keep(c["rows"], c["cols"], c["p"], *_seed_of(seed))
    return {"y": y if resid is None else resid[:, :c["cols"]].double() + y}


def _exact_rope(c, seed):
    x, pos = _rope_inputs(c, seed)
    heads, dh = c["H"] + c["Hkv"], c["dh"]
    z = torch.view_as_complex(x[:, :heads * dh].double().reshape(c["rows"], heads, dh // 2, 2).contiguous()).clone()
    pair = 0
    for axis, count in enumerate(c["sections"].split()):
        for j in range(int(count)):
            frequency = THETA ** (-j / int(count) if c["own_ladder"] else -2.0 * pair / dh)
            turn = pos[:, axis].double() * frequency * (-1.0 if c["inverse"] else 1.0)
            z[:, :, pair] *= torch.polar(torch.ones_like(turn), turn)[:, None]
            pair += 1
    return {"y": torch.view_as_real(z).reshape(c["rows"], heads * dh)}


def exact(case, seed):
    """What `run` returns, from the definitions in 64 bits."""
    return {"linear": _exact_linear, "product": _exact_linear, "values": _exact_values, "residual": _exact_residual, "dropout": _exact_dropout,
            "rope": _exact_rope}[case["kind"]](case, seed)
