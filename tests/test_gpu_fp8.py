"""GPU: matrices stored in 8-bit floating point with a power of two per block of 128, and their products, against the definition in 64 bits."""
import numpy as np
import pytest

import layer8lib as l8

pytestmark = pytest.mark.gpu


def _values(rows, cols, dtype, seed=0):
    rng = np.random.default_rng(rows * 1000 + cols + seed)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 7, (rows, 1))) * np.exp2(rng.integers(-3, 4, (1, cols)))
    return l8.rounded(x.astype(np.float32), dtype)


def _store(x, dtype, form, tiles, which="both"):
    """(buffer or None, buffer or None) of x and of its transposed; nothing behind them is written"""
    import torch
    import paper_2506_06472_amd as tio
    rows, cols = x.shape
    t = l8.padded(x, dtype)
    need = tio.tio_fp8_bytes(rows, cols), tio.tio_fp8_bytes(cols, rows)
    bufs = [torch.full((n + 64,), 77, device="cuda", dtype=torch.uint8) if which in ("both", w) else None for n, w in zip(need, ("plain", "transposed"))]
    tio.tio_op_fp8_store(0, dtype, form, tiles, rows, cols, t.data_ptr(), t.stride(0), *[0 if b is None else b.data_ptr() for b in bufs])
    for b, n in zip(bufs, need):
        assert b is None or (b[n:] == 77).all()
    return bufs


def _load(buf, dtype, form, rows, cols):
    import torch
    import paper_2506_06472_amd as tio
    out = torch.full((rows + 1, (cols + 7) // 8 * 8 + 8), 7.0, device="cuda", dtype=l8.types(dtype))
    tio.tio_op_fp8_load(0, dtype, form, rows, cols, buf.data_ptr(), out.data_ptr(), out.stride(0))
    return l8.clean(out, cols, 7.0, rows)


def _same(got, want):
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.nan_to_num(got, nan=5.0), np.nan_to_num(want, nan=5.0))


SIZES = [(1, 1), (1, 128), (3, 129), (16, 8), (17, 100), (64, 256), (65, 127), (128, 128), (129, 300), (257, 515), (1021, 96)]


@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("form", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_round_trip(rows, cols, dtype, form, tiles):
    x = _values(rows, cols, dtype)
    want = l8.stored(x, form, tiles)
    want_t = want.T if tiles else l8.stored(np.ascontiguousarray(x.T), form)
    plain, trans = _store(x, dtype, form, tiles)
    for d in ("bf16", "fp32"):                                  # the values are exact in both
        _same(_load(plain, d, form, rows, cols), want)
        _same(_load(trans, d, form, cols, rows), want_t)
    import torch
    a, b = _store(x, dtype, form, tiles, "plain")[0], _store(x, dtype, form, tiles, "transposed")[1]
    assert torch.equal(a, plain) and torch.equal(b, trans)      # either form alone has the same bytes


@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("form", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_special_values(dtype, form, tiles):
    """Zeros, ties, the largest codes, subnormal codes and numbers, huge magnitudes, blocks that are not finite."""
    x = np.zeros((16, 256))
    top = 448.0 if form == "e4m3" else 57344.0
    x[0, :128] = np.arange(128) / 16 + 1.0 / 32
    x[1, :5] = [top, top * (1 - 2.0 ** -7), -top, 1.0, 0.5]
    x[2, :4] = [1.75, 1.7578125, -1.5, 2.0 ** -9]               # at and above 1.75: the next power of two
    x[3, :3] = [2.0, 1.0625, 1.1875]                            # ties to even
    x[4, :64] = np.exp2(-np.arange(64.0))                       # down to subnormal codes and zero
    x[5, :3] = [2.0 ** -120, 2.0 ** -126, -2.0 ** -119]         # the smallest block
    x[5, 128:131] = [2.0 ** -127, 1.5 * 2.0 ** -128, 2.0 ** -133]
    x[6, 0] = 1.75 * 2.0 ** 127
    x[7, :2] = [1.9921875 * 2.0 ** 127, 2.0 ** 120]             # rounds to 2^128
    x[8, 3] = np.inf
    x[9, 200] = np.nan
    x[10, 255] = -np.inf
    x[11, :] = -0.0
    if tiles:                                                   # one power for all of them: a case at a time
        cases = [np.concatenate([x[i:i + 1], np.full((2, 256), 2.0 ** -130)]) for i in range(12)]
    else:
        cases = [x]
    for c in cases:
        if dtype == "bf16":
            c = l8.rounded(c, dtype)
        want = l8.stored(c, form, tiles)
        plain, trans = _store(c, dtype, form, tiles)
        _same(_load(plain, dtype, form, *c.shape), want)
        _same(_load(trans, dtype, form, c.shape[1], c.shape[0]), want.T if tiles else l8.stored(np.ascontiguousarray(c.T), form))


def _product(a, b, dtype, fa, fb, bias=None, resid=None, tiles_b=False, in_place=False):
    """C of stored a [M, K] and b [N, K], and the values that they stand for"""
    import torch
    import paper_2506_06472_amd as tio
    (M, K), N = a.shape, b.shape[0]
    qa, qb = _store(a, "fp32", fa, False, "plain")[0], _store(b, "fp32", fb, tiles_b, "plain")[0]
    t = [None if v is None else l8.padded(v, dtype) for v in (bias, resid)]
    c = torch.full((M + 1, (N + 7) // 8 * 8 + 8), 7.0, device="cuda", dtype=l8.types(dtype))
    if in_place:
        c[:M, :N] = t[1][:, :N]
        t[1] = c
    work = torch.full((tio.tio_op_gemm_fp8_work(M, N, K) + 64,), 255, device="cuda", dtype=torch.uint8)
    ptr = [0 if v is None else v.data_ptr() for v in t]
    tio.tio_op_gemm_fp8(0, dtype, M, N, K, fa, qa.data_ptr(), fb, qb.data_ptr(), c.data_ptr(), c.stride(0), ptr[0], ptr[1], 0 if t[1] is None else t[1].stride(0),
                        work.data_ptr())
    assert (work[-64:] == 255).all()
    return l8.clean(c, N, 7.0, M), l8.stored(a, fa), l8.stored(b, fb, tiles_b)


def _bound(a, b, want, dtype, extra=0.0):
    """Rounding of the result (twice: the type's half step of a value off by the rest), a rounding of 32 bits for each of K sums and two more, and in bf16 what the
    matrix cores cut off: of each product in a block of 128 at most 2^-13 of the largest."""
    K = a.shape[1]
    total = np.abs(a) @ np.abs(b).T + extra
    err = (K + 4) * l8.E32 * total
    if dtype == "bf16":
        for k in range(0, K, 128):
            err += 128 * 2.0 ** -13 * np.max(np.abs(a[:, None, k:k + 128] * b[None, :, k:k + 128]), axis=2)
    return l8.U[dtype] * np.abs(want) + 1.01 * err + 1e-37


PRODUCTS = [(1, 1, 1), (1, 40, 129), (2, 515, 352), (4, 1000, 256), (15, 16, 640), (16, 17, 128), (17, 33, 127), (33, 64, 1000), (64, 200, 384), (100, 64, 4200),
            (128, 128, 256), (130, 257, 136), (256, 256, 512), (257, 300, 100), (512, 520, 1152), (20, 24, 20000), (300, 200, 5000)]


@pytest.mark.parametrize("forms", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product(M, N, K, dtype, forms):
    if forms != ("e4m3", "e4m3") and M > 256:
        pytest.skip("large sizes with one pair of forms")
    a, b = _values(M, K, "fp32"), _values(N, K, "fp32", 1)
    got, qa, qb = _product(a, b, dtype, *forms, tiles_b=forms[1] == "e4m3")
    want = qa @ qb.T
    assert (np.abs(got - want) <= _bound(qa, qb, want, dtype)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(1, 40, 129), (33, 64, 1000), (130, 257, 136), (257, 300, 1100), (700, 900, 300)])
def test_product_of_small_whole_numbers_is_exact(M, N, K, dtype):
    """Products up to 2^6 with sums below 2^24 are exact however they are added, and a misplaced element shows; results are rounded once."""
    rng = np.random.default_rng(K)
    a, b = rng.integers(-8, 9, (M, K)).astype(float), rng.integers(-8, 9, (N, K)).astype(float)
    a[:, 0], b[:, 0] = 8, 8
    got, qa, qb = _product(a, b, dtype, "e4m3", "e4m3")
    assert np.array_equal(qa, a) and np.array_equal(qb, b)
    assert np.array_equal(got, l8.rounded(a @ b.T, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(4, 100, 300), (70, 77, 128), (300, 270, 520)])
@pytest.mark.parametrize("in_place", [False, True])
def test_product_with_bias_and_residual(M, N, K, dtype, in_place):
    a, b = _values(M, K, "fp32"), _values(N, K, "fp32", 1)
    rng = np.random.default_rng(5)
    bias, resid = l8.rounded(rng.standard_normal((1, N)) * 30, dtype), l8.rounded(rng.standard_normal((M, N)) * 100, dtype)
    for x, r in ((bias, None), (None, resid), (bias, resid)):
        if in_place and r is None:
            continue
        got, qa, qb = _product(a, b, dtype, "e4m3", "e5m2", x, r, in_place=in_place)
        add = (0 if x is None else x) + (0 if r is None else r)
        want = qa @ qb.T + add
        assert (np.abs(got - want) <= _bound(qa, qb, want, dtype, np.abs(0 if x is None else x) + np.abs(0 if r is None else r))).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(4, 40, 300), (300, 270, 260)])
def test_product_with_blocks_that_are_not_finite(M, N, K, dtype):
    """An infinity or a NaN spoils its rows and columns, and no others."""
    a, b = _values(M, K, "fp32"), _values(N, K, "fp32", 1)
    a[2, K - 1], a[3, 0], b[N - 1, 5] = np.inf, np.nan, -np.inf
    got, qa, qb = _product(a, b, dtype, "e4m3", "e4m3")
    bad = np.zeros((M, N), bool)
    bad[2], bad[3], bad[:, N - 1] = True, True, True
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()
    fine = np.ix_([i for i in range(M) if i not in (2, 3)], range(N - 1))
    want = (qa @ qb.T)[fine]
    rows = [i for i in range(M) if i not in (2, 3)]
    assert (np.abs(got[fine] - want) <= _bound(qa[rows], qb[:-1], want, dtype)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scales_far_apart(dtype):
    """Blocks from 2^-100 to 2^100 in the two operands of one product."""
    a, b = _values(20, 384, "fp32"), _values(30, 384, "fp32", 1)
    s = np.repeat([100.0, 0.0, -100.0], 128)
    got, qa, qb = _product((a * np.exp2(s)).astype(np.float32).astype(float), (b * np.exp2(-s)).astype(np.float32).astype(float), dtype, "e4m3", "e4m3")
    want = qa @ qb.T
    assert (np.abs(got - want) <= _bound(qa, qb, want, dtype)).all()


WAYS = [("bf16", 9, 700, 1000, (16, 16, 1, 4)), ("bf16", 33, 500, 9000, (16, 16, 1, 8)), ("bf16", 70, 1101, 9000, (32, 16, 1, 8)),
        ("bf16", 1000, 500, 300, (32, 32, 1, 4)), ("bf16", 1113, 158, 7105, (32, 32, 1, 8)), ("bf16", 802, 588, 5470, (64, 32, 1, 8)),
        ("bf16", 768, 768, 8000, (64, 128, 3, 3)), ("bf16", 143, 8633, 2554, (64, 128, 3, 1)),
        ("bf16", 1443, 458, 16388, (128, 128, 4, 5)), ("bf16", 61, 3, 28095, (128, 128, 4, 32)),
        ("bf16", 1000, 4000, 4000, (128, 128, 4, 1)),
        ("bf16", 4100, 770, 700, (64, 128, 3, 1)), ("bf16", 8000, 750, 780, (128, 128, 2, 1)), ("bf16", 4000, 4100, 1000, (256, 256, 2, 1)),
        ("bf16", 2048, 768, 30000, (128, 128, 4, 2)), ("bf16", 17, 4163, 38991, (64, 128, 3, 7)),
        ("bf16", 1786, 1439, 29596, (128, 128, 2, 3)), ("bf16", 154, 5450, 30935, (256, 256, 2, 11)),
        ("bf16", 6000, 5000, 130, (256, 256, 2, 1)), ("fp32", 9, 700, 1000, (16, 16, 1, 4)), ("fp32", 33, 500, 9000, (16, 16, 1, 8)),
        ("fp32", 70, 1101, 9000, (32, 16, 1, 8)), ("fp32", 1000, 500, 300, (32, 32, 1, 4)), ("fp32", 1113, 158, 7105, (32, 32, 1, 8)),
        ("fp32", 1000, 1000, 8000, (64, 32, 1, 8)), ("fp32", 5093, 803, 26396, (128, 128, 2, 3)), ("fp32", 4000, 1500, 500, (128, 128, 2, 1)),
        ("fp32", 2000, 2050, 300, (128, 128, 2, 1))]


@pytest.mark.parametrize("dtype,M,N,K,way", WAYS)
def test_every_way_to_take_a_product(dtype, M, N, K, way):
    """Small whole numbers, whose products and sums are exact however they are added (up to 2^6 each, 2^24 in all): the rounded result, alone and with bias and
    residual, whose sum with a product is exact too."""
    import torch
    import paper_2506_06472_amd as tio
    assert tio.tio_op_gemm_fp8_route(dtype, M, N, K) == way
    t, up = l8.types(dtype), lambda n: (n + 7) // 8 * 8
    g = torch.Generator(device="cuda").manual_seed(K)
    whole = lambda r, c, top: torch.randint(-top, top + 1, (r, c), device="cuda", generator=g).float()

    def padded(v, fill):
        b = torch.full((v.shape[0], up(v.shape[1]) + 8), fill, device="cuda", dtype=t)
        b[:, :v.shape[1]] = v
        return b
    a, b, bias, resid = whole(M, K, 8), whole(N, K, 8), whole(1, N, 100), whole(M, N, 100)
    assert K * 64 < 1 << 24
    q = []
    for v, rows in ((a, M), (b, N)):
        v[:, ::128] = 8.0                                       # blocks have a scale of their own, but the same for all
        p = padded(v, float("nan"))
        q.append(torch.empty(tio.tio_fp8_bytes(rows, K), device="cuda", dtype=torch.uint8))
        tio.tio_op_fp8_store(0, dtype, "e4m3", False, rows, K, p.data_ptr(), p.stride(0), q[-1].data_ptr())
    work = torch.full((tio.tio_op_gemm_fp8_work(M, N, K) + 64,), 255, device="cuda", dtype=torch.uint8)
    pb, pr = padded(bias, float("nan")), padded(resid, float("nan"))
    want = a.double() @ b.double().t()
    for with_bias, with_resid in ((0, 0), (1, 1)):
        c = torch.full((M + 1, up(N) + 8), 7.0, device="cuda", dtype=t)
        tio.tio_op_gemm_fp8(0, dtype, M, N, K, "e4m3", q[0].data_ptr(), "e4m3", q[1].data_ptr(), c.data_ptr(), c.stride(0), pb.data_ptr() * with_bias,
                            pr.data_ptr() * with_resid, pr.stride(0), work.data_ptr())
        ref = want + with_bias * bias + with_resid * resid
        assert torch.equal(c[:M, :N], ref.to(t)) and (c[:M, N:up(N)] == 0).all() and (c[:M, up(N):] == 7.0).all() and (c[M:] == 7.0).all()
    assert (work[-64:] == 255).all()


def test_calls_in_a_graph_and_on_another_stream():
    """A linear layer's calls captured once and replayed on new values, with eager work in between; the same bits as eager calls."""
    import torch
    import paper_2506_06472_amd as tio
    S, K, N = 200, 260, 150
    up = lambda n: (n + 7) // 8 * 8
    x, w, y = (torch.zeros((r, up(c)), device="cuda", dtype=torch.bfloat16) for r, c in ((S, K), (N, K), (S, N)))
    xq, wq = (torch.zeros(tio.tio_fp8_bytes(r, K), device="cuda", dtype=torch.uint8) for r in (S, N))
    work = torch.zeros(tio.tio_op_gemm_fp8_work(S, N, K) + 16, device="cuda", dtype=torch.uint8)

    def calls():
        s = torch.cuda.current_stream().cuda_stream
        tio.tio_op_fp8_store(s, "bf16", "e4m3", False, S, K, x.data_ptr(), x.stride(0), xq.data_ptr())
        tio.tio_op_fp8_store(s, "bf16", "e4m3", True, N, K, w.data_ptr(), w.stride(0), wq.data_ptr())
        tio.tio_op_gemm_fp8(s, "bf16", S, N, K, "e4m3", xq.data_ptr(), "e4m3", wq.data_ptr(), y.data_ptr(), y.stride(0), work_ptr=work.data_ptr())
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        x[:, :K], w[:, :K] = torch.randn(S, K, device="cuda") * 3 ** i, torch.randn(N, K, device="cuda")
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        y.zero_()
        calls()
        torch.cuda.synchronize()
        assert torch.equal(got, y) and y.abs().sum() > 0


def test_rows_past_4_gib():
    """Matrices whose rows lie past 4 GiB of their buffer have the bits of rows side by side."""
    import torch
    import paper_2506_06472_amd as tio
    R, C, far = 40, 200, 1 << 26
    flat = torch.full(((R - 1) * far + C + 8,), 7.0, device="cuda", dtype=torch.bfloat16)
    wide = flat.as_strided((R, C), (far, 1))
    x = torch.randn((R, C), device="cuda").to(torch.bfloat16)
    wide.copy_(x)
    q = torch.zeros((4, max(tio.tio_fp8_bytes(R, C), tio.tio_fp8_bytes(C, R))), device="cuda", dtype=torch.uint8)
    for i, (v, ld) in enumerate(((x, C), (wide, far))):
        tio.tio_op_fp8_store(0, "bf16", "e4m3", False, R, C, v.data_ptr(), ld, q[2 * i].data_ptr(), q[2 * i + 1].data_ptr())
    assert torch.equal(q[:2], q[2:])
    near = torch.empty_like(x)
    tio.tio_op_fp8_load(0, "bf16", "e4m3", R, C, q[0].data_ptr(), near.data_ptr(), C)
    tio.tio_op_fp8_load(0, "bf16", "e4m3", R, C, q[0].data_ptr(), flat.data_ptr(), far)
    assert torch.equal(wide, near)
    for M, N, tile in ((40, 200, 16), (1000, 600, 32), (2000, 2000, 64), (2000, 4000, 128), (4000, 4104, 256)):
        assert tio.tio_op_gemm_fp8_route("bf16", M, N, 1000)[0] == tile
        a, b = torch.randn((M, 1000), device="cuda"), torch.randn((N, 1000), device="cuda")
        s = [torch.zeros(tio.tio_fp8_bytes(len(v), 1000), device="cuda", dtype=torch.uint8) for v in (a, b)]
        for v, to in zip((a, b), s):
            tio.tio_op_fp8_store(0, "fp32", "e4m3", False, len(v), 1000, v.data_ptr(), 1000, to.data_ptr())
        work = torch.empty(tio.tio_op_gemm_fp8_work(M, N, 1000) + 16, device="cuda", dtype=torch.uint8)
        ld = flat.numel() // M // 8 * 8
        big = torch.as_strided(flat, (M, N), (ld, 1))
        near = torch.empty((M, N), device="cuda", dtype=torch.bfloat16)
        big.copy_(torch.randn((M, N), device="cuda"))
        resid = big.clone()
        for c, c_ld, r, r_ld in ((near, N, resid, N), (big, ld, big, ld)):
            tio.tio_op_gemm_fp8(0, "bf16", M, N, 1000, "e4m3", s[0].data_ptr(), "e4m3", s[1].data_ptr(), c.data_ptr(), c_ld, 0, r.data_ptr(), r_ld, work.data_ptr())
        assert torch.equal(big, near) and not torch.equal(near, resid)


def test_stored_matrix_past_4_gib():
    """Codes behind the first 4 GiB: values read back, and products of them, of whole numbers, which are exact."""
    import torch
    import paper_2506_06472_amd as tio
    R, C, N = (1 << 17) + 17, 1 << 15, 264
    x = torch.randint(-8, 9, (R, C), device="cuda", dtype=torch.bfloat16)
    q = torch.empty(tio.tio_fp8_bytes(R, C), device="cuda", dtype=torch.uint8)
    tio.tio_op_fp8_store(0, "bf16", "e4m3", False, R, C, x.data_ptr(), C, q.data_ptr())
    back = torch.empty_like(x)
    tio.tio_op_fp8_load(0, "bf16", "e4m3", R, C, q.data_ptr(), back.data_ptr(), C)
    assert q.numel() > 1 << 32 and torch.equal(back, x)
    del back
    w = torch.randint(-8, 9, (N, C), device="cuda", dtype=torch.bfloat16)
    wq = torch.empty(tio.tio_fp8_bytes(N, C), device="cuda", dtype=torch.uint8)
    tio.tio_op_fp8_store(0, "bf16", "e4m3", False, N, C, w.data_ptr(), C, wq.data_ptr())
    work = torch.empty(tio.tio_op_gemm_fp8_work(R, N, C) + 16, device="cuda", dtype=torch.uint8)
    for dtype in ("fp32", "bf16"):
        y = torch.empty((R, N), device="cuda", dtype=l8.types(dtype))
        tio.tio_op_gemm_fp8(0, dtype, R, N, C, "e4m3", q.data_ptr(), "e4m3", wq.data_ptr(), y.data_ptr(), N, work_ptr=work.data_ptr())
        for at in (0, 1 << 16, R - 500):
            assert torch.equal(y[at:at + 500], (x[at:at + 500].float() @ w.float().t()).to(y.dtype))
    del y, q, work, wq
    xt = torch.empty(tio.tio_fp8_bytes(C, R), device="cuda", dtype=torch.uint8)
    even = x // 2 * 2                                           # up to 8: two bits
    tio.tio_op_fp8_store(0, "bf16", "e5m2", True, R, C, even.data_ptr(), C, 0, xt.data_ptr())
    back = torch.empty((C, (R + 7) // 8 * 8), device="cuda", dtype=torch.bfloat16)
    tio.tio_op_fp8_load(0, "bf16", "e5m2", C, R, xt.data_ptr(), back.data_ptr(), back.stride(0))
    for at in (0, C // 2, C - 300):
        assert torch.equal(back[at:at + 300, :R], even[:, at:at + 300].t()) and (back[at:at + 300, R:] == 0).all()


def test_two_products_at_once():
    """On two streams, each with a work memory of its own: the bits of one after the other."""
    import torch
    import paper_2506_06472_amd as tio
    M, N, K = 768, 768, 16000
    assert tio.tio_op_gemm_fp8_route("bf16", M, N, K)[3] > 1
    q = []
    for i in range(4):
        v = torch.randn((M, K), device="cuda")
        q.append(torch.empty(tio.tio_fp8_bytes(M, K), device="cuda", dtype=torch.uint8))
        tio.tio_op_fp8_store(0, "fp32", "e4m3", False, M, K, v.data_ptr(), K, q[-1].data_ptr())
    work = [torch.empty(tio.tio_op_gemm_fp8_work(M, N, K), device="cuda", dtype=torch.uint8) for _ in range(2)]
    y = torch.zeros((2, 2, M, N), device="cuda", dtype=torch.bfloat16)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]

    def call(i, out, stream):
        tio.tio_op_gemm_fp8(stream, "bf16", M, N, K, "e4m3", q[2 * i].data_ptr(), "e4m3", q[2 * i + 1].data_ptr(), out.data_ptr(), N, work_ptr=work[i].data_ptr())
    for _ in range(8):
        for i in range(2):
            call(i, y[0, i], streams[i].cuda_stream)
    torch.cuda.synchronize()
    for i in range(2):
        call(i, y[1, i], 0)
    torch.cuda.synchronize()
    assert torch.equal(y[0], y[1]) and not torch.equal(y[0, 0], y[0, 1])


@pytest.mark.parametrize("M,N", [(1 << 22, 5), (5, 1 << 22)])
def test_the_most_rows(M, N):
    """The largest number of rows of either operand, whole numbers: exact."""
    import torch
    import paper_2506_06472_amd as tio
    K, ops, q = 100, [], []
    for rows in (M, N):
        v = torch.randint(-8, 9, (rows, 104), device="cuda", dtype=torch.bfloat16)
        q.append(torch.empty(tio.tio_fp8_bytes(rows, K), device="cuda", dtype=torch.uint8))
        tio.tio_op_fp8_store(0, "bf16", "e4m3", False, rows, K, v.data_ptr(), 104, q[-1].data_ptr())
        ops.append(v[:, :K])
    up = (N + 7) // 8 * 8
    work = torch.empty(tio.tio_op_gemm_fp8_work(M, N, K) + 16, device="cuda", dtype=torch.uint8)
    y = torch.full((M, up), 7.0, device="cuda", dtype=torch.bfloat16)
    tio.tio_op_gemm_fp8(0, "bf16", M, N, K, "e4m3", q[0].data_ptr(), "e4m3", q[1].data_ptr(), y.data_ptr(), up, work_ptr=work.data_ptr())
    assert torch.equal(y[:, :N], (ops[0].float() @ ops[1].float().t()).to(torch.bfloat16)) and (y[:, N:] == 0).all()
