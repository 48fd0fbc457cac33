"""Sizes and refusals of the operators of layers in 8-bit floating point: nothing here reaches a GPU."""
import pytest

import layer8lib as l8
import paper_2506_06472_amd as tio

P = 1 << 20                     # an aligned address that no refused call looks at
Q = P + 8


def _refused(call, *args, **kw):
    with pytest.raises(tio.TioError) as e:
        call(*args, **kw)
    assert e.value.code == -1


@pytest.mark.parametrize("rows,cols", [(1, 1), (16, 128), (17, 129), (64, 4096), (1021, 352), (1 << 22, 16), (16, 1 << 22)])
def test_bytes(rows, cols):
    blocks = -(-cols // 128)
    assert tio.tio_fp8_bytes(rows, cols) == -(-rows // 16) * blocks * 2048 + -(-rows // 64) * blocks * 64


@pytest.mark.parametrize("rows,cols", [(0, 1), (1, 0), (-1, 8), ((1 << 22) + 1, 1), (1, (1 << 22) + 1), (1 << 22, 1 << 20)])
def test_bytes_refused(rows, cols):
    _refused(tio.tio_fp8_bytes, rows, cols)
    _refused(tio.tio_op_gemm_fp8_work, rows, 8, cols)
    _refused(tio.tio_op_fp8_store, 0, "bf16", "e4m3", False, rows, cols, P, 1 << 23, P)
    _refused(tio.tio_op_fp8_load, 0, "bf16", "e4m3", rows, cols, P, P, 1 << 23)


def test_store_and_load_refused():
    ok = dict(rows=4, cols=20, x=P, ld=24, out=P, out_t=0)

    def store(**kw):
        a = {**ok, **kw}
        _refused(tio.tio_op_fp8_store, 0, "bf16", "e4m3", False, a["rows"], a["cols"], a["x"], a["ld"], a["out"], a["out_t"])
        if "out_t" not in kw and kw.get("out", P):
            _refused(tio.tio_op_fp8_load, 0, "fp32", "e5m2", a["rows"], a["cols"], a["out"], a["x"], a["ld"])
    store(x=0)
    store(out=0)
    store(x=Q)
    store(out=Q)
    store(out_t=Q)
    store(ld=20)
    store(ld=16)
    store(ld=-24)
    L = tio.binding.lib()
    for dtype, form in ((2, 0), (0, 2), (-1, 0), (1, -1)):
        assert L.tio_op_fp8_store(0, dtype, form, 0, 4, 20, P, 24, P, 0) == -1
        assert L.tio_op_fp8_load(0, dtype, form, 4, 20, P, P, 24) == -1
        assert L.tio_op_gemm_fp8(0, dtype, 4, 8, 16, form, P, 0, P, 0, 0, 0, P, 8, P) == -1
        assert L.tio_op_gemm_fp8(0, dtype, 4, 8, 16, 0, P, form, P, 0, 0, 0, P, 8, P) == -1


def test_product_refused():
    ok = dict(M=4, N=20, K=16, A=P, B=P, C=P, ldc=24, bias=0, resid=0, ldr=0, work=P)

    def product(**kw):
        a = {**ok, **kw}
        _refused(tio.tio_op_gemm_fp8, 0, "bf16", a["M"], a["N"], a["K"], "e4m3", a["A"], "e4m3", a["B"], a["C"], a["ldc"], a["bias"], a["resid"], a["ldr"], a["work"])
    for name in ("A", "B", "C"):
        product(**{name: 0})
        product(**{name: Q})
    for name in ("M", "N", "K"):
        product(**{name: 0})
        product(**{name: (1 << 22) + 1, "ldc": 1 << 23})
    product(ldc=20)
    product(ldc=16)
    product(resid=P, ldr=16)
    product(resid=P, ldr=0)
    product(resid=Q, ldr=24)
    product(bias=Q)
    product(work=Q)
    product(resid=P, ldr=32)                                    # in place, with another stride
    for M, N, K in ((0, 8, 8), (8, 0, 8), (8, 8, 0), ((1 << 22) + 1, 8, 8), (8, (1 << 22) + 1, 8), (8, 8, (1 << 22) + 1), (1 << 22, 8, 1 << 22)):
        _refused(tio.tio_op_gemm_fp8_route, "bf16", M, N, K)


def test_product_without_the_work_it_needs_refused():
    M, N, K = 768, 768, 16000
    assert tio.tio_op_gemm_fp8_work(M, N, K) >= M * N * 8 and tio.tio_op_gemm_fp8_work(4, 1000, 1000) == 0
    _refused(tio.tio_op_gemm_fp8, 0, "bf16", M, N, K, "e4m3", P, "e4m3", P, P, N, 0, 0, 0, 0)


@pytest.mark.parametrize("p", [-0.1, 1.0, 1.5, float("nan"), float("inf"), 65535.6 / 65536])
def test_probabilities_refused(p):
    _refused(tio.tio_op_dropout, 0, "bf16", 4, 20, P, 24, 0, 0, P, 24, p, 1, 2)
    _refused(tio.tio_op_residual_norm, 0, "bf16", tio.tio_residual_cfg(True, p=p), 4, 20, 24, P, P, 0, 0, 0, 0, P, 0, P, P, P)


def test_dropout_refused():
    def drop(rows=4, cols=20, x=P, ldx=24, resid=0, ldr=0, y=P, ldy=24):
        _refused(tio.tio_op_dropout, 0, "bf16", rows, cols, x, ldx, resid, ldr, y, ldy, 0.1, 1, 2)
    drop(rows=0)
    drop(cols=0)
    drop(rows=1 << 31)
    drop(rows=1 << 30)                                          # times three groups of eight
    drop(x=0)
    drop(y=0)
    drop(x=Q)
    drop(y=Q)
    drop(resid=Q, ldr=24)
    drop(resid=P, ldr=16)
    drop(ldx=20)
    drop(ldy=16)
    drop(ldx=32)                                                # in place, with another stride
    drop(x=2 * P, resid=P, ldr=32)
    assert tio.binding.lib().tio_op_dropout(0, 2, 4, 20, P, 24, 0, 0, P, 24, 0.1, 1, 2) == -1


FORWARD = dict(rows=4, d=20, ld=24, branch=P, x=P, gate=0, ldg=0, post_gain=0, post_bias=0, gain=P, bias=0, y=P, h=P, stats=P)
BACKWARD = dict(rows=4, d=20, ld=24, branch=P, y=P, gate=0, ldg=0, post_gain=0, post_bias=0, gain=P, stats=P, dy=P, dh=P, dx=P, dbranch=P, dgate=0, dpost_gain=0,
                dpost_bias=0, dgain=P, dbias=0, work=P)


@pytest.mark.parametrize("call,ok", [(tio.tio_op_residual_norm, FORWARD), (tio.tio_op_residual_norm_bwd, BACKWARD)])
def test_residual_norm_refused(call, ok):
    def no(cfg=tio.tio_residual_cfg(False), **kw):
        _refused(call, 0, "bf16", cfg, *{**ok, **kw}.values())
    for name, v in ok.items():
        if v == P:
            no(**{name: 0})
            no(**{name: Q})
    no(rows=0)
    no(rows=(1 << 31) + 1)
    no(d=0)
    no(d=8193, ld=8200)
    no(ld=20)
    no(ld=16)
    no(post_bias=P)
    no(tio.tio_residual_cfg(False, eps=-1.0))
    no(tio.tio_residual_cfg(False, eps=float("nan")))
    no(tio.tio_residual_cfg(False, resid_scale=float("inf")))
    no(tio.tio_residual_cfg(False, branch_scale=float("nan")))
    gate = dict(gate=P, **({"dgate": P} if "dgate" in ok else {}))
    no(**{**gate, "gate": Q})
    no(**gate, ldg=16)
    no(**gate, ldg=20)
    bias = "bias" if "bias" in ok else "dbias"
    no(**{bias: Q})
    no(tio.tio_residual_cfg(True), **{bias: P})
    if "dgate" in ok:
        no(gate=P)
        no(dgate=P)
        no(post_gain=P)
        no(dpost_gain=P)
        no(dpost_bias=P)
        no(tio.tio_residual_cfg(True), post_gain=P, dpost_gain=P, dpost_bias=P)


@pytest.mark.parametrize("rows,d", [(0, 8), (8, 0), (8, 8193), ((1 << 31) + 1, 8)])
def test_residual_norm_work_refused(rows, d):
    _refused(tio.tio_op_residual_norm_bwd_work, rows, d)


def test_rope_refused():
    def rope(rows=4, heads=2, dh=32, x=P, ldx=64, y=P, ldy=64, pos=P, sections=(8, 8), theta=1e4):
        _refused(tio.tio_op_rope_axes, 0, "bf16", rows, heads, dh, x, ldx, y, ldy, pos, list(sections), theta)
    for kw in (dict(rows=0), dict(rows=1 << 31), dict(heads=0), dict(heads=65537, ldx=1 << 22, ldy=1 << 22), dict(dh=0), dict(dh=12), dict(dh=264, ldx=528, ldy=528),
               dict(x=0), dict(y=0), dict(pos=0), dict(x=Q), dict(y=Q), dict(pos=P + 2), dict(sections=()), dict(sections=(8, 0)), dict(sections=(8, -1)),
               dict(sections=(8, 9)), dict(sections=(1,) * 9), dict(sections=(2147483647,)), dict(theta=0.0), dict(theta=-1.0),
               dict(theta=float("nan")), dict(theta=float("inf")), dict(ldx=56), dict(ldy=60), dict(ldy=72)):
        rope(**kw)


def test_generator_against_its_published_vectors():
    f = 0xffffffff
    assert l8.philox([(0, 0, 0, 0)], (0, 0)) == [[0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]]
    assert l8.philox([(f, f, f, f)], (f, f)) == [[0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]]
    assert l8.philox([(0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344)], (0xa4093822, 0x299f31d0)) == [[0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]]
