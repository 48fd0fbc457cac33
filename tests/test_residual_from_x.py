"""The backward pass of the norms around a block from the forward pass's x: the gradients of what the forward pass computed, with no rounding of y among them."""
import itertools

import numpy as np
import pytest

import layer8lib as l8
import paper_2506_06472_amd as tio
from paper_2506_06472_amd import build
from test_gpu_layer8_rows import _Case
from test_kernel_resources import _code_objects, _kernels

A16 = 1 << 20                                                  # some aligned address; nothing is read there


def _call(**change):
    """the entry with arguments that all hold, but for `change`; no GPU"""
    a = dict(cfg=tio.tio_residual_cfg(True), rows=4, d=24, ld=32, branch=A16, x=A16, gate=A16, ldg=0, post_gain=A16, post_bias=0, gain=A16, stats=A16, dy=A16, dh=A16, dx=A16,
             dbranch=A16, dgate=A16, dpost_gain=A16, dpost_bias=0, dgain=A16, dbias=0, work=A16, dtype="bf16")
    a.update(change)
    dtype = a.pop("dtype")
    tio.tio_op_residual_norm_bwd_from_x(0, dtype, *a.values())


@pytest.mark.parametrize("change", [{n: 0} for n in ("branch", "x", "gain", "stats", "dy", "dh", "dx", "dbranch", "dgain", "work")]
                         + [{n: A16 + 8} for n in ("branch", "x", "gate", "post_gain", "gain", "stats", "dy", "dh", "dx", "dbranch", "dgate", "dpost_gain", "dgain", "work")]
                         + [{"rows": 0}, {"d": 0}, {"d": 8193, "ld": 8200}, {"ld": 28}, {"ld": 16}, {"ldg": 4}, {"rows": (1 << 31) + 1}, {"gate": 0}, {"dgate": 0},
                            {"post_gain": 0}, {"dpost_gain": 0}, {"post_bias": A16}, {"dbias": A16}, {"cfg": tio.tio_residual_cfg(True, eps=-1.0)},
                            {"cfg": tio.tio_residual_cfg(True, p=1.0)}, {"cfg": tio.tio_residual_cfg(True, resid_scale=float("inf"))}], ids=str)
def test_refusals(change):
    with pytest.raises(tio.TioError):
        _call(**change)


def test_the_kernels_keep_everything_in_registers():
    """in every form that a call may take, and in no other (see test_layer8_kernel_resources)"""
    tio.binding.lib()
    with open(build.LIB, "rb") as f:
        mine = {k[".name"]: k for obj in _code_objects(f.read()) for k in _kernels(obj) if "21residual_norm_bwd_x_k" in k[".name"]}
    forms = [f"I{t}Li{w}ELb{rms}ELb{post}E" for t, w, rms, post in itertools.product(("NS_6bf16_tE", "f"), (1, 2, 4, 8, 16), (0, 1), (0, 1))]
    assert len(mine) == len(forms) and all(sum(f in n for n in mine) == 1 for f in forms)
    assert not any(k[".vgpr_spill_count"] or k[".private_segment_fixed_size"] for k in mine.values())


class _FromX(_Case):
    def run(self, backward=True, tensors=None):
        """as _Case.run, with x in y's place in the backward pass"""
        if not backward:
            return super().run(backward, tensors)
        call, seen = tio.tio_op_residual_norm_bwd_from_x, []

        def from_x(stream, dtype, cfg, rows, d, ld, branch, y, *rest):
            seen.append(y)
            assert y == self.raw["y"].data_ptr()
            call(stream, dtype, cfg, rows, d, ld, branch, self.t["x"].data_ptr(), *rest)
        kept, tio.tio_op_residual_norm_bwd = tio.tio_op_residual_norm_bwd, from_x
        try:
            out = super().run(True, tensors)
        finally:
            tio.tio_op_residual_norm_bwd = kept
        assert len(seen) == 1
        return out

    def check(self, backward=True, got=None):
        got = got or self.run(backward)
        want = self.want(self.want(got["y"])["y"][0])           # the gradients at y itself, in 64 bits
        assert set(got) == set(want)
        for n, t in got.items():
            w, bound = want[n]
            off = np.abs(t - w) - l8.U[self.dtype] * np.abs(w) - 1.01 * bound
            assert (off <= 0).all(), (n, off.max(), np.abs(w).max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rms,post,gate,p", [(True, True, "shared", 0.1), (True, False, None, 0.0), (False, True, "rows", 0.5), (False, False, "shared", 0.1),
                                             (True, True, "rows", 0.0), (False, True, None, 0.0), (True, False, "rows", 0.3), (False, False, "rows", 0.0)])
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 8), (5, 100), (130, 128), (9, 513), (6, 1024), (5, 1030), (33, 2048), (4, 2056), (3, 4096), (2, 5001), (2, 7000)])
def test_gradients(rows, d, dtype, rms, post, gate, p):
    """Within a rounding of the result and the arithmetic of 32 bits that _Case.want counts: of y's rounding to bf16, 2^-9 of it in vh, nothing is left."""
    _FromX(rows, d, dtype, rms, post, gate, p).check()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rms,rows,d", [(True, 5000, 64), (False, 2100, 1032), (False, 3, 8192)])
def test_many_and_wide(rms, rows, d, dtype):
    _FromX(rows, d, dtype, rms, True, "shared", 0.1, extra=0).check()
    _FromX(rows, d, dtype, rms, False, "rows", 0.1, extra=0).check()


@pytest.mark.gpu
def test_from_y_it_is_another_gradient():
    """The bound of the test above tells the two apart: from y as bf16 has it dgain is off by more."""
    c = _FromX(130, 128, "bf16", True, True, "shared", 0.1)
    exact = c.want(c.want(c.run()["y"])["y"][0])["dgain"]
    other = _Case(130, 128, "bf16", True, True, "shared", 0.1).run()["dgain"]
    assert (np.abs(other - exact[0]) > l8.U["bf16"] * np.abs(exact[0]) + 1.01 * exact[1]).any()


@pytest.mark.gpu
def test_a_dropped_infinity_does_no_harm():
    """In a branch without a norm: y is made without it, as in the forward pass."""
    c = _FromX(9, 64, "fp32", True, False, None, 0.5)
    m = l8.mask(9, 64, 0.5, c.seed, c.offset)
    clean = c.run()
    c.v["branch"][4, int(np.argmin(m[4]))] = np.inf
    got = c.run()
    for n in ("y", "h", "dx", "dbranch", "dgain"):
        assert np.array_equal(got[n], clean[n]), n


@pytest.mark.gpu
@pytest.mark.parametrize("rms,gate", [(True, None), (False, "rows")])
def test_in_a_graph_and_over_dy(rms, gate):
    """Captured with the forward pass and replayed on other values, dx over dy, eager work between: the bits of eager calls on buffers of their own."""
    import torch
    rows, d = 700, 264
    c = _FromX(rows, d, "bf16", rms, True, gate, 0.1)
    c.run()
    t, ld = c.t, c.t["x"].stride(0)
    ldg = t["gate"].stride(0) if gate == "rows" else 0
    cfg = tio.tio_residual_cfg(rms, c.eps, c.rs, c.bs, c.p, c.seed, c.offset)
    out = {n: torch.zeros_like(v) for n, v in c.raw.items()}
    stats, work = torch.empty((rows, 4), device="cuda"), torch.empty(tio.tio_op_residual_norm_bwd_work(rows, d), device="cuda", dtype=torch.uint8)
    P, G = lambda n: t[n].data_ptr() if n in t else 0, lambda n: out[n].data_ptr() if n in out else 0
    both = t["dy"].clone()

    def calls(dy, dx):
        s = torch.cuda.current_stream().cuda_stream
        tio.tio_op_residual_norm(s, "bf16", cfg, rows, d, ld, P("branch"), P("x"), P("gate"), ldg, P("post_gain"), P("post_bias"), P("gain"), P("bias"), G("y"), G("h"),
                                 stats.data_ptr())
        tio.tio_op_residual_norm_bwd_from_x(s, "bf16", cfg, rows, d, ld, P("branch"), P("x"), P("gate"), ldg, P("post_gain"), P("post_bias"), P("gain"), stats.data_ptr(), dy,
                                            P("dh"), dx, G("dbranch"), G("dgate"), G("dpost_gain"), G("dpost_bias"), G("dgain"), G("dbias"), work.data_ptr())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(both.data_ptr(), both.data_ptr())
    for _ in range(4):
        t["x"][:, :d] += 1.0
        t["dh"][:, :d] *= 1.5
        both.copy_(t["dy"])
        graph.replay()
        torch.cuda.synchronize()
        got = {n: v.clone() for n, v in out.items()}
        got["dx"] = both.clone()
        for v in out.values():
            v.zero_()
        calls(P("dy"), G("dx"))
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(got[n][:, :d], out[n][:, :d]), n
