"""GPU: norms around a block with gate, dropout and residual, dropout alone, rotary positions with several axes, against their definitions in 64 bits."""
import numpy as np
import pytest

import layer8lib as l8

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols,p,seed,offset", [(1, 1, 0.5, 0, 0), (1, 9, 0.5, 1, 2), (3, 64, 0.1, 2 ** 63 + 7, 2 ** 40 + 3), (129, 100, 0.9, 5, 2 ** 64 - 1),
                                                     (40, 333, 0.0, 3, 3), (7, 128, 65535 / 65536, 9, 9), (64, 8, 1e-9, 4, 4)])
@pytest.mark.parametrize("resid", [False, True])
def test_dropout(rows, cols, p, seed, offset, resid, dtype):
    import torch
    import paper_2506_06472_amd as tio
    rng = np.random.default_rng(cols)
    x, r = (l8.rounded(rng.standard_normal((rows, cols)) * 4, dtype) for _ in range(2))
    tx, tr = l8.padded(x, dtype), l8.padded(r, dtype, extra=16)
    y = torch.full_like(l8.padded(x, dtype, extra=24), 7.0)
    tio.tio_op_dropout(0, dtype, rows, cols, tx.data_ptr(), tx.stride(0), tr.data_ptr() if resid else 0, tr.stride(0) if resid else 0, y.data_ptr(), y.stride(0),
                       p, seed, offset)
    got = l8.clean(y, cols, 7.0)
    m = l8.mask(rows, cols, p, seed, offset)
    want = x * m + (r if resid else 0)
    err = 3 * l8.E32 * (np.abs(x * m) + np.abs(r if resid else 0))          # the factor, the product, the sum in 32 bits
    assert (np.abs(got - want) <= l8.U[dtype] * np.abs(want) + 1.01 * err).all()
    if not resid:
        assert (got[m == 0] == 0).all()


@pytest.mark.parametrize("over", ["x", "resid"])
def test_dropout_in_place_and_of_values_that_are_not_finite(over):
    """A dropped infinity or NaN is a zero; y over either operand."""
    import torch
    import paper_2506_06472_amd as tio
    rows, cols = 70, 40
    rng = np.random.default_rng(1)
    x, r = rng.standard_normal((rows, cols)).astype(np.float32), rng.standard_normal((rows, cols)).astype(np.float32)
    m = l8.mask(rows, cols, 0.5, 11, 12)
    x[m == 0] = np.where(rng.random(int((m == 0).sum())) < 0.5, np.inf, np.nan)
    tx, tr = torch.from_numpy(x).cuda(), torch.from_numpy(r).cuda()
    y = tx if over == "x" else tr
    tio.tio_op_dropout(0, "fp32", rows, cols, tx.data_ptr(), cols, tr.data_ptr(), cols, y.data_ptr(), cols, 0.5, 11, 12)
    with np.errstate(invalid="ignore"):
        want = np.where(m == 0, 0.0, x * m) + r
    assert (np.abs(y.cpu().numpy() - want) <= 4 * l8.E32 * (np.abs(want) + 2 * np.abs(r))).all()


def test_dropout_rows_past_2_to_the_32():
    """Elements whose counter and whose byte offset need more than 32 bits: rows of one group far apart, at the ends of a buffer of 5 GiB."""
    import torch
    import paper_2506_06472_amd as tio
    rows, ld = 3, 1 << 30
    x = torch.zeros((rows - 1) * ld + 8, device="cuda", dtype=torch.bfloat16)
    y = torch.zeros_like(x)
    for r in range(rows):
        x[r * ld:r * ld + 8] = float(r + 1)
    tio.tio_op_dropout(0, "bf16", rows, 8, x.data_ptr(), ld, 0, 0, y.data_ptr(), ld, 0.5, 3, 4)
    want = l8.mask(rows, 8, 0.5, 3, 4) * np.arange(1, rows + 1)[:, None]
    for r in range(rows):
        assert np.array_equal(y[r * ld:r * ld + 8].double().cpu().numpy(), want[r])


# ------------------------------------------------------------------ norms around a block
class _Case:
    def __init__(self, rows, d, dtype, rms, post, gate, p, bias=True, seed=0, extra=8):
        self.rows, self.d, self.dtype, self.rms, self.post, self.gate, self.p, self.extra = rows, d, dtype, rms, post, gate, p, extra
        rng = np.random.default_rng(rows * 100 + d + seed)
        new = lambda n, std, mean=0.0: l8.rounded(rng.standard_normal((n, d)) * std + mean, dtype)
        self.v = dict(branch=new(rows, 0.7, 0.2), x=new(rows, 2.0), gain=new(1, 0.1, 1.0), dy=new(rows, 0.5), dh=new(rows, 0.5))
        if post:
            self.v["post_gain"] = new(1, 0.1, 1.0)
        if not rms and bias:
            self.v["bias"] = new(1, 0.3)
            if post:
                self.v["post_bias"] = new(1, 0.3)
        if gate:
            self.v["gate"] = new(rows if gate == "rows" else 1, 0.3, 0.5)
        self.eps, self.rs, self.bs, self.seed, self.offset = 1e-5, 0.9375, 0.5, 77, 2 ** 33 + 5
        self.eps = float(np.float32(self.eps))

    def run(self, backward=True, tensors=None):
        """outputs as float64, by name; the rounded y among them"""
        import torch
        import paper_2506_06472_amd as tio
        t = tensors or {n: l8.padded(v, self.dtype, extra=self.extra) for n, v in self.v.items()}
        self.t = t
        P = lambda n: t[n].data_ptr() if n in t else 0
        ld, rows, d = t["x"].stride(0), self.rows, self.d
        cfg = tio.tio_residual_cfg(self.rms, self.eps, self.rs, self.bs, self.p, self.seed, self.offset)
        new = lambda like: torch.full_like(t[like], 7.0)
        y, h, stats = new("x"), new("x"), torch.full((rows + 1, 4), 7.0, device="cuda")
        ldg = t["gate"].stride(0) if self.gate == "rows" else 0
        tio.tio_op_residual_norm(0, self.dtype, cfg, rows, d, ld, P("branch"), P("x"), P("gate"), ldg, P("post_gain"), P("post_bias"), P("gain"), P("bias"),
                                 y.data_ptr(), h.data_ptr(), stats.data_ptr())
        assert (stats[rows:] == 7.0).all()
        self.raw = dict(y=y, h=h)
        if backward:
            for n in ("x", "branch", "gate", "post_gain", "post_bias", "gain", "bias"):
                if n in t:
                    self.raw["d" + n] = new(n)
            G = lambda n: self.raw[n].data_ptr() if n in self.raw else 0
            work = torch.full((tio.tio_op_residual_norm_bwd_work(rows, d) + 64,), 255, device="cuda", dtype=torch.uint8)
            tio.tio_op_residual_norm_bwd(0, self.dtype, cfg, rows, d, ld, P("branch"), y.data_ptr(), P("gate"), ldg, P("post_gain"), P("post_bias"), P("gain"),
                                         stats.data_ptr(), P("dy"), P("dh"), G("dx"), G("dbranch"), G("dgate"), G("dpost_gain"), G("dpost_bias"), G("dgain"),
                                         G("dbias"), work.data_ptr())
            assert (work[-64:] == 255).all()
        vector = lambda n: "gain" in n or "bias" in n or (n == "dgate" and not ldg)
        return {n: (l8.untouched if vector(n) else l8.clean)(v, d, 7.0) for n, v in self.raw.items()}

    def want(self, y_rounded):
        """{name: (value, bound of the error without the result's rounding)}.  Arithmetic in 32 bits: c roundings of the magnitudes that meet in a sum, c = 64 for
        the chains here (a row's sums are trees of at most 48 additions in a thread's chunk, a wavefront and its row), and for column sums one more per row.
        The gradients are taken at the rounded y, whose norm is taken with the statistics of y before its rounding, as the kernel has it."""
        v, c = {n: a.astype(np.float64) for n, a in self.v.items()}, 64 * l8.E32
        A = np.abs
        m = l8.mask(self.rows, self.d, self.p, self.seed, self.offset)
        gate = v.get("gate", np.ones((1, 1)))
        n, big = v["branch"], A(v["branch"])
        if self.post:
            n, pm, pr = l8.norm(n, self.rms, v["post_gain"], v.get("post_bias", 0.0), self.eps)
            bh, bhm = (v["branch"] - pm) * pr, (A(v["branch"]) + A(pm)) * pr
            big = bhm * A(v["post_gain"]) + A(v.get("post_bias", 0.0))
        u, um = n * m, big * m
        y = self.rs * v["x"] + self.bs * gate * u
        ym = self.rs * A(v["x"]) + self.bs * A(gate) * um
        h, mean, rstd = l8.norm(y, self.rms, v["gain"], v.get("bias", 0.0), self.eps)
        yhm = (ym + A(mean) + ym.mean(1, keepdims=True)) * rstd
        hm = yhm * A(v["gain"]) * 2 + A(v.get("bias", 0.0))
        out = {"y": (y, c * ym), "h": (h, c * hm)}

        def back(g, gm, vh, vhm, rs):
            """N^T without gain and with it: value and magnitude"""
            val = g - vh * (g * vh).mean(1, keepdims=True) - (0 if self.rms else g.mean(1, keepdims=True))
            mag = gm + vhm * (gm * vhm).mean(1, keepdims=True) + (0 if self.rms else gm.mean(1, keepdims=True))
            return val * rs, mag * rs
        yh = (y_rounded - mean) * rstd
        g, gm = v["dh"] * v["gain"], A(v["dh"] * v["gain"])
        D, Dm = back(g, gm, yh, yhm, rstd)
        D, Dm = D + v["dy"], Dm * 2 + A(v["dy"])
        col = lambda t, tm: (t.sum(0, keepdims=True), (c + self.rows * l8.E32) * tm.sum(0, keepdims=True))
        out["dx"] = (self.rs * D, c * self.rs * Dm)
        out["dgain"] = col(v["dh"] * yh, A(v["dh"]) * yhm * 2)
        if "bias" in v:
            out["dbias"] = col(v["dh"], A(v["dh"]))
        if self.gate:
            dg, dgm = self.bs * u * D, 2 * self.bs * um * Dm
            out["dgate"] = (dg, c * dgm) if self.gate == "rows" else col(dg, dgm)
        dn, dnm = self.bs * gate * m * D, self.bs * A(gate) * m * Dm
        if self.post:
            out["dpost_gain"] = col(dn * bh, 2 * dnm * bhm)
            if "post_bias" in v:
                out["dpost_bias"] = col(dn, dnm)
            dn, dnm = back(dn * v["post_gain"], dnm * A(v["post_gain"]), bh, bhm, pr)
        out["dbranch"] = (dn, 2 * c * dnm)
        return out

    def check(self, backward=True, got=None):
        got = got or self.run(backward)
        want = self.want(got["y"])
        assert set(got) == {n for n in want if backward or n in "yh"}
        for n, t in got.items():
            w, bound = want[n]
            off = np.abs(t - w) - l8.U[self.dtype] * np.abs(w) - 1.01 * bound
            assert (off <= 0).all(), (n, off.max(), np.abs(w).max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rms,post,gate,p", [(True, True, "shared", 0.1), (True, False, None, 0.0), (False, True, "rows", 0.5), (False, False, "shared", 0.1),
                                             (True, True, "rows", 0.0), (False, True, None, 0.0)])
@pytest.mark.parametrize("rows,d", [(1, 1), (3, 8), (5, 100), (130, 128), (9, 513), (6, 1024), (5, 1030), (33, 2048), (4, 2056), (3, 4096), (2, 5001)])
def test_residual_norm(rows, d, dtype, rms, post, gate, p):
    _Case(rows, d, dtype, rms, post, gate, p).check()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rms,rows,d", [(True, 2, 7000), (False, 3, 8192), (True, 5000, 64), (False, 2100, 1032)])
def test_residual_norm_wide_and_many(rms, rows, d, dtype):
    _Case(rows, d, dtype, rms, True, "shared", 0.1, extra=0).check()


@pytest.mark.parametrize("post", [False, True])
def test_residual_norm_without_biases_and_forward_alone(post):
    _Case(7, 72, "fp32", False, post, None, 0.0, bias=False).check()
    _Case(7, 72, "bf16", True, post, "rows", 0.3).check(backward=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_residual_norm_in_place(dtype):
    """y over x and dx over dy have the bits of separate buffers."""
    import torch
    import paper_2506_06472_amd as tio
    c = _Case(300, 520, dtype, True, True, "shared", 0.1)
    c.run()
    t, ld = c.t, c.t["x"].stride(0)
    cfg = tio.tio_residual_cfg(True, c.eps, c.rs, c.bs, c.p, c.seed, c.offset)
    x, dy, h, dbranch = t["x"].clone(), t["dy"].clone(), torch.full_like(t["x"], 7.0), torch.full_like(t["x"], 7.0)
    stats, one = torch.empty((300, 4), device="cuda"), [torch.full_like(t["gain"], 7.0) for _ in range(3)]
    work = torch.empty(tio.tio_op_residual_norm_bwd_work(300, 520), device="cuda", dtype=torch.uint8)
    P = lambda n: t[n].data_ptr()
    tio.tio_op_residual_norm(0, dtype, cfg, 300, 520, ld, P("branch"), x.data_ptr(), P("gate"), 0, P("post_gain"), 0, P("gain"), 0, x.data_ptr(), h.data_ptr(),
                             stats.data_ptr())
    tio.tio_op_residual_norm_bwd(0, dtype, cfg, 300, 520, ld, P("branch"), x.data_ptr(), P("gate"), 0, P("post_gain"), 0, P("gain"), stats.data_ptr(),
                                 dy.data_ptr(), P("dh"), dy.data_ptr(), dbranch.data_ptr(), one[0].data_ptr(), one[1].data_ptr(), 0, one[2].data_ptr(), 0,
                                 work.data_ptr())
    r = c.raw
    for a, b in ((x, r["y"]), (h, r["h"]), (dy, r["dx"]), (dbranch, r["dbranch"]), (one[0], r["dgate"]), (one[1], r["dpost_gain"]), (one[2], r["dgain"])):
        assert torch.equal(a[:, :520], b[:, :520])


def test_residual_norm_gradients_against_differences():
    """A directional derivative along each operand, from the forward pass in fp32 alone: two-sided differences of step 2^-6 along unit directions are off by
    the rounding of the outputs and by the third derivative, together below 2 % of the derivative's scale."""
    c = _Case(6, 40, "fp32", False, True, "rows", 0.3)
    got = c.run()
    base = {n: v.copy() for n, v in c.v.items()}

    def loss():
        o = c.run(backward=False)
        return (o["y"] * base["dy"]).sum() + (o["h"] * base["dh"]).sum()
    rng = np.random.default_rng(3)
    for n in ("x", "branch", "gate", "post_gain", "post_bias", "gain", "bias"):
        along = rng.standard_normal(base[n].shape)
        along += 2 * got["d" + n] / np.linalg.norm(got["d" + n]) * np.sqrt(along.size)
        along /= np.linalg.norm(along)
        step = 2.0 ** -6
        value = []
        for sign in (1, -1):
            c.v[n] = l8.rounded(base[n] + sign * step * along, "fp32")
            value.append(loss())
            c.v[n] = base[n]
        slope = (value[0] - value[1]) / (2 * step)
        assert abs(slope - (got["d" + n] * along).sum()) <= 0.02 * np.linalg.norm(got["d" + n]), n


def test_residual_norm_rows_that_are_not_finite():
    """An infinity or NaN in a row stays in it (and in the column sums); a dropped one in branch without a norm does no harm."""
    c = _Case(9, 64, "fp32", True, False, None, 0.5)
    m = l8.mask(9, 64, 0.5, c.seed, c.offset)
    col = int(np.argmin(m[4]))
    clean = c.run()
    c.v["branch"][4, col] = np.inf
    got = c.run()
    for n in ("y", "h", "dx", "dbranch"):
        assert np.array_equal(got[n], clean[n]), n
    c.v["x"][2, 5] = np.nan
    got = c.run()
    for n in ("y", "h", "dx", "dbranch"):
        keep = [i for i in range(9) if i != 2]
        assert np.array_equal(got[n][keep], clean[n][keep]), n
    assert np.isnan(got["h"][2]).all()


def test_residual_norm_of_constant_and_zero_rows():
    """Variance zero: 1 / sqrt(eps), and no NaN."""
    c = _Case(4, 48, "fp32", False, True, None, 0.0)
    c.v["branch"][0], c.v["x"][0] = 0.0, 0.0
    c.v["branch"][1], c.v["x"][1] = 3.0, -2.0
    got = c.run()
    assert all(np.isfinite(v).all() for v in got.values())
    assert np.allclose(got["y"][0], 0.5 * c.v["post_bias"][0], rtol=0, atol=1e-6)


def test_residual_norm_in_a_graph():
    """Both passes captured and replayed on other values, with eager work between, the same bits each time."""
    import torch
    import paper_2506_06472_amd as tio
    c = _Case(700, 264, "bf16", True, True, "shared", 0.1)
    c.run()
    t, ld = c.t, c.t["x"].stride(0)
    cfg = tio.tio_residual_cfg(True, c.eps, c.rs, c.bs, c.p, c.seed, c.offset)
    out = {n: torch.zeros_like(v) for n, v in c.raw.items()}
    stats = torch.empty((700, 4), device="cuda")
    work = torch.empty(tio.tio_op_residual_norm_bwd_work(700, 264), device="cuda", dtype=torch.uint8)
    P, G = lambda n: t[n].data_ptr(), lambda n: out[n].data_ptr()

    def calls():
        s = torch.cuda.current_stream().cuda_stream
        tio.tio_op_residual_norm(s, "bf16", cfg, 700, 264, ld, P("branch"), P("x"), P("gate"), 0, P("post_gain"), 0, P("gain"), 0, G("y"), G("h"), stats.data_ptr())
        tio.tio_op_residual_norm_bwd(s, "bf16", cfg, 700, 264, ld, P("branch"), G("y"), P("gate"), 0, P("post_gain"), 0, P("gain"), stats.data_ptr(), P("dy"), P("dh"),
                                     G("dx"), G("dbranch"), G("dgate"), G("dpost_gain"), 0, G("dgain"), 0, work.data_ptr())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for i in range(4):
        t["x"][:, :264] += 1.0
        t["dh"][:, :264] *= 1.5
        graph.replay()
        torch.cuda.synchronize()
        got = {n: v.clone() for n, v in out.items()}
        for v in out.values():
            v.zero_()
        calls()
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(got[n], out[n]), n


def test_residual_norm_rows_past_4_gib():
    """Rows whose places need more than 32 bits, all matrices side by side in one buffer: the bits of rows one behind the other."""
    import torch
    import paper_2506_06472_amd as tio
    rows, d, far = 5, 72, 1 << 29
    c = _Case(rows, d, "bf16", False, True, "rows", 0.3)
    c.run()
    flat = torch.full(((rows - 1) * far + 16 * 128,), 7.0, device="cuda", dtype=torch.bfloat16)
    place = {n: flat.as_strided((rows, d), (far, 1), 128 * i) for i, n in enumerate(("branch", "x", "gate", "y", "h", "dy", "dh", "dx", "dbranch", "dgate"))}
    for n in ("branch", "x", "gate", "dy", "dh"):
        place[n].copy_(c.t[n][:, :d])
    one = {n: torch.full_like(c.t["gain"], 7.0) for n in ("dpost_gain", "dpost_bias", "dgain", "dbias")}
    stats, work = torch.empty((rows, 4), device="cuda"), torch.empty(tio.tio_op_residual_norm_bwd_work(rows, d), device="cuda", dtype=torch.uint8)
    P = lambda n: (place.get(n) if n in place else one[n] if n in one else c.t[n]).data_ptr()
    cfg = tio.tio_residual_cfg(False, c.eps, c.rs, c.bs, c.p, c.seed, c.offset)
    tio.tio_op_residual_norm(0, "bf16", cfg, rows, d, far, P("branch"), P("x"), P("gate"), far, P("post_gain"), P("post_bias"), P("gain"), P("bias"), P("y"), P("h"),
                             stats.data_ptr())
    tio.tio_op_residual_norm_bwd(0, "bf16", cfg, rows, d, far, P("branch"), P("y"), P("gate"), far, P("post_gain"), P("post_bias"), P("gain"), stats.data_ptr(),
                                 P("dy"), P("dh"), P("dx"), P("dbranch"), P("dgate"), P("dpost_gain"), P("dpost_bias"), P("dgain"), P("dbias"), work.data_ptr())
    for n in ("y", "h", "dx", "dbranch", "dgate"):
        assert torch.equal(place[n], c.raw[n][:, :d]), n
    for n, v in one.items():
        assert torch.equal(v, c.raw[n]), n


def test_two_backward_passes_at_once():
    """On two streams, each with a work memory of its own: the bits of one after the other."""
    import torch
    import paper_2506_06472_amd as tio
    cases = [_Case(700, 264, "fp32", True, True, "shared", 0.1, seed=i) for i in range(2)]
    want = [c.run() for c in cases]
    streams, outs, keep = [torch.cuda.Stream(), torch.cuda.Stream()], [], []
    for c in cases:
        cfg = tio.tio_residual_cfg(True, c.eps, c.rs, c.bs, c.p, c.seed, c.offset)
        o = {n: torch.full_like(v, 7.0) for n, v in c.raw.items()}
        outs.append(o)
        keep.append((cfg, torch.empty((700, 4), device="cuda"), torch.empty(tio.tio_op_residual_norm_bwd_work(700, 264), device="cuda", dtype=torch.uint8)))
    torch.cuda.synchronize()
    for _ in range(4):
        for c, o, (cfg, stats, work), s in zip(cases, outs, keep, streams):
            t, ld, P, G = c.t, c.t["x"].stride(0), lambda n: c.t[n].data_ptr(), lambda n: o[n].data_ptr()
            tio.tio_op_residual_norm(s.cuda_stream, "fp32", cfg, 700, 264, ld, P("branch"), P("x"), P("gate"), 0, P("post_gain"), 0, P("gain"), 0, G("y"), G("h"),
                                     stats.data_ptr())
            tio.tio_op_residual_norm_bwd(s.cuda_stream, "fp32", cfg, 700, 264, ld, P("branch"), G("y"), P("gate"), 0, P("post_gain"), 0, P("gain"), stats.data_ptr(),
                                         P("dy"), P("dh"), G("dx"), G("dbranch"), G("dgate"), G("dpost_gain"), 0, G("dgain"), 0, work.data_ptr())
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        for n, v in o.items():
            assert np.array_equal(v[:, :264].double().cpu().numpy(), w[n]), n


def test_dropout_and_rope_in_a_graph_and_on_another_stream():
    """Captured once and replayed on other values and positions, with eager work between: the bits of eager calls."""
    import torch
    import paper_2506_06472_amd as tio
    rows, heads, dh = 300, 5, 64
    x = torch.zeros((rows, heads * dh), device="cuda", dtype=torch.bfloat16)
    y, z = torch.zeros_like(x), torch.zeros_like(x)
    pos = torch.zeros((rows, 2), device="cuda", dtype=torch.int32)

    def calls():
        s = torch.cuda.current_stream().cuda_stream
        tio.tio_op_dropout(s, "bf16", rows, heads * dh, x.data_ptr(), heads * dh, x.data_ptr(), heads * dh, y.data_ptr(), heads * dh, 0.25, 9, 10)
        tio.tio_op_rope_axes(s, "bf16", rows, heads, dh, y.data_ptr(), heads * dh, z.data_ptr(), heads * dh, pos.data_ptr(), [20, 12], 10000.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    side = torch.cuda.Stream()
    for i in range(4):
        x.copy_(torch.randn((rows, heads * dh), device="cuda") * (i + 1))
        pos.copy_(torch.randint(0, 1000, (rows, 2), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = z.clone()
        y.zero_()
        z.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            calls()
        torch.cuda.synchronize()
        assert torch.equal(got, z) and z.abs().sum() > 0


# ------------------------------------------------------------------ rotary positions
def _turned(x, pos, heads, dh, sections, theta, own, inverse):
    """value, and the angles' magnitudes and the pairs' that the bound needs"""
    z = x[:, :heads * dh].reshape(len(x), heads, dh).copy()
    turned, size = z.copy(), np.zeros_like(z)
    i = 0
    for a, n in enumerate(sections):
        for j in range(n):
            angle = pos[:, a].astype(np.longdouble) * np.longdouble(theta) ** np.longdouble(-j / n if own else -2.0 * i / dh)
            w = (angle if not inverse else -angle)[:, None]
            p, q = z[:, :, 2 * i], z[:, :, 2 * i + 1]
            c, s = np.cos(w).astype(np.float64), np.sin(w).astype(np.float64)
            turned[:, :, 2 * i], turned[:, :, 2 * i + 1] = p * c - q * s, p * s + q * c
            size[:, :, 2 * i] = size[:, :, 2 * i + 1] = (np.abs(p) + np.abs(q)) * (16 * l8.E32 + 2.0 ** -50 * np.abs(angle[:, None].astype(np.float64)))
            i += 1
    return turned.reshape(len(x), -1), size.reshape(len(x), -1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,heads,dh,sections,own,inverse,far", [
    (1, 1, 8, (4,), False, False, 0), (1, 1, 8, (1,), True, True, 5), (3, 2, 32, (6, 4), True, True, 1 << 20), (70, 5, 64, (16, 8, 8), False, False, 100),
    (33, 40, 128, (16, 24, 24), False, True, 0), (9, 3, 256, (100, 20, 8), False, False, -40000), (5, 7, 40, (3, 3, 3, 3, 2, 2, 2, 2), True, False, 2 ** 31 - 400),
    (2100, 4, 32, (16,), False, False, -2 ** 31 + 10)])
def test_rope_axes(rows, heads, dh, sections, own, inverse, far, dtype):
    """Frequencies are powers in 64 bits, angles their products with positions: 2^-52 of an angle each, times two, and 16 roundings of 32 bits for sine, cosine
    and the sums of two products."""
    import torch
    import paper_2506_06472_amd as tio
    rng = np.random.default_rng(rows)
    x = l8.rounded(rng.standard_normal((rows, heads * dh)), dtype)
    pos = (far + rng.integers(0, 300, (rows, len(sections)))).astype(np.int32)
    t, p = l8.padded(x, dtype), torch.from_numpy(pos).cuda()
    y = torch.full((rows + 1, heads * dh + 16), 7.0, device="cuda", dtype=t.dtype)
    for src, out in ((t, y), (t, t)):
        tio.tio_op_rope_axes(0, dtype, rows, heads, dh, src.data_ptr(), src.stride(0), out.data_ptr(), out.stride(0), p.data_ptr(), sections, 10000.0, own, inverse)
    got = l8.clean(y, heads * dh, 7.0, rows)
    assert torch.equal(t[:, :heads * dh], y[:rows, :heads * dh]) and torch.isnan(t[:, heads * dh:]).all()
    want, size = _turned(x, pos, heads, dh, sections, 10000.0, own, inverse)
    assert (np.abs(got - want) <= l8.U[dtype] * np.abs(want) + 1.01 * size).all()
    left = np.arange(dh) >= 2 * sum(sections)
    assert np.array_equal(got.reshape(rows, heads, dh)[:, :, left], x.reshape(rows, heads, dh)[:, :, left])


def test_rope_of_one_axis_is_the_steps_rotation():
    """With one axis over all pairs and positions 0 .. T - 1 it is the rotation that a training step applies: on relative positions alone."""
    import torch
    import paper_2506_06472_amd as tio
    T, dh = 50, 64
    x = torch.randn((1, dh), device="cuda").repeat(T, 1).contiguous()
    y = torch.empty_like(x)
    pos = torch.arange(T, device="cuda", dtype=torch.int32)
    tio.tio_op_rope_axes(0, "fp32", T, 1, dh, x.data_ptr(), dh, y.data_ptr(), dh, pos.data_ptr(), [dh // 2], 10000.0)
    s = (y.double() @ y.double().t()).cpu().numpy()
    scale = float((x[0].double() ** 2).sum())
    for k in range(T):
        diagonal = np.diagonal(s, k)
        assert np.abs(diagonal - diagonal[0]).max() <= 64 * l8.E32 * scale


def test_rope_rows_past_4_gib():
    import torch
    import paper_2506_06472_amd as tio
    rows, far = 5, 1 << 29
    flat = torch.full(((rows - 1) * far + 256,), 7.0, device="cuda", dtype=torch.bfloat16)
    x = torch.randn((rows, 128), device="cuda").to(torch.bfloat16)
    pos = torch.randint(0, 1 << 20, (rows, 1), device="cuda", dtype=torch.int32)
    wide, y = flat.as_strided((rows, 128), (far, 1)), torch.empty_like(x)
    wide.copy_(x)
    tio.tio_op_rope_axes(0, "bf16", rows, 2, 64, x.data_ptr(), 128, y.data_ptr(), 128, pos.data_ptr(), [32], 10000.0)
    tio.tio_op_rope_axes(0, "bf16", rows, 2, 64, flat.data_ptr(), far, flat.data_ptr(), far, pos.data_ptr(), [32], 10000.0)
    assert torch.equal(wide, y) and (flat[128:256] == 7.0).all()
