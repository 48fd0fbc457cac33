"""GPU: a decoder layer trained in 8-bit floating point, forward and backward, through the operators together: dropout of the embedding, attention over packed
sequences with positions of several axes, norms around the attention with gate, dropout and residual, SwiGLU whose inputs are kept in 8 bits, every product on
stored matrices, weights stored once and read as they are and transposed."""
import numpy as np
import pytest

import layer8lib as l8

pytestmark = pytest.mark.gpu
SECTIONS = {32: [4, 6, 6], 64: [8, 12, 10], 128: [16, 24, 24]}
P_DROP, SEED = 0.25, 1234567


class _Layer:
    def __init__(self, dtype, lens, d, H, Hkv, dh, f, grad, seed=0):
        import torch
        self.dtype, self.t, self.lens, self.S, self.d, self.H, self.Hkv, self.dh, self.f, self.grad = dtype, l8.types(dtype), lens, sum(lens), d, H, Hkv, dh, f, grad
        g = torch.Generator().manual_seed(seed)
        new = lambda rows, cols, std, mean=0.0: (torch.randn((rows, cols), generator=g) * std + mean).to(self.t)
        self.wide, self.hd = (H + 2 * Hkv) * dh, H * dh
        self.w = {n: new(r, c, c ** -0.5) for n, (r, c) in dict(qkv=(self.wide, d), o=(d, self.hd), gate=(f, d), up=(f, d), down=(d, f)).items()}
        self.v = {n: new(1, d, 0.1, m) for n, m in dict(gain=1.0, post_gain=1.0, rgate=0.5).items()}
        self.e, self.dz = new(self.S, d, 1.0), new(self.S, d, 1.0)
        self.pos = torch.randint(0, 50, (self.S, 3), generator=g, dtype=torch.int32)

    def run(self):
        """Outputs in self.out, what the stored matrices stand for in self.kept[name], of the transposed ones in self.kept_t."""
        import torch
        import paper_2506_06472_amd as tio
        import packedlib as pl
        S, d, f, dt, H, Hkv, dh = self.S, self.d, self.f, self.dtype, self.H, self.Hkv, self.dh
        P = lambda t: 0 if t is None else t.data_ptr()
        up8 = lambda n: (n + 7) // 8 * 8
        new = lambda rows, cols: torch.full((rows, up8(cols)), float("nan"), device="cuda", dtype=self.t)

        def put(a):
            b = torch.zeros((a.shape[0], up8(a.shape[1])), device="cuda", dtype=self.t)
            b[:, :a.shape[1]] = a.cuda()
            return b
        self.kept, self.kept_t, q, qt = {}, {}, {}, {}

        def store(name, t, rows, cols, form="e4m3", tiles=False):
            q[name], qt[name] = (torch.empty(tio.tio_fp8_bytes(r, c), device="cuda", dtype=torch.uint8) for r, c in ((rows, cols), (cols, rows)))
            tio.tio_op_fp8_store(0, dt, form, tiles, rows, cols, P(t), t.stride(0), P(q[name]), P(qt[name]))
            for kept, buf, r, c in ((self.kept, q, rows, cols), (self.kept_t, qt, cols, rows)):
                b = new(r, c)
                tio.tio_op_fp8_load(0, dt, form, r, c, P(buf[name]), P(b), b.stride(0))
                kept[name] = b[:, :c].double().cpu()

        def product(M, N, K, a, b, form="e4m3", resid=None):
            c = new(M, N)
            work = torch.empty(tio.tio_op_gemm_fp8_work(M, N, K) + 16, device="cuda", dtype=torch.uint8)
            tio.tio_op_gemm_fp8(0, dt, M, N, K, form, P(a), "e4m3", P(b), P(c), c.stride(0), 0, P(resid), 0 if resid is None else resid.stride(0), P(work))
            return c
        shape = dict(qkv=(self.wide, d), o=(d, self.hd), gate=(f, d), up=(f, d), down=(d, f))
        for n, t in self.w.items():
            store("w_" + n, put(t), *shape[n], tiles=True)
        e, dz, pos = put(self.e), put(self.dz), self.pos.cuda()
        v = {n: put(t) for n, t in self.v.items()}
        # forward
        x = new(S, d)
        tio.tio_op_dropout(0, dt, S, d, P(e), e.stride(0), 0, 0, P(x), x.stride(0), P_DROP, SEED, 0)
        store("x", x, S, d)
        qkv = product(S, self.wide, d, q["x"], q["w_qkv"])
        rope = lambda t, inverse: tio.tio_op_rope_axes(0, dt, S, H + Hkv, dh, P(t), t.stride(0), P(t), t.stride(0), P(pos), SECTIONS[dh], 100.0, False, inverse)
        rope(qkv, False)
        pk, dev = pl.packing(self.lens, dt, H, Hkv, dh)
        o, lse = new(S, self.hd), torch.empty((H, S), device="cuda")
        tio.tio_op_attention_packed(0, pk, P(dev), P(qkv), qkv.stride(0), P(o), o.stride(0), P(lse))
        store("o", o, S, self.hd)
        a = product(S, d, self.hd, q["o"], q["w_o"])
        cfg = tio.tio_residual_cfg(True, 1e-5, 0.9375, 0.5, P_DROP, SEED, 1)
        y, h, stats = new(S, d), new(S, d), torch.empty((S, 4), device="cuda")
        tio.tio_op_residual_norm(0, dt, cfg, S, d, x.stride(0), P(a), P(x), P(v["rgate"]), 0, P(v["post_gain"]), 0, P(v["gain"]), 0, P(y), P(h), P(stats))
        store("h", h, S, d)
        gate, up = product(S, f, d, q["h"], q["w_gate"]), product(S, f, d, q["h"], q["w_up"])
        act, half = new(S, f), tio.tio_ckpt8_bytes(S, f)
        ck = torch.empty(2 * half, device="cuda", dtype=torch.uint8)
        tio.tio_op_act_ckpt8(0, dt, "swiglu", S, f, P(gate), P(up), gate.stride(0), P(act), act.stride(0), P(ck))
        store("act", act, S, f)
        z = product(S, d, f, q["act"], q["w_down"], resid=y)
        out = dict(x=x, o=o, y=y, h=h, act=act, z=z)
        # backward
        G = self.grad
        store("dz", dz, S, d, G)
        dact = product(S, f, d, q["dz"], qt["w_down"], G)
        out["w_down"] = product(d, f, S, qt["dz"], qt["act"], G)
        dgate, dup, again = new(S, f), new(S, f), new(S, f)
        tio.tio_op_act_ckpt8_bwd(0, dt, "swiglu", S, f, P(ck), P(dact), dact.stride(0), P(dgate), P(dup), dgate.stride(0), P(again), again.stride(0))
        store("dgate", dgate, S, f, G)
        store("dup", dup, S, f, G)
        d_h = product(S, d, f, q["dup"], qt["w_up"], G, product(S, d, f, q["dgate"], qt["w_gate"], G))
        out["w_gate"], out["w_up"] = (product(f, d, S, qt[n], qt["h"], G) for n in ("dgate", "dup"))
        dx, da, (drg, dpg, dg) = new(S, d), new(S, d), (new(1, d) for _ in range(3))
        work = torch.empty(tio.tio_op_residual_norm_bwd_work(S, d), device="cuda", dtype=torch.uint8)
        tio.tio_op_residual_norm_bwd(0, dt, cfg, S, d, x.stride(0), P(a), P(y), P(v["rgate"]), 0, P(v["post_gain"]), 0, P(v["gain"]), P(stats), P(dz), P(d_h), P(dx), P(da),
                                     P(drg), P(dpg), 0, P(dg), 0, P(work))
        out.update(rgate=drg, post_gain=dpg, gain=dg)
        store("da", da, S, d, G)
        do = product(S, self.hd, d, q["da"], qt["w_o"], G)
        out["w_o"] = product(d, self.hd, S, qt["da"], qt["o"], G)
        dqkv = new(S, self.wide)
        work = torch.empty(tio.tio_op_attention_packed_work(pk), device="cuda", dtype=torch.uint8)
        tio.tio_op_attention_packed_bwd(0, pk, P(dev), P(qkv), qkv.stride(0), P(o), P(do), o.stride(0), P(lse), P(work), P(dqkv))
        rope(dqkv, True)
        store("dqkv", dqkv, S, self.wide, G)
        out["w_qkv"] = product(self.wide, d, S, qt["dqkv"], qt["x"], G)
        dx2, de = product(S, d, self.wide, q["dqkv"], qt["w_qkv"], G, dx), new(S, d)
        tio.tio_op_dropout(0, dt, S, d, P(dx2), dx2.stride(0), 0, 0, P(de), de.stride(0), P_DROP, SEED, 0)
        out["e"] = de
        for i, n in enumerate(("gate", "up")):
            b = new(S, f)
            tio.tio_op_ckpt8_load(0, dt, S, f, P(ck) + i * half, P(b), b.stride(0))
            self.kept["ck_" + n] = b[:, :f].double().cpu()
        torch.cuda.synchronize()
        cols = dict(o=self.hd, act=f, w_down=f, w_o=self.hd)
        self.out = {n: t[:, :cols.get(n, d)].double().cpu() for n, t in out.items()}
        return self.out

    def reference(self):
        """In 64 bits, from what the stored matrices stand for: a product's operands, its input's gradient and its weight's are theirs."""
        import torch
        kept, kept_t, dt = self.kept, self.kept_t, self.dtype

        class Linear(torch.autograd.Function):
            @staticmethod
            def forward(ctx, a, w, a_name, w_name, dy_name):
                ctx.names = a_name, w_name, dy_name
                return kept[a_name] @ kept["w_" + w_name].t()

            @staticmethod
            def backward(ctx, dy):
                a_name, w_name, dy_name = ctx.names
                seen[dy_name] = dy
                return kept[dy_name] @ kept["w_" + w_name], kept_t[dy_name] @ kept_t[a_name].t(), None, None, None

        class SwiGLU(torch.autograd.Function):
            @staticmethod
            def forward(ctx, g, u):
                return torch.nn.functional.silu(g) * u

            @staticmethod
            def backward(ctx, dy):
                g, u = kept["ck_gate"], kept["ck_up"]
                s = torch.sigmoid(g)
                return dy * u * (s + g * s * (1 - s)), dy * g * s
        seen = {}
        S, d, H, Hkv, dh = self.S, self.d, self.H, self.Hkv, self.dh
        w = {n: t.double().requires_grad_() for n, t in self.w.items()}
        v = {n: t.double().requires_grad_() for n, t in self.v.items()}
        e = self.e.double().requires_grad_()
        mask = [torch.from_numpy(l8.mask(S, d, P_DROP, SEED, i)) for i in range(2)]
        rms = lambda t, g: t / torch.sqrt((t * t).mean(1, keepdim=True) + float(np.float32(1e-5))) * g
        x = e * mask[0]
        qkv = Linear.apply(x, w["qkv"], "x", "qkv", "dqkv").view(S, H + 2 * Hkv, dh)
        n = sum(SECTIONS[dh])
        axis = torch.tensor([a for a, k in enumerate(SECTIONS[dh]) for _ in range(k)])
        angle = self.pos[:, axis].double() * 100.0 ** (-2.0 * torch.arange(n).double() / dh)
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        p, r = qkv[:, :H + Hkv, 0:2 * n:2], qkv[:, :H + Hkv, 1:2 * n:2]
        turned = torch.stack((p * c - r * s, p * s + r * c), -1).flatten(2)
        qk = torch.cat((turned, qkv[:, :H + Hkv, 2 * n:]), 2)
        parts, at = [], 0
        for length in self.lens:
            rows = slice(at, at + length)
            at += length
            q_, k_, v_ = (t.transpose(0, 1) for t in (qk[rows, :H], qk[rows, H:].repeat_interleave(H // Hkv, 1), qkv[rows, H + Hkv:].repeat_interleave(H // Hkv, 1)))
            score = (q_ @ k_.transpose(1, 2)) / np.sqrt(dh)
            score = score.masked_fill(torch.ones((length, length), dtype=torch.bool).triu(1), -torch.inf)
            parts.append((torch.softmax(score, -1) @ v_).transpose(0, 1).reshape(length, H * dh))
        o = torch.cat(parts)
        a = Linear.apply(o, w["o"], "o", "o", "da")
        y = 0.9375 * x + 0.5 * v["rgate"] * (rms(a, v["post_gain"]) * mask[1])
        h = rms(y, v["gain"])
        act = SwiGLU.apply(Linear.apply(h, w["gate"], "h", "gate", "dgate"), Linear.apply(h, w["up"], "h", "up", "dup"))
        z = y + Linear.apply(act, w["down"], "act", "down", "dz")
        names = ["w_" + n for n in w] + list(v) + ["e"]
        grads = torch.autograd.grad(z, list(w.values()) + list(v.values()) + [e], self.dz.double())
        self.seen = seen
        return {**dict(zip(names, grads)), **{n: t.detach() for n, t in dict(x=x, o=o, y=y, h=h, act=act, z=z).items()}}


@pytest.mark.parametrize("dtype,lens,d,H,Hkv,dh,f,grad", [("fp32", [20, 13, 0, 30], 96, 4, 2, 32, 100, "e4m3"), ("fp32", [33, 1, 64], 130, 3, 1, 64, 72, "e5m2"),
                                                         ("bf16", [70, 65, 129, 30], 192, 6, 2, 64, 264, "e5m2"), ("bf16", [300, 40, 200], 256, 4, 1, 128, 712, "e4m3")])
def test_layer(dtype, lens, d, H, Hkv, dh, f, grad):
    """Relative 2-norms.  Between two stored matrices there are at most seven results (a product, the rotation, attention with P and dS inside, the norm's two, and a
    residual), each rounded once, and sums of up to 712 terms in 32 bits; the matrix cores' cut adds 1.2e-5 of a product's norm, taken as 2^-14."""
    print(f"fp8 layer {dtype} lens={lens} d={d} H={H} Hkv={Hkv} dh={dh} f={f} {grad}", flush=True)
    s = _Layer(dtype, lens, d, H, Hkv, dh, f, grad)
    got = s.run()
    want = s.reference()
    tol = 7 * 712 * 2.0 ** -24 if dtype == "fp32" else 7 * (2.0 ** -8 + 2.0 ** -14)
    for n in want:
        rel = float((got[n] - want[n]).norm() / want[n].norm())
        print(f"  {n}: {rel:.2e}", flush=True)
        assert rel <= tol, (n, rel)
    # what the stored gradients stand for is what they were stored from, to half a step of 2^-3 (e4m3) or 2^-2 (e5m2) of an element, or of the smallest normal
    # number at 2^-14 and less of a block's largest (both forms' smallest steps are below 2^-16 of it)
    for n, dy in s.seen.items():
        top = dy.abs().amax(1, keepdim=True)
        step = {"e4m3": 2.0 ** -4, "e5m2": 2.0 ** -3}[grad]
        off = (s.kept[n] - dy).abs() - (step * dy.abs() + (2.0 ** -16 + 2 * tol) * top)
        assert off.max() <= 0, (n, float(off.max()))


def test_layer_twice_gives_the_same_bits():
    import torch
    s = _Layer("bf16", [70, 65, 129, 30], 192, 6, 2, 64, 264, "e4m3")
    first = {n: t.clone() for n, t in s.run().items()}
    for n, t in s.run().items():
        assert torch.equal(first[n], t), n
