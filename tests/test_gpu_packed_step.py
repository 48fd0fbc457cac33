"""GPU: the operators on packed batches together, as a preference-tuning step has them: one decoder layer (attention over packed pairs, SwiGLU whose
inputs are kept in 8 bits) and a head with the paired loss, forward and backward, products through tio_op_gemm; every gradient against autograd in
64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


class _Step:
    """The step through the library: outputs in self.out, what the checkpoints stand for in self.kept."""

    def __init__(self, dtype, lens, prompts, d, H, Hkv, dh, f, V, seed=0):
        import torch
        self.dtype, self.t = dtype, torch.bfloat16 if dtype == "bf16" else torch.float32
        self.lens, self.d, self.H, self.Hkv, self.dh, self.f, self.V = lens, d, H, Hkv, dh, f, V
        self.S = sum(lens)
        g = torch.Generator().manual_seed(seed)
        shapes = dict(qkv=((H + 2 * Hkv) * dh, d), o=(d, H * dh), gate=(f, d), up=(f, d), down=(d, f), head=(V, d))
        self.w = {k: (torch.randn(s, generator=g) / np.sqrt(s[1])).to(self.t) for k, s in shapes.items()}
        self.x = torch.randn((self.S, d), generator=g).to(self.t)
        self.labels = torch.randint(0, V, (self.S,), generator=g)
        r = 0
        for n, p in zip(lens, prompts):
            self.labels[r:r + p] = -100
            r += n
        self.ref = -torch.rand(len(lens), generator=g) * 20 - 2 * torch.tensor(lens)

    def run(self, beta=0.1, smoothing=0.1):
        import torch
        import paper_2506_06472_amd as tio
        import packedlib as pl
        S, d, f, V, dt, t = self.S, self.d, self.f, self.V, self.dtype, self.t
        up8 = lambda n: (n + 7) // 8 * 8

        def new(rows, cols):
            return torch.full((rows, up8(cols)), float("nan"), device="cuda", dtype=t)

        def put(a):
            b = torch.zeros((a.shape[0], up8(a.shape[1])), device="cuda", dtype=t)
            b[:, :a.shape[1]] = a.cuda()
            return b
        w, x = {k: put(v) for k, v in self.w.items()}, put(self.x)
        P = lambda b: 0 if b is None else b.data_ptr()

        def product(a_km, b_km, M, N, K, a, b, c, resid=None):
            tio.tio_op_gemm(0, dt, a_km, b_km, M, N, K, P(a), a.stride(0), P(b), b.stride(0), 0, P(resid), 0 if resid is None else resid.stride(0), P(c), c.stride(0))
            return c
        linear = lambda a, name, n, k, resid=None: product(0, 0, S, n, k, a, w[name], new(S, n), resid)
        back = lambda dy, name, n, k, resid=None: product(0, 1, S, k, n, dy, w[name], new(S, k), resid)     # dy W
        weight = lambda dy, a, n, k: product(1, 1, n, k, S, dy, a, new(n, k))                               # dy^T a
        pk, dev = pl.packing(self.lens, dt, self.H, self.Hkv, self.dh)
        wide, hd = (self.H + 2 * self.Hkv) * self.dh, self.H * self.dh
        kx = torch.zeros(tio.tio_ckpt8_bytes(S, d), device="cuda", dtype=torch.uint8)
        half = tio.tio_ckpt8_bytes(S, f)
        kgu = torch.zeros(2 * half, device="cuda", dtype=torch.uint8)
        # forward
        tio.tio_op_ckpt8_store(0, dt, S, d, P(x), x.stride(0), P(kx))
        qkv = linear(x, "qkv", wide, d)
        o, lse = new(S, hd), torch.empty((self.H, S), device="cuda")
        tio.tio_op_attention_packed(0, pk, P(dev), P(qkv), qkv.stride(0), P(o), o.stride(0), P(lse))
        h = linear(o, "o", d, hd, x)
        gate, up = linear(h, "gate", f, d), linear(h, "up", f, d)
        y = new(S, f)
        tio.tio_op_act_ckpt8(0, dt, "swiglu", S, f, P(gate), P(up), gate.stride(0), P(y), y.stride(0), P(kgu))
        z = linear(y, "down", d, f, h)
        logits = linear(z, "head", V, d)
        labels, ref = self.labels.int().cuda(), self.ref.cuda()
        seq, losses, loss = torch.empty(len(self.lens), device="cuda"), torch.empty(len(self.lens) // 2, device="cuda"), torch.empty(1, device="cuda")
        work = torch.empty(tio.tio_op_preference_loss_work(pk), device="cuda", dtype=torch.uint8)
        tio.tio_op_preference_loss(0, dt, pk, P(dev), V, P(logits), logits.stride(0), P(labels), P(ref), beta, smoothing, P(seq), P(losses), P(loss), P(work),
                                   P(logits))
        dlogits = logits
        # backward
        out = dict(loss=loss, seq=seq, head=weight(dlogits, z, V, d))
        dz = back(dlogits, "head", V, d)
        dy = back(dz, "down", d, f)
        dgate, dup, again = new(S, f), new(S, f), new(S, f)
        tio.tio_op_act_ckpt8_bwd(0, dt, "swiglu", S, f, P(kgu), P(dy), dy.stride(0), P(dgate), P(dup), dgate.stride(0), P(again), again.stride(0))
        out["down"] = weight(dz, again, d, f)
        out["gate"], out["up"] = weight(dgate, h, f, d), weight(dup, h, f, d)
        dh = back(dup, "up", f, d, back(dgate, "gate", f, d, dz))
        out["o"] = weight(dh, o, d, hd)
        do, dqkv = back(dh, "o", d, hd), new(S, wide)
        work = torch.empty(tio.tio_op_attention_packed_work(pk), device="cuda", dtype=torch.uint8)
        tio.tio_op_attention_packed_bwd(0, pk, P(dev), P(qkv), qkv.stride(0), P(o), P(do), o.stride(0), P(lse), P(work), P(dqkv))
        x8 = new(S, d)
        tio.tio_op_ckpt8_load(0, dt, S, d, P(kx), P(x8), x8.stride(0))
        out["qkv"] = weight(dqkv, x8, wide, d)
        out["x"] = back(dqkv, "qkv", wide, d, dh)
        kept = {"x": x8}
        for i, name in enumerate(("gate", "up")):
            kept[name] = new(S, f)
            tio.tio_op_ckpt8_load(0, dt, S, f, P(kgu) + i * half, P(kept[name]), kept[name].stride(0))
        torch.cuda.synchronize()
        cols = dict(head=d, down=f, gate=d, up=d, o=hd, qkv=d, x=d)
        self.out = {k: (v if k not in cols else v[:, :cols[k]]).double().cpu() for k, v in out.items()}
        self.kept = {k: v[:, :(d if k == "x" else f)].double().cpu() for k, v in kept.items()}
        self.gate_up = (gate[:, :f].double().cpu(), up[:, :f].double().cpu())
        return self.out


def _reference(s, beta=0.1, smoothing=0.1):
    """The same in 64 bits; where the library takes a checkpoint's values in the backward pass, those it read back."""
    import torch

    class Linear(torch.autograd.Function):
        """a w^T whose weight gradient is that of another input"""
        @staticmethod
        def forward(ctx, a, w, other):
            ctx.save_for_backward(w, other)
            return a @ w.t()

        @staticmethod
        def backward(ctx, g):
            w, other = ctx.saved_tensors
            return g @ w, g.t() @ other, None

    class SwiGLU(torch.autograd.Function):
        """silu(g) u whose gradients are taken at other values"""
        @staticmethod
        def forward(ctx, g, u, kg, ku):
            ctx.save_for_backward(kg, ku)
            return torch.nn.functional.silu(g) * u

        @staticmethod
        def backward(ctx, dy):
            kg, ku = ctx.saved_tensors
            sg = torch.sigmoid(kg)
            return dy * ku * (sg + kg * sg * (1 - sg)), dy * kg * sg, None, None
    w = {k: v.double().requires_grad_() for k, v in s.w.items()}
    x = s.x.double().requires_grad_()
    G = s.H // s.Hkv
    qkv = Linear.apply(x, w["qkv"], s.kept["x"]).view(s.S, s.H + 2 * s.Hkv, s.dh)
    parts, r = [], 0
    for n in s.lens:
        q, k, v = (qkv[r:r + n, a:b].transpose(0, 1) for a, b in ((0, s.H), (s.H, s.H + s.Hkv), (s.H + s.Hkv, s.H + 2 * s.Hkv)))
        k, v = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
        a = (q @ k.transpose(1, 2)) / np.sqrt(s.dh)
        a = a.masked_fill(torch.ones((n, n), dtype=torch.bool).triu(1), -torch.inf)
        parts.append((torch.softmax(a, -1) @ v).transpose(0, 1).reshape(n, -1))
        r += n
    o = torch.cat(parts)
    h = x + o @ w["o"].t()
    y = SwiGLU.apply(h @ w["gate"].t(), h @ w["up"].t(), s.kept["gate"], s.kept["up"])
    z = h + Linear.apply(y, w["down"], torch.nn.functional.silu(s.kept["gate"]) * s.kept["up"])
    logits = z @ w["head"].t()
    counted = s.labels >= 0
    lp = -torch.nn.functional.cross_entropy(logits, s.labels.clamp(min=0), reduction="none") * counted
    seq = torch.stack([p.sum() for p in torch.split(lp, s.lens)])
    m = seq - s.ref.double()
    zed = beta * (m[0::2] - m[1::2])
    ls = torch.nn.functional.logsigmoid
    loss = (-(1 - smoothing) * ls(zed) - smoothing * ls(-zed)).mean()
    names = list(w)
    grads = torch.autograd.grad(loss, [w[n] for n in names] + [x])
    out = dict(zip(names + ["x"], grads))
    out["loss"], out["seq"] = loss.detach().view(1), seq.detach()
    return out


@pytest.mark.parametrize("dtype,lens,prompts,d,H,Hkv,dh,f,V", [("fp32", [20, 13, 9, 30], [5, 5, 0, 0], 96, 4, 2, 32, 100, 301),
                                                              ("fp32", [33, 1, 64, 70], [0, 0, 30, 30], 64, 3, 1, 64, 72, 520),
                                                              ("bf16", [70, 65, 129, 30], [10, 10, 20, 20], 192, 6, 2, 64, 264, 1000),
                                                              ("bf16", [300, 40, 17, 200], [33, 33, 0, 0], 256, 4, 1, 128, 200, 777)])
def test_step(dtype, lens, prompts, d, H, Hkv, dh, f, V):
    """Relative 2-norms.  fp32: sums of up to 520 terms, 520 * 2^-24 at worst for each of six products behind one another.  bf16: the twelve tensors
    between the loss and the first weight are rounded by at most 2^-8 each, and P and dS within attention."""
    import packedlib as pl
    print(f"packed step {dtype} lens={lens} d={d} H={H} Hkv={Hkv} dh={dh} f={f} V={V}", flush=True)
    s = _Step(dtype, lens, prompts, d, H, Hkv, dh, f, V)
    got, want = s.run(), None
    assert np.array_equal(s.kept["x"].numpy(), pl.kept_values(s.x.double().numpy()))
    for name, v in zip(("gate", "up"), s.gate_up):
        assert np.array_equal(s.kept[name].numpy(), pl.kept_values(v.numpy())), name
    want = _reference(s)
    tol = 6 * 520 * 2.0 ** -24 if dtype == "fp32" else 14 * 2.0 ** -8
    for name in want:
        rel = float((got[name] - want[name]).norm() / want[name].norm())
        print(f"  {name}: {rel:.2e}", flush=True)
        assert rel <= tol, (name, rel)


def test_step_twice_gives_the_same_bits():
    import torch
    a = _Step("bf16", [70, 65, 129, 30], [10, 10, 20, 20], 192, 6, 2, 64, 264, 1000)
    first = {k: v.clone() for k, v in a.run().items()}
    for k, v in a.run().items():
        assert torch.equal(first[k], v), k
