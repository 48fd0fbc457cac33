"""The operators of fine-tuning on packed sequences, as cases that can be timed and checked.

A batch of examples of different lengths lies in memory one sequence behind the other, without padding.  Three operators
belong to its training step:

  attention   causal self-attention of every sequence over itself, query heads in groups that share a key and value head,
              q | k | v side by side in a row; forward alone, or forward and backward;
  checkpoint  activations kept from the forward to the backward pass in 8 bits: blocks of 32 neighbours of a row share a
              power of two and keep eight bits each.  Stored and read back, or as the input of an activation (GELU in the
              tanh form; SwiGLU of a gate and an up half) whose gradient and recomputed output come from the eight bits;
  preference  the paired loss of preference tuning: sequences 2 i and 2 i + 1 are a preferred and a rejected answer, the loss
              of a pair is -(1 - s) log sigmoid(beta h) - s log sigmoid(-beta h) with h the difference of their summed log
              probabilities, each less the reference model's; forward alone, or with the gradient of the logits.

`run` computes them with plain torch operations in 32 bits, or (`own`) through the library.  Widths are those of the
repository's workloads (tiny GPT in fp32; GPT-2 small, Llama 7B and 30B in bf16), the query heads in groups.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = 32                 # neighbours of a row that share a power of two in an 8-bit checkpoint
MIN_EXP = -120             # smallest power: the values stay normal numbers of 32 bits


def _attention(name, dtype, H, Hkv, dh, lens, train=True):
    return dict(name=name, kind="attention", dtype=dtype, H=H, Hkv=Hkv, dh=dh, lens=lens, train=train)


def _checkpoint(name, dtype, act, rows, cols):
    return dict(name=name, kind="checkpoint", dtype=dtype, act=act, rows=rows, cols=cols)


def _preference(name, dtype, V, lens, prompts, beta=0.1, smoothing=0.0, train=True):
    return dict(name=name, kind="preference", dtype=dtype, V=V, lens=lens, prompts=prompts, beta=beta, smoothing=smoothing, train=train)


def listed():
    return [
        # a few short prompts at GPT-2-small widths, evaluated: the time of a launch is what counts
        _attention("attention_short_prompts", "bf16", 12, 4, 64, "1 45 17 33", train=False),
        # a training batch of 8192 tokens at GPT-2-small widths: many documents, most of them short
        _attention("attention_gpt2_small", "bf16", 12, 4, 64, "1024 777 64 513 1024 31 300 1 888 640 129 450 975 260 96 511 509"),
        # a training batch at Llama-7B widths with eight key heads, packed from long and short documents
        _attention("attention_llama_7b", "bf16", 32, 8, 128, "2048 1531 257 2011 40 1024 640 641"),
        # two long prompts at Llama-30B widths, thirteen query heads to a key head, evaluated
        _attention("attention_llama_30b_prompts", "bf16", 52, 4, 128, "4096 3211", train=False),
        # fp32 training at the tiny workloads' head size, odd lengths
        _attention("attention_ragged_fp32", "fp32", 4, 2, 32, "333 64 190 1 257 31"),
        # the inputs of a linear layer of Llama 7B, stored in the forward pass and read back for its weight gradient
        _checkpoint("checkpoint_llama_7b_inputs", "bf16", "none", 8192, 4096),
        # SwiGLU of Llama 7B on a whole batch: output and checkpoint, then both gradients and the output again
        _checkpoint("checkpoint_llama_7b_swiglu", "bf16", "swiglu", 8192, 11008),
        # GELU of the tiny GPT: the smallest call
        _checkpoint("checkpoint_tiny_gelu", "fp32", "gelu", 128, 512),
        # a width that is no multiple of a block, an odd number of rows
        _checkpoint("checkpoint_ragged_swiglu", "bf16", "swiglu", 1021, 2730),
        # two pairs at the tiny GPT's vocabulary
        _preference("preference_tiny_fp32", "fp32", 1024, "64 41 33 64", "20 20 9 9"),
        # pairs at GPT-2 small's odd vocabulary, half of a sequence its prompt, label smoothing
        _preference("preference_gpt2_small", "bf16", 50257, "1024 777 513 640 129 450 300 260", "400 400 256 256 64 64 3 3", smoothing=0.1),
        # a batch of 8192 tokens at Llama 7B's vocabulary
        _preference("preference_llama_7b", "bf16", 32000, "2048 1531 1024 2011 257 640 40 641", "300 300 512 512 100 100 0 0"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(ns):
    return " ".join(str(n) for n in ns)


def _ints(text):
    return [int(n) for n in text.split()]


def draw(rng):
    kind = rng.choice(["attention", "checkpoint", "preference"])
    if kind == "attention":
        dtype, dh = rng.choice([("bf16", 64), ("bf16", 128), ("bf16", 64), ("bf16", 128), ("bf16", 32), ("fp32", 32), ("fp32", 64)])
        fast = dtype == "bf16" and dh > 32
        while True:
            Hkv, group = _log_uniform(rng, 1, 12 if fast else 4), rng.choice([1, 2, 3, 4, 5, 7, 8])
            lens = [_log_uniform(rng, 1, 4096 if fast else 600) for _ in range(_log_uniform(rng, 1, 24))]
            if sum(n * n for n in lens) * Hkv * group * dh <= (52 * 2.7e7 * 128 / 3.5 if fast else 5e8) and sum(lens) <= 8192 and Hkv * group <= 52:
                break
        c = _attention("", dtype, Hkv * group, Hkv, dh, _text(lens), rng.random() < 0.75)
    elif kind == "checkpoint":
        act = rng.choice(["none", "gelu", "swiglu"])
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        while True:
            rows, cols = _log_uniform(rng, 1, 8192), _log_uniform(rng, 8, 11008)
            cols = cols if rng.random() < 0.5 else max(8, cols // 8 * 8)
            if rows * cols <= 8192 * 11008 // 2:
                break
        c = _checkpoint("", dtype, act, rows, cols)
    else:
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        while True:
            V = _log_uniform(rng, 500, 50257)
            lens, prompts = [], []
            for _ in range(_log_uniform(rng, 1, 16)):
                p = rng.choice([0, _log_uniform(rng, 1, 400)])
                lens += [p + _log_uniform(rng, 1, 1500) for _ in range(2)]
                prompts += [p, p]
            if sum(lens) * V <= (8192 if dtype == "bf16" else 4096) * 32000 and sum(lens) <= 16384:
                break
        c = _preference("", dtype, V, _text(lens), _text(prompts), rng.choice([0.05, 0.1, 0.5]), rng.choice([0.0, 0.0, 0.1]), rng.random() < 0.75)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _up8(n):
    return (n + 7) // 8 * 8


def _normal(g, shape, dtype, std=1.0):
    return (torch.randn(shape, device=DEV, generator=g) * std).to(TYPES[dtype])


def _offsets(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _attention_inputs(c, seed):
    g = _gen(seed)
    rows, dh = sum(_ints(c["lens"])), c["dh"]
    qkv = _normal(g, (rows, (c["H"] + 2 * c["Hkv"]) * dh), c["dtype"])
    do = _normal(g, (rows, c["H"] * dh), c["dtype"], 1e-2) if c["train"] else None
    return qkv, do


def _checkpoint_inputs(c, seed):
    """Values of a norm's output or of a linear layer in front of an activation: normal, a few columns a hundred times as large."""
    g = _gen(seed)
    rows, n = c["rows"], c["cols"]
    x = torch.zeros((rows, 2 if c["act"] == "swiglu" else 1, _up8(n)), device=DEV, dtype=TYPES[c["dtype"]])
    size = torch.ones((x.shape[1], n), device=DEV)
    size[:, torch.randint(0, n, (max(1, n // 500),), device=DEV, generator=g)] = 100.0 if c["act"] == "none" else 4.0
    x[:, :, :n] = (torch.randn((rows, x.shape[1], n), device=DEV, generator=g) * size).to(x.dtype)
    dy = None
    if c["act"] != "none":
        dy = torch.zeros((rows, _up8(n)), device=DEV, dtype=x.dtype)
        dy[:, :n] = _normal(g, (rows, n), c["dtype"], 1e-2)
    return x, dy


def _preference_inputs(c, seed):
    """Logits in which the label is likelier than most tokens, and a reference a little off the policy on every sequence."""
    g = _gen(seed)
    lens, prompts, V = _ints(c["lens"]), _ints(c["prompts"]), c["V"]
    rows = sum(lens)
    logits = torch.zeros((rows, _up8(V)), device=DEV, dtype=TYPES[c["dtype"]])
    labels = torch.randint(0, V, (rows,), device=DEV, generator=g)
    logits[:, :V] = _normal(g, (rows, V), c["dtype"], 2.0)
    at = torch.arange(rows, device=DEV)
    logits[at, labels] += 8.0
    logp = torch.empty(rows, device=DEV, dtype=torch.float64)
    for r in range(0, rows, 1024):
        part = logits[r:r + 1024, :V].float()
        logp[r:r + 1024] = (part.gather(1, labels[r:r + 1024, None])[:, 0] - torch.logsumexp(part, 1)).double()
    noise = torch.randn(len(lens), device=DEV, generator=g, dtype=torch.float64) * 4.0
    ref, r = [], 0
    for n, p in zip(lens, prompts):
        labels[r:r + min(p, n)] = -1
        ref.append(logp[r + min(p, n):r + n].sum())
        r += n
    return logits, labels.to(torch.int32), (torch.stack(ref) + noise).float()


class _Attention:
    def __init__(self, c, seed):
        self.qkv, self.do = _attention_inputs(c, seed)
        self.lens = _ints(c["lens"])
        if own:
            import paper_2506_06472_amd as tio
            H, dh, rows = c["H"], c["dh"], self.qkv.shape[0]
            self.packing = tio.tio_packing_build(_offsets(self.lens), c["dtype"], H, c["Hkv"], dh)
            self.packed = torch.from_numpy(self.packing.export()["data"]).to(DEV)
            self.o = torch.empty((rows, H * dh), device=DEV, dtype=self.qkv.dtype)
            self.lse = torch.empty((H, rows), device=DEV)
            if c["train"]:
                self.dqkv = torch.empty_like(self.qkv)
                self.work = torch.empty(tio.tio_op_attention_packed_work(self.packing), device=DEV, dtype=torch.uint8)

    def run_own(self, c):
        import paper_2506_06472_amd as tio
        stream = torch.cuda.current_stream().cuda_stream
        ld, ldo = self.qkv.stride(0), self.o.stride(0)
        tio.tio_op_attention_packed(stream, self.packing, self.packed.data_ptr(), self.qkv.data_ptr(), ld, self.o.data_ptr(), ldo,
                                    self.lse.data_ptr())
        if not c["train"]:
            return {"o": self.o, "lse": self.lse}
        tio.tio_op_attention_packed_bwd(stream, self.packing, self.packed.data_ptr(), self.qkv.data_ptr(), ld, self.o.data_ptr(),
                                        self.do.data_ptr(), ldo, self.lse.data_ptr(), self.work.data_ptr(), self.dqkv.data_ptr())
        return {"o": self.o, "lse": self.lse, "dqkv": self.dqkv}

    def run_plain(self, c):
        H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
        G, rows, dt = H // Hkv, self.qkv.shape[0], self.qkv.dtype
        scale = 1.0 / math.sqrt(dh)
        o = torch.empty((rows, H, dh), device=DEV, dtype=dt)
        lse = torch.empty((H, rows), device=DEV)
        dqkv = torch.empty((rows, H + 2 * Hkv, dh), device=DEV, dtype=dt) if c["train"] else None
        x = self.qkv.view(rows, H + 2 * Hkv, dh)
        r = 0
        for n in self.lens:
            if n == 0:
                continue
            mask = torch.arange(n, device=DEV)[None, :] > torch.arange(n, device=DEV)[:, None]
            step = max(1, min(Hkv, (1 << 27) // (n * n * G)))
            for h in range(0, Hkv, step):
                e = min(Hkv, h + step)
                q = x[r:r + n, h * G:e * G].float().transpose(0, 1).reshape(e - h, G * n, dh)          # a group's heads below one another
                k = x[r:r + n, H + h:H + e].float().transpose(0, 1).contiguous()
                v = x[r:r + n, H + Hkv + h:H + Hkv + e].float().transpose(0, 1).contiguous()
                s = torch.matmul(q, k.transpose(1, 2).contiguous()).view(e - h, G, n, n) * scale
                s.masked_fill_(mask, -math.inf)
                m = s.amax(-1, keepdim=True)
                p = torch.exp_(s - m)
                total = p.sum(-1, keepdim=True)
                p /= total
                p = p.view(e - h, G * n, n)
                ob = torch.matmul(p, v)
                o[r:r + n, h * G:e * G] = ob.view((e - h) * G, n, dh).transpose(0, 1).to(dt)
                lse[h * G:e * G, r:r + n] = (m + torch.log(total)).view((e - h) * G, n)
                if c["train"]:
                    g = self.do.view(rows, H, dh)[r:r + n, h * G:e * G].float().transpose(0, 1).reshape(e - h, G * n, dh)
                    ds = torch.matmul(g, v.transpose(1, 2).contiguous())
                    ds -= (g * ob).sum(-1, keepdim=True)
                    ds *= p
                    dqkv[r:r + n, h * G:e * G] = (torch.matmul(ds, k) * scale).view((e - h) * G, n, dh).transpose(0, 1).to(dt)
                    dqkv[r:r + n, H + h:H + e] = (torch.matmul(ds.transpose(1, 2).contiguous(), q) * scale).transpose(0, 1).to(dt)
                    dqkv[r:r + n, H + Hkv + h:H + Hkv + e] = torch.matmul(p.transpose(1, 2).contiguous(), g).transpose(0, 1).to(dt)
            r += n
        out = {"o": o.view(rows, H * dh), "lse": lse}
        if c["train"]:
            out["dqkv"] = dqkv.view(rows, -1)
        return out


def _plain_round_trip(x):
    """[rows, n] in 32 bits -> the values that eight bits and a power of two for each block stand for."""
    rows, n = x.shape
    full = (n + BLOCK - 1) // BLOCK * BLOCK
    b = torch.nn.functional.pad(x, (0, full - n)).view(rows, full // BLOCK, BLOCK)
    top = b.abs().amax(-1, keepdim=True)
    e = ((top.view(torch.int32) >> 23) - 127).clamp(min=MIN_EXP)                   # floor(log2), from the bits
    up = ((6 - e + 127) << 23).view(torch.float32)                                 # 2^(6 - e) and its inverse, exact
    down = ((e - 6 + 127) << 23).view(torch.float32)
    v = torch.round(b * up).clamp(-127.0, 127.0) * down
    v = torch.where(torch.isfinite(top), v, torch.full_like(v, math.nan))
    return v.view(rows, full)[:, :n]


class _Checkpoint:
    def __init__(self, c, seed):
        self.x, self.dy = _checkpoint_inputs(c, seed)
        if own:
            import paper_2506_06472_amd as tio
            rows, n = c["rows"], c["cols"]
            need = tio.tio_ckpt8_bytes(rows, n)                                        # of SwiGLU: the gate half's, then the up half's
            self.kept = torch.empty(need * self.x.shape[1], device=DEV, dtype=torch.uint8)
            self.dx = torch.empty_like(self.x)
            if c["act"] != "none":
                self.y = torch.empty_like(self.dy)
                self.again = torch.empty_like(self.dy)

    def run_own(self, c):
        import paper_2506_06472_amd as tio
        rows, n, dt, act = c["rows"], c["cols"], c["dtype"], c["act"]
        stream = torch.cuda.current_stream().cuda_stream
        ldx = self.x.stride(0)
        if act == "none":
            tio.tio_op_ckpt8_store(stream, dt, rows, n, self.x.data_ptr(), ldx, self.kept.data_ptr())
            tio.tio_op_ckpt8_load(stream, dt, rows, n, self.kept.data_ptr(), self.dx.data_ptr(), ldx)
            return {"x": self.dx[:, 0, :n]}
        ldy, two = self.dy.stride(0), act == "swiglu"
        tio.tio_op_act_ckpt8(stream, dt, act, rows, n, self.x.data_ptr(), self.x[:, 1].data_ptr() if two else 0, ldx, self.y.data_ptr(), ldy,
                             self.kept.data_ptr())
        tio.tio_op_act_ckpt8_bwd(stream, dt, act, rows, n, self.kept.data_ptr(), self.dy.data_ptr(), ldy, self.dx.data_ptr(),
                                 self.dx[:, 1].data_ptr() if two else 0, ldx, self.again.data_ptr(), ldy)
        return {"y": self.y[:, :n], "dx": self.dx[:, :, :n], "again": self.again[:, :n]}

    def run_plain(self, c):
        n, act, dt = c["cols"], c["act"], self.x.dtype
        x = [self.x[:, i, :n].float() for i in range(self.x.shape[1])]
        kept = [_plain_round_trip(t) for t in x]
        if act == "none":
            return {"x": kept[0].to(dt)}
        dy = self.dy[:, :n].float()
        if act == "swiglu":
            y = x[0] / (1.0 + torch.exp(-x[0])) * x[1]
            gate, up = kept
            sg = 1.0 / (1.0 + torch.exp(-gate))
            dx = torch.stack((dy * up * (sg + gate * sg * (1.0 - sg)), dy * gate * sg), 1)
            again = gate * sg * up
        else:
            a, b = math.sqrt(2.0 / math.pi), 0.044715
            x, k = x[0], kept[0]
            y = 0.5 * x * (1.0 + torch.tanh(a * (x + b * x * x * x)))
            t = torch.tanh(a * (k + b * k * k * k))
            dx = (dy * (0.5 * (1.0 + t) + 0.5 * k * (1.0 - t * t) * a * (1.0 + 3.0 * b * k * k)))[:, None]
            again = 0.5 * k * (1.0 + t)
        return {"y": y.to(dt), "dx": dx.to(dt), "again": again.to(dt)}


class _Preference:
    def __init__(self, c, seed):
        self.logits, self.labels, self.ref = _preference_inputs(c, seed)
        self.lens = _ints(c["lens"])
        if own:
            import paper_2506_06472_amd as tio
            pairs = len(self.lens) // 2
            self.packing = tio.tio_packing_build(_offsets(self.lens))
            self.packed = torch.from_numpy(self.packing.export()["data"]).to(DEV)
            self.seq = torch.empty(2 * pairs, device=DEV)
            self.losses = torch.empty(pairs, device=DEV)
            self.loss = torch.empty(1, device=DEV)
            self.work = torch.empty(tio.tio_op_preference_loss_work(self.packing), device=DEV, dtype=torch.uint8)
            self.dlogits = torch.empty_like(self.logits) if c["train"] else None

    def run_own(self, c):
        import paper_2506_06472_amd as tio
        stream = torch.cuda.current_stream().cuda_stream
        tio.tio_op_preference_loss(stream, c["dtype"], self.packing, self.packed.data_ptr(), c["V"], self.logits.data_ptr(),
                                   self.logits.stride(0), self.labels.data_ptr(), self.ref.data_ptr(), c["beta"], c["smoothing"],
                                   self.seq.data_ptr(), self.losses.data_ptr(), self.loss.data_ptr(), self.work.data_ptr(),
                                   self.dlogits.data_ptr() if c["train"] else 0)
        out = {"seq": self.seq, "losses": self.losses, "loss": self.loss}
        if c["train"]:
            out["dlogits"] = self.dlogits[:, :c["V"]]
        return out

    def run_plain(self, c):
        V, beta, s, rows = c["V"], c["beta"], c["smoothing"], self.logits.shape[0]
        pairs = len(self.lens) // 2
        counted = self.labels >= 0
        at = self.labels.clamp(min=0).long()
        lse = torch.empty(rows, device=DEV)
        logp = torch.empty(rows, device=DEV, dtype=torch.float64)
        for r in range(0, rows, 2048):
            x = self.logits[r:r + 2048, :V].float()
            m = x.amax(1)
            log_sum = torch.log(torch.exp(x - m[:, None]).sum(1))
            lse[r:r + 2048] = m + log_sum
            picked = x.gather(1, at[r:r + 2048, None])[:, 0]
            logp[r:r + 2048] = (picked.double() - m.double()) - log_sum.double()          # sums over a sequence lose in 32 bits
        logp = torch.where(counted, logp, torch.zeros_like(logp))
        offsets = _offsets(self.lens)
        seq = torch.stack([logp[a:b].sum() for a, b in zip(offsets, offsets[1:])])
        h = seq - self.ref.double()
        z = beta * (h[0::2] - h[1::2])
        log_sigmoid = torch.minimum(z, torch.zeros_like(z)) - torch.log1p(torch.exp(-z.abs()))
        losses = -(1.0 - s) * log_sigmoid - s * (log_sigmoid - z)
        out = {"seq": seq.float(), "losses": losses.float(), "loss": losses.mean().float().view(1)}
        if c["train"]:
            up = 1.0 / (1.0 + torch.exp(z))                                                # sigmoid(-z)
            w = (-beta / pairs * ((1.0 - s) * up - s * (1.0 - up))).float()
            w = torch.stack((w, -w), 1).view(-1)
            of_row = torch.repeat_interleave(w, torch.tensor(self.lens, device=DEV), output_size=rows) * counted
            d = torch.empty((rows, V), device=DEV, dtype=self.logits.dtype)
            for r in range(0, rows, 2048):
                wr = of_row[r:r + 2048, None]
                g = torch.exp(self.logits[r:r + 2048, :V].float() - lse[r:r + 2048, None])
                g = -wr * g
                g.scatter_add_(1, at[r:r + 2048, None], wr)
                d[r:r + 2048] = g.to(d.dtype)
            out["dlogits"] = d
        return out


def prepare(case, seed):
    state = {"attention": _Attention, "checkpoint": _Checkpoint, "preference": _Preference}[case["kind"]](case, seed)
    return case, state


def run(state):
    case, s = state
    return s.run_own(case) if own else s.run_plain(case)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "attention":
        lens, H, Hkv, dh = _ints(c["lens"]), c["H"], c["Hkv"], c["dh"]
        rows = sum(lens)
        flops = sum(n * (n + 1) // 2 for n in lens) * H * dh * 4.0                 # two products of the visible pairs
        nbytes = rows * ((2 * H + 2 * Hkv) * dh * e + H * 4)
        if c["train"]:
            flops *= 3.5
            nbytes += rows * (2 * H + 2 * Hkv) * dh * e                            # dO in, the gradients out
        return {"bytes": nbytes, "flops": flops}
    if c["kind"] == "checkpoint":
        rows, n, act = c["rows"], c["cols"], c["act"]
        halves = 2 if act == "swiglu" else 1
        kept = rows * halves * (n + (n + BLOCK - 1) // BLOCK)                      # written by one pass, read by the other
        elems = rows * halves * n * 2 + (rows * n * 3 if act != "none" else 0)
        return {"bytes": elems * e + 2 * kept, "flops": rows * halves * n * 4.0 + (rows * n * 30.0 if act != "none" else 0.0)}
    lens, prompts, V = _ints(c["lens"]), _ints(c["prompts"]), c["V"]
    counted = sum(n - min(n, p) for n, p in zip(lens, prompts))
    nbytes = counted * V * e + sum(lens) * 4
    if c["train"]:
        nbytes += sum(lens) * V * e                                                # rows of prompts are written too: zeros
    return {"bytes": nbytes, "flops": counted * V * (8.0 if c["train"] else 4.0)}


# ------------------------------------------------------------------ the same in 64 bits
def _exact_attention(c, seed):
    qkv, do = _attention_inputs(c, seed)
    H, Hkv, dh, rows = c["H"], c["Hkv"], c["dh"], qkv.shape[0]
    G = H // Hkv
    o = torch.empty((rows, H * dh), device=DEV, dtype=torch.float64)
    lse = torch.empty((H, rows), device=DEV, dtype=torch.float64)
    dqkv = torch.zeros((rows, (H + 2 * Hkv) * dh), device=DEV, dtype=torch.float64) if c["train"] else None
    first = 0
    for n in _ints(c["lens"]):
        part = slice(first, first + n)
        first += n
        seen = torch.ones((n, n), device=DEV, dtype=torch.bool).tril()
        for h in range(H):                                                         # one query head at a time
            cols = [slice(i * dh, (i + 1) * dh) for i in (h, H + h // G, H + Hkv + h // G)]
            q, k, v = (qkv[part, s].double().contiguous().requires_grad_(c["train"]) for s in cols)
            s = torch.where(seen, (q @ k.t().contiguous()) * dh ** -0.5, -math.inf)
            l = torch.logsumexp(s, 1)
            y = torch.exp(s - l[:, None]) @ v
            o[part, cols[0]], lse[h, part] = y.detach(), l.detach()
            if c["train"]:
                grads = torch.autograd.grad(y, (q, k, v), do[part, cols[0]].double())
                for col, g in zip(cols, grads):
                    dqkv[part, col] += g
    out = {"o": o, "lse": lse}
    if c["train"]:
        out["dqkv"] = dqkv
    return out


def _exact_kept(x):
    rows, n = x.shape
    out = torch.empty_like(x)
    for c in range(0, n, 1 << 12):                                                 # whole blocks at a time
        part = x[:, c:c + (1 << 12)]
        pieces = torch.zeros((rows, (part.shape[1] + BLOCK - 1) // BLOCK * BLOCK), device=x.device, dtype=x.dtype)
        pieces[:, :part.shape[1]] = part
        pieces = pieces.unflatten(1, (-1, BLOCK))
        exponent = torch.frexp(pieces.abs().amax(2, keepdim=True))[1].to(torch.int64) - 1
        exponent = torch.where(pieces.abs().amax(2, keepdim=True) == 0, MIN_EXP, exponent).clamp(min=MIN_EXP)
        unit = ((exponent - 6 + 1023) << 52).view(torch.float64)
        out[:, c:c + (1 << 12)] = (torch.clip(torch.round(pieces / unit), -127, 127) * unit).flatten(1)[:, :part.shape[1]]
    return out


def _exact_checkpoint(c, seed):
    x, dy = _checkpoint_inputs(c, seed)
    n, act = c["cols"], c["act"]
    x = x[:, :, :n].double()
    kept = torch.stack([_exact_kept(x[:, i]) for i in range(x.shape[1])], 1)
    if act == "none":
        return {"x": kept[:, 0]}

    def f(t):
        if act == "gelu":
            return torch.nn.functional.gelu(t[:, 0], approximate="tanh")
        return torch.nn.functional.silu(t[:, 0]) * t[:, 1]
    y = f(x)
    del x
    kept.requires_grad_()
    again = f(kept)
    (dx,) = torch.autograd.grad(again, kept, dy[:, :n].double())
    return {"y": y, "dx": dx, "again": again.detach()}


def _exact_preference(c, seed):
    logits, labels, ref = _preference_inputs(c, seed)
    V, rows = c["V"], logits.shape[0]
    lens = _ints(c["lens"])
    pair_of = torch.repeat_interleave(torch.arange(len(lens), device=DEV), torch.tensor(lens, device=DEV))
    counted = (labels >= 0).double()
    at = labels.clamp(min=0).long()
    logp = torch.empty(rows, device=DEV, dtype=torch.float64)
    for r in range(0, rows, 512):
        logp[r:r + 512] = -torch.nn.functional.cross_entropy(logits[r:r + 512, :V].double(), at[r:r + 512], reduction="none")
    seq = torch.zeros(len(lens), device=DEV, dtype=torch.float64).index_add_(0, pair_of, logp * counted).requires_grad_()
    margin = ((seq - ref.double()).view(-1, 2) * torch.tensor([1.0, -1.0], device=DEV, dtype=torch.float64)).sum(1) * c["beta"]
    ls = torch.nn.functional.logsigmoid
    losses = -(1 - c["smoothing"]) * ls(margin) - c["smoothing"] * ls(-margin)
    out = {"seq": seq.detach(), "losses": losses.detach(), "loss": losses.mean().detach().view(1)}
    if c["train"]:
        (w,) = torch.autograd.grad(losses.mean(), seq)
        w = w[pair_of] * counted
        d = torch.empty((rows, V), device=DEV, dtype=torch.float64)
        for r in range(0, rows, 512):
            p = torch.softmax(logits[r:r + 512, :V].double(), 1)
            p[torch.arange(p.shape[0], device=DEV), at[r:r + 512]] -= 1.0
            d[r:r + 512] = -w[r:r + 512, None] * p
        out["dlogits"] = d
    return out


def exact(case, seed):
    """What `run` returns, from the definitions in 64 bits."""
    return {"attention": _exact_attention, "checkpoint": _exact_checkpoint, "preference": _exact_preference}[case["kind"]](case, seed)
