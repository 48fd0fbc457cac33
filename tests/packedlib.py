"""Helpers of the tests on packed batches: plain definitions in 64 bits on the host, and marshalling."""
import numpy as np

import paper_2506_06472_amd as tio


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def packing(lens, *heads):
    """(packing, its copy on the GPU)"""
    import torch
    p = tio.tio_packing_build(offsets(lens), *heads)
    return p, torch.from_numpy(p.export()["data"]).cuda()


def attention(lens, H, Hkv, dh, qkv, dO, u):
    """o, lse, dqkv of the definition, and bounds of o's and dqkv's errors, element by element.

    u: twice a rounding of the storage type.  The kernels round the probabilities P and the score gradients dS to it before the second
    product and every result once, and take delta = rowsum(dO * O) from the stored O (in a sequence's first rows not even that):
      |O - ref| <= u (|O| + P|V|)        E_i = u sum_d |dO_id| (|O_id| + (P|V|)_id)        (error of delta_i)
      |dQ - ref| <= u |dQ| + (E (P|K|) + u |dS||K|) / sqrt(dh),  dK likewise with |Q|,  |dV - ref| <= u (|dV| + P^T |dO|)
    dK and dV are sums over the query heads of a group, and so are their bounds (|dK| once more for the sum's own rounding)."""
    G, rows = H // Hkv, int(np.sum(lens))
    x = qkv.astype(np.float64).reshape(rows, H + 2 * Hkv, dh)
    g = dO.astype(np.float64).reshape(rows, H, dh)
    o, lse = np.zeros((rows, H, dh)), np.zeros((H, rows))
    d, ob, db = np.zeros_like(x), np.zeros((rows, H, dh)), np.zeros_like(x)
    rs = 1.0 / np.sqrt(dh)
    first = 0
    for n in lens:
        r = slice(first, first + n)
        first += n
        if n == 0:
            continue
        hidden = np.triu(np.ones((n, n), bool), 1)
        for h in range(H):
            ik, iv = H + h // G, H + Hkv + h // G
            q, k, v, go = x[r, h], x[r, ik], x[r, iv], g[r, h]
            s = np.where(hidden, -np.inf, q @ k.T * rs)
            m = s.max(1, keepdims=True)
            e = np.exp(s - m)
            total = e.sum(1, keepdims=True)
            p = e / total
            lse[h, r] = (m + np.log(total))[:, 0]
            o[r, h] = p @ v
            pv = p @ np.abs(v)
            ob[r, h] = u * (np.abs(o[r, h]) + pv)
            dS = p * (go @ v.T - (go * o[r, h]).sum(1, keepdims=True))
            d[r, h] = dS @ k * rs
            dk, dv = dS.T @ q * rs, p.T @ go
            d[r, ik] += dk
            d[r, iv] += dv
            E = u * (np.abs(go) * (np.abs(o[r, h]) + pv)).sum(1, keepdims=True)
            aS = u * np.abs(dS) + p * E
            db[r, h] = u * np.abs(d[r, h]) + aS @ np.abs(k) * rs
            db[r, ik] += u * np.abs(dk) + aS.T @ np.abs(q) * rs
            db[r, iv] += u * (np.abs(dv) + p.T @ np.abs(go))
    return o.reshape(rows, -1), lse, d.reshape(rows, -1), ob.reshape(rows, -1), db.reshape(rows, -1)


def attention_on(device, lens, H, Hkv, dh, qkv, dO, u):
    """attention() by torch in 64 bits on `device`, for batches that the host would take long over; the same values and bounds as numpy arrays."""
    import torch
    G, rows = H // Hkv, int(np.sum(lens))
    x = torch.from_numpy(np.ascontiguousarray(qkv)).to(device).double().view(rows, H + 2 * Hkv, dh)
    g = torch.from_numpy(np.ascontiguousarray(dO)).to(device).double().view(rows, H, dh)
    rs = 1.0 / np.sqrt(dh)
    o, lse, ob = torch.zeros_like(g), torch.zeros((H, rows), device=device, dtype=torch.float64), torch.zeros_like(g)
    d, db = torch.zeros_like(x), torch.zeros_like(x)
    first = 0
    for n in lens:
        r = slice(first, first + n)
        first += n
        if n == 0:
            continue
        hidden = torch.ones((n, n), device=device, dtype=torch.bool).triu(1)
        for h in range(H):
            ik, iv = H + h // G, H + Hkv + h // G
            q, k, v, go = (t.contiguous() for t in (x[r, h], x[r, ik], x[r, iv], g[r, h]))
            s = (q @ k.t().contiguous() * rs).masked_fill(hidden, -torch.inf)
            l = torch.logsumexp(s, 1, keepdim=True)
            p = torch.exp(s - l)
            pt = p.t().contiguous()
            out, pv = p @ v, p @ v.abs()
            o[r, h], lse[h, r], ob[r, h] = out, l[:, 0], u * (out.abs() + pv)
            dS = p * (go @ v.t().contiguous() - (go * out).sum(1, keepdim=True))
            dst = dS.t().contiguous()
            dq, dk, dv = dS @ k * rs, dst @ q * rs, pt @ go
            d[r, h] = dq
            d[r, ik] += dk
            d[r, iv] += dv
            E = u * (go.abs() * (out.abs() + pv)).sum(1, keepdim=True)
            aS = u * dS.abs() + p * E
            db[r, h] = u * dq.abs() + aS @ k.abs() * rs
            db[r, ik] += u * dk.abs() + aS.t().contiguous() @ q.abs() * rs
            db[r, iv] += u * (dv.abs() + pt @ go.abs())
    return tuple(t.reshape(t.shape[0], -1).cpu().numpy() for t in (o, lse, d, ob, db))


def blocks(lens, H, Hkv, dh):
    """(rows of a forward block, keys of a backward block, blocks of keys that are cut) of a bf16 packing with head size 64 or 128, from its lists: each
    query list covers the batch once in blocks of its size, the list of keys in its."""
    off, G = offsets(lens), H // Hkv
    data = tio.tio_packing_build(off, "bf16", H, Hkv, dh).export()["data"]
    data = data[(len(off) + 3) // 4 * 4:]
    at = [(int(a), n) for a, n in zip(off, lens) if n]

    def queries(i, rows):
        """where the list that starts at word i ends, None if it is not one of blocks of `rows`"""
        want = {(a, n, v) for a, n in at for v in range(0, n * G, rows)}
        got = data[i:i + 4 * len(want)]
        return i + len(got) if len(got) == 4 * len(want) and {tuple(map(int, w[:3])) for w in got.reshape(-1, 4)} == want else None
    found = set()
    for fwd in (64, 128):
        for keys in (64, 128 if dh == 64 else 256):
            end = queries(0, fwd)
            if end is not None and keys != fwd:
                end = queries(end, keys)
            if end is None or (len(data) - end) % 8:
                continue
            rest = data[end:].reshape(-1, 8)
            if {tuple(map(int, w[:3])) for w in rest[rest[:, 6] == 0]} == {(a, n, k) for a, n in at for k in range(0, n, keys)}:
                found.add((fwd, keys, int((rest[:, 6] > 0).sum())))
    assert len(found) == 1, found
    return found.pop()


def run_attention(lens, dtype, H, Hkv, dh, qkv, dO, extra_rows=0, pad=0, pad_o=0, stream=0, packed=None):
    """o, lse, dqkv as torch tensors with everything that is not to be written set to 7: extra rows behind the batch, pad columns."""
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rows, wq, wo = int(np.sum(lens)), (H + 2 * Hkv) * dh, H * dh
    p, dev = packed or packing(lens, dtype, H, Hkv, dh)

    def put(a, width, more):
        out = torch.full((rows + extra_rows, width + more), float("nan"), device="cuda", dtype=t)
        out[:rows, :width] = a if torch.is_tensor(a) else torch.from_numpy(a).cuda().to(t)
        return out
    q, g = put(qkv, wq, pad), put(dO, wo, pad_o)
    o = torch.full((rows + extra_rows, wo + pad_o), 7.0, device="cuda", dtype=t)
    dqkv = torch.full((rows + extra_rows, wq + pad), 7.0, device="cuda", dtype=t)
    lse = torch.full((H * rows + 8,), 7.0, device="cuda")
    need = tio.tio_op_attention_packed_work(p)
    work = torch.full((need + 64,), 255, device="cuda", dtype=torch.uint8)
    torch.cuda.synchronize()
    tio.tio_op_attention_packed(stream, p, dev.data_ptr(), q.data_ptr(), q.stride(0), o.data_ptr(), o.stride(0), lse.data_ptr())
    tio.tio_op_attention_packed_bwd(stream, p, dev.data_ptr(), q.data_ptr(), q.stride(0), o.data_ptr(), g.data_ptr(), o.stride(0), lse.data_ptr(),
                                    work.data_ptr(), dqkv.data_ptr())
    torch.cuda.synchronize()
    assert (work[need:] == 255).all() and (lse[H * rows:] == 7.0).all()
    assert (o[rows:] == 7.0).all() and (o[:, wo:] == 7.0).all(), "o outside its heads and rows"
    assert (dqkv[rows:] == 7.0).all() and (dqkv[:, wq:] == 7.0).all(), "dqkv outside its heads and rows"
    return o[:rows, :wo], lse[:H * rows].view(H, rows), dqkv[:rows, :wq]


def kept_values(x):
    """What an 8-bit checkpoint of the [rows, cols] array stands for."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    b = np.zeros((rows, (cols + 31) // 32 * 32))
    b[:, :cols] = x
    b = b.reshape(rows, -1, 32)
    with np.errstate(all="ignore"):
        top = np.abs(b).max(2, keepdims=True)
        e = np.maximum(np.where(top == 0, -120, np.frexp(np.where(np.isfinite(top), top, 1.0))[1] - 1), -120)
        v = np.clip(np.rint(b * np.exp2(6.0 - e)), -127, 127) * np.exp2(e - 6.0)
    v = np.where(np.isfinite(top), v, np.nan)
    return v.reshape(rows, -1)[:, :cols]
