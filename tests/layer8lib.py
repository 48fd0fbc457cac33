"""Helpers of the tests on layers in 8-bit floating point: definitions in 64 bits on the host, and marshalling."""
import numpy as np

U = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}                     # half a step of a rounding, relative to the value
E32 = 2.0 ** -24
TOP, MANTISSA, LOWEST = {"e4m3": 8, "e5m2": 15}, {"e4m3": 3, "e5m2": 2}, {"e4m3": -6, "e5m2": -14}


def types(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def rounded(x, dtype):
    """float64 -> the nearest numbers of the type, as float64"""
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).to(types(dtype)).double().numpy()


def padded(a, dtype, fill=float("nan"), extra=8):
    """[rows, cols] on the GPU, in rows of the next multiple of eight and `extra` more, which hold `fill`"""
    import torch
    rows, cols = a.shape
    t = torch.full((rows, (cols + 7) // 8 * 8 + extra), fill, device="cuda", dtype=types(dtype))
    t[:, :cols] = torch.from_numpy(np.ascontiguousarray(a)).cuda().to(t.dtype)
    return t


def clean(t, cols, fill, rows=None):
    """columns up to the next eight hold zeros, what is behind them (and rows from `rows` on) `fill`; the values as float64"""
    import torch
    same = torch.isnan if fill != fill else (lambda v: v == fill)
    n = t.shape[0] if rows is None else rows
    up = (cols + 7) // 8 * 8
    assert (t[:n, cols:up] == 0).all() and same(t[:n, up:]).all() and same(t[n:]).all()
    return t[:n, :cols].double().cpu().numpy()


def untouched(t, cols, fill):
    """a vector [1, ..]: everything behind the last column holds `fill`; the values as float64"""
    assert (t[:, cols:] == fill).all()
    return t[:, :cols].double().cpu().numpy()


def stored(x, form, tiles=False):
    """The values that a stored matrix [rows, cols] stands for, in blocks along the columns."""
    rows, cols = x.shape
    out = np.empty((rows, cols))
    high = 128 if tiles else 1
    for r in range(0, rows, high):
        for c in range(0, cols, 128):
            b = np.asarray(x[r:r + high, c:c + 128], np.float64)
            a = np.abs(b).max()
            if not np.isfinite(a):
                out[r:r + high, c:c + 128] = np.nan
                continue
            e = -110
            if a > 0:
                f, k = np.frexp(a)                              # a = f 2^k, 1/2 <= f < 1; the largest code is 0.875 2^(TOP + 1)
                e = max(e, int(k) - 1 - TOP[form] + (1 if f > 0.875 else 0))
            v = np.ldexp(b, -e)
            k = np.maximum(np.frexp(v)[1] - 1, LOWEST[form])
            k = np.where(v == 0, LOWEST[form], k) - MANTISSA[form]
            with np.errstate(over="ignore"):
                out[r:r + high, c:c + 128] = np.ldexp(np.ldexp(np.rint(np.ldexp(v, -k)), k), e).astype(np.float32)      # 2^128: infinite
    return out


def philox(counters, key):
    """Philox-4x32-10: counters [n, 4] and a key of two, all below 2^32, as Python's whole numbers."""
    out = []
    for c in counters:
        c, k = [int(v) for v in c], list(key)
        for _ in range(10):
            a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
            c = [(b >> 32) ^ c[1] ^ k[0], b & 0xffffffff, (a >> 32) ^ c[3] ^ k[1], a & 0xffffffff]
            k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
        out.append(c)
    return out


def mask(rows, cols, p, seed, offset):
    """0 for a dropped element, the factor elsewhere"""
    groups, limit = (cols + 7) // 8, round(p * 65536)
    if not limit:
        return np.ones((rows, cols))
    low = 0xffffffff
    words = philox([(i & low, i >> 32, offset & low, offset >> 32) for i in range(rows * groups)], (seed & low, seed >> 32))
    halves = np.array([[h for w in c for h in (w & 0xffff, w >> 16)] for c in words]).reshape(rows, groups * 8)[:, :cols]
    return (halves >= limit) * (65536 / (65536 - limit))


def norm(v, rms, gain, bias, eps, exact=True):
    mean = 0.0 if rms else v.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((v - mean) ** 2).mean(1, keepdims=True) + eps)
    return (v - mean) * rstd * gain + bias, mean, rstd
