"""Plain 64-bit implementations of the norm, the paged cache and attention over it, for the tests (CPU, float64 throughout)."""
import math

import torch

HALF_BF16 = 2.0 ** -8         # the most a rounding to bf16 changes a value, relative (half a step)
HALF_E4M3 = 2.0 ** -4
SUB_E4M3 = 2.0 ** -10         # half the step of e4m3 subnormals
F32 = 2.0 ** -24


def rmsnorm(x, residual, weight, eps):
    """(y, h) in float64."""
    h = x.double() if residual is None else x.double() + residual.double()
    return h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * weight.double(), h


def rmsnorm_backward(dy, h, weight, eps, dh):
    """(dx, dw, bound of dx's terms, bound of dw's terms): the bounds are the sums of absolute values that fp32 errors scale with."""
    dy, h, w = dy.double(), h.double(), weight.double()
    r = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    g = dy * w
    k = r * r * (g * h).mean(1, keepdim=True)
    dx = r * (g - h * k)
    size = r * (g.abs() + h.abs() * r * r * (g * h).abs().mean(1, keepdim=True))
    if dh is not None:
        dx = dx + dh.double()
        size = size + dh.double().abs()
    return dx, (dy * h * r).sum(0), size, (dy * h * r).abs().sum(0)


def e4m3_values(codes):
    """uint8 e4m3 bit patterns -> float64 (NaN for the NaN codes)."""
    c = codes.to(torch.int64) & 127
    e, f = c >> 3, (c & 7).double()
    v = torch.where(e == 0, f * 2.0 ** -9, (8 + f) * torch.exp2(e.double() - 10))
    v = torch.where(c == 127, torch.full_like(v, math.nan), v)
    return torch.where(codes.to(torch.int64) >= 128, -v, v)


def cached(cache_k, scales, table, n, page_size):
    """float64 [n, heads, dim]: positions 0 .. n - 1 of the sequence whose pages are `table`; rows of bad pages are None in `ok`."""
    pages, heads, _, dim = cache_k.shape
    out = torch.zeros((n, heads, dim), dtype=torch.float64)
    ok = torch.zeros((n,), dtype=torch.bool)
    for p in range(n):
        if p // page_size >= len(table):
            continue
        page = int(table[p // page_size])
        if not 0 <= page < pages:
            continue
        ok[p] = True
        row = cache_k[page, :, p % page_size]
        out[p] = row.double() if scales is None else e4m3_values(row) * scales[page, :, p % page_size].double()[:, None]
    return out, ok


def attention(q, k, v, ok, kv_len, scale, window):
    """q [n, Hq, D], k, v [kv_len, Hkv, D] -> (out, lse, sum of p |v|, bound of the scores' fp32 error), float64; only visible rows are touched."""
    n, Hq, D = q.shape
    Hkv = k.shape[1]
    out = torch.zeros((n, Hq, D), dtype=torch.float64)
    mag = torch.zeros((n, Hq, D), dtype=torch.float64)
    lse = torch.full((n, Hq), -math.inf, dtype=torch.float64)
    zerr = torch.zeros((n, Hq), dtype=torch.float64)
    for i in range(n):
        p = kv_len - n + i
        lo = max(0, p - window + 1) if window else 0
        see = [j for j in range(lo, min(p + 1, k.shape[0])) if ok[j]]
        if not see:
            continue
        kk, vv, qq = k[see].permute(1, 0, 2), v[see].permute(1, 0, 2), q[i].double().view(Hkv, Hq // Hkv, D)
        z = scale * (qq @ kk.transpose(1, 2))                                   # [Hkv, group, visible]
        e = torch.logsumexp(z, 2, keepdim=True)
        w = torch.exp(z - e)
        lse[i] = e.view(Hq)
        out[i], mag[i] = (w @ vv).view(Hq, D), (w @ vv.abs()).view(Hq, D)
        zerr[i] = (abs(scale) * (qq.abs() @ kk.abs().transpose(1, 2))).amax(2).view(Hq) * (D + 8) * F32
    return out, lse, mag, zerr
