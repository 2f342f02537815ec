"""Plain 64-bit implementations of the 4-bit cache's values and of sampling, for the tests (CPU)."""
import math

import numpy as np
import torch


def e2m1_values(codes, scales):
    """uint8 [..., dim / 2] of two e2m1 codes and uint8 [..., 4] of scale bytes -> (values, scales), float64 [..., dim]"""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)
    c = codes.to(torch.int64)
    v = torch.stack([table[c & 15], table[c >> 4]], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    s = torch.where(scales == 255, torch.tensor(math.nan, dtype=torch.float64), torch.exp2(scales.double() - 127)).repeat_interleave(v.shape[-1] // 4, -1)
    return v * s, s


def e2m1_quantized(x):
    """float64 [..., dim] -> (codes uint8 [..., dim / 2], scale bytes uint8 [..., 4]); -0 becomes +0"""
    part = x.double().view(*x.shape[:-1], 4, -1)
    top = part.abs().amax(-1)
    bad = ~part.isfinite().all(-1)
    e = torch.full(top.shape, -100, dtype=torch.int64)
    for k in range(-100, 125):
        e = torch.where(top > 6.0 * 2.0 ** k, k + 1, e)
    t = part.nan_to_num(0.0, 0.0, 0.0) / torch.exp2(e.double())[..., None]
    a = t.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)     # ties to the even code
    code = torch.where((t < 0) & (code > 0), code + 8, code)
    code = torch.where(bad[..., None], 0, code).reshape(x.shape).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.where(bad, 255, e + 127).to(torch.uint8)


def sample(row, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob, kept logprob, tokens kept) of one row: float64 sums over the sorted tokens"""
    z = np.asarray(row, dtype=np.float64)
    f = lambda v: float(np.float32(v))          # noqa: E731  (what the call is given)
    t, u, top_p, min_p = f(temperature), f(u), f(top_p), f(min_p)
    if np.isnan(z).any() or (z == np.inf).any() or not np.isfinite(z).any() or not 0 <= t < np.inf:
        return -1, math.nan, math.nan, 0
    order = np.lexsort((np.arange(len(z)), -z))
    order = order[z[order] > -np.inf]
    y = (z[order] - z[order[0]]) / (t or 1.0)
    w = np.exp(y)
    n = len(order)
    if t == 0:
        n = 1
    elif top_k > 0:
        n = min(n, top_k)
    cum = np.cumsum(w)
    if top_p < 1:
        mass = cum[n - 1]
        n = max(1, int(((cum[:n] - w[:n]) < top_p * mass).sum()))
    if min_p > 0:
        n = max(1, min(n, int((w >= min_p).sum())))
    goal = (u if u >= 0 else 0.0) * cum[n - 1]
    at = min(int((cum[:n] <= goal).sum()), n - 1)
    return int(order[at]), y[at] - math.log(math.fsum(w)), y[at] - math.log(math.fsum(w[:n])), n
