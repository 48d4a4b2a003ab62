"""Plain 64-bit forms of attention over cached windows, for its tests, with the magnitudes that the tests' bounds count."""
import math

import torch

from block_ops_util import U, floor_step, half_step, rope64

EXP = 1e-4      # relative error of a probability: 2^x by a polynomial (7.5e-5) or the special-function unit (2^-22)


def head64(x, w, positions, widths, theta, halves, whole, eps, norm=True, inverse=False):
    """(y, magnitude): x [tokens, heads, d] in 64 bits normalised per head, times w, rotated."""
    if norm:
        x = x / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + eps)
        if w is not None:
            x = x * w
    if not widths:
        return x, x.abs()
    return rope64(x, positions, widths, theta, halves, whole, inverse)


def head_grads64(x, w, dy, positions, widths, theta, halves, whole, eps):
    """dx, dw and magnitudes, from the formula: g = R^T dy, n = x r, dw = sum g n, dx = r (g w - n mean(g w n))."""
    g, gm = rope64(dy, positions, widths, theta, halves, whole, True) if widths else (dy, dy.abs())
    r = 1 / torch.sqrt((x * x).mean(dim=-1, keepdim=True) + eps)
    n = x * r
    h, hm = (g, gm) if w is None else (g * w, gm * w.abs())
    dx = r * (h - n * (h * n).mean(dim=-1, keepdim=True))
    mag = r * (hm + n.abs() * (hm * n.abs()).mean(dim=-1, keepdim=True))
    return dx, mag, (g * n).sum(dim=(0, 1)), (gm * n.abs()).sum(dim=(0, 1))


def sees(new, keys, group, window):
    """[new, keys] truth values: which cached tokens each of a sequence's last `new` tokens sees."""
    p = torch.arange(keys - new, keys)[:, None]
    t = torch.arange(keys)[None, :]
    if group == 0:
        return torch.ones((new, keys), dtype=torch.bool)
    see = (t // group <= torch.div(p, group, rounding_mode="floor")) & (p >= 0)
    if window:
        see &= t // group > torch.div(p, group, rounding_mode="floor") - window
    return see


def attend64(q, k, v, see, scale, dtype):
    """(out, lse, bound of |out - kernel|, bound of |lse - kernel|): q [new, hq, d], k and v [keys, hk, d] in 64 bits."""
    new, hq, d = q.shape
    share = hq // k.shape[1]
    out, lse = torch.zeros_like(q), torch.full((new, hq), -math.inf, dtype=torch.float64, device=q.device)
    bound, lse_bound = torch.zeros_like(q), torch.zeros_like(lse)
    see = see.to(q.device)
    some = see.any(dim=1)
    for a in range(hq if k.shape[0] else 0):
        kk, vv = k[:, a // share], v[:, a // share]
        vv = torch.where(see.any(dim=0)[:, None], vv, torch.zeros_like(vv))      # what nobody sees may be anything
        kk = torch.where(see.any(dim=0)[:, None], kk, torch.zeros_like(kk))
        x = torch.where(see, scale * (q[:, a] @ kk.t()), -math.inf)
        size = torch.where(see, scale * (q[:, a].abs() @ kk.abs().t()), 0.0).amax(dim=1, keepdim=True)
        top = torch.where(some[:, None], x.amax(dim=1, keepdim=True), 0.0)
        e = torch.exp(x - top)
        total = e.sum(dim=1, keepdim=True)
        w = torch.where(some[:, None], e / total, 0.0)
        out[:, a] = w @ vv
        lse[:, a] = torch.where(some, (top + torch.log(total))[:, 0], -math.inf)
        # errors of a score: d products and sums in fp32, its scale and the reference's subtraction
        score = (d + 8) * U * size + 4 * U * (top.abs() + 32)
        share_error = half_step(dtype) + 2 * (EXP + score) + (k.shape[0] + 16) * U
        bound[:, a] = share_error * (w @ vv.abs()) + half_step(dtype) * out[:, a].abs() + floor_step(dtype)
        if dtype == torch.float16:      # probabilities below 2^-14 of the reference are subnormal; the sum is at least 1
            bound[:, a] += 2.0 ** -25 * (see.double() @ vv.abs())
        lse_bound[:, a] = (EXP + score + (k.shape[0] + 16) * U)[:, 0] + 4 * U * (lse[:, a].abs().nan_to_num(posinf=0.0) + 32)
    return out, lse, bound, lse_bound


def scatter_pages(keys, page, order, gen, spare=2):
    """A table [sequences, pages] of distinct pages in random order (entries behind a sequence's last page: 10^6, which no
    call may read), and the number of pages."""
    need = [-(-m // page) for m in keys]
    n = sum(need) + spare
    perm = torch.randperm(n, generator=gen)
    table = torch.full((len(keys), max(max(need), 1)), 10 ** 6, dtype=torch.int32)
    at = 0
    for s, m in enumerate(need):
        table[s, :m] = perm[at:at + m].int()
        at += m
    return table, n


def slots_of(table, s, keys, page):
    t = torch.arange(keys)
    return table[s, t // page].long(), t % page
