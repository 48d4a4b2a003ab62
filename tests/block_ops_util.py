"""Plain 64-bit forms of the operators around a block's attention, for their tests.  Every function also returns (or
takes) magnitudes -- the same formula on absolute values -- from which the tests derive their bounds."""
import math

import torch

U = 2.0 ** -24                       # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def floor_step(dtype):
    """Half the distance of neighbouring values next to zero, where a rounding is no longer relative: fp16's subnormal
    values are 2^-24 apart, so a rounding there is off by up to 2^-25; bf16 and fp32 reach below 2^-126."""
    return 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126


def norm64(t, kind, eps):
    if kind == 1:
        t = t - t.mean(dim=1, keepdim=True)
    return t / torch.sqrt((t * t).mean(dim=1, keepdim=True) + eps)


def rows_of(table, per, n):
    return table[torch.arange(n, device=table.device) // per]


def block_norm64(x, y, p, norm, post, alpha, per, eps):
    """(x', h) in 64 bits; p: dict of gate, post_weight, weight, bias, scale, shift (or absent)."""
    n = x.shape[0]
    t = x
    if y is not None:
        z = norm64(y, post, eps) if post else y
        if p.get("post_weight") is not None:
            z = z * p["post_weight"]
        if p.get("gate") is not None:
            z = z * rows_of(p["gate"], per, n)
        t = alpha * x + z
    if not norm:
        return t, None
    h = norm64(t, norm, eps)
    if p.get("weight") is not None:
        h = h * p["weight"]
    if p.get("bias") is not None:
        h = h + p["bias"]
    if p.get("scale") is not None:
        h = h * (1 + rows_of(p["scale"], per, n))
    if p.get("shift") is not None:
        h = h + rows_of(p["shift"], per, n)
    return t, h


def rope64(x, positions, widths, theta, halves, whole, inverse):
    """Rotation by complex multiplication; x [n, heads, d] in 64 bits."""
    total, turn, j = sum(widths), [], 0
    for a, w in enumerate(widths):
        for i in range(w // 2):
            f = theta ** (-2.0 * j / total) if whole else theta ** (-2.0 * i / w)
            turn.append(positions[a].double() * f)
            j += 1
    ang = torch.stack(turn, dim=1)[:, None, :]
    if inverse:
        ang = -ang
    lo, hi = (slice(0, total, 2), slice(1, total, 2)) if not halves else (slice(0, total // 2), slice(total // 2, total))
    out = x.clone()
    a, b = x[..., lo], x[..., hi]
    out[..., lo] = a * ang.cos() - b * ang.sin()
    out[..., hi] = a * ang.sin() + b * ang.cos()
    size = x.abs()
    mag = size.clone()
    mag[..., lo] = size[..., lo] + size[..., hi]
    mag[..., hi] = mag[..., lo]
    return out, mag


GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def pow2(k):
    """2^k for whole k in [-1022, 1023], exactly (a library pow on the GPU may be an ulp off, which undoes a tie)."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def mx_codes64(x):
    """(codes [rows, blocks, 32], scale bytes [rows, blocks]) of 64-bit values by search for the nearest code."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    v = torch.zeros((rows, nb * 32), dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, nb, 32)
    top = v.abs().amax(dim=2)
    bad = ~torch.isfinite(v).all(dim=2)
    top = torch.where(bad, torch.zeros_like(top), top)
    e = ((top.view(torch.int64) >> 52) - 1023 - 2).clamp_min(-127)        # top is 0 or a normal 64-bit value
    byte = torch.where(bad, torch.full_like(e, 255), torch.where(top > 0, e + 127, torch.zeros_like(e)))
    m = torch.where(bad.unsqueeze(2), torch.zeros_like(v), v * pow2(127 - byte).unsqueeze(2))
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    d = (m.abs().unsqueeze(3) - grid).abs()
    near = d.amin(dim=3, keepdim=True)
    code = torch.zeros(m.shape, dtype=torch.int64, device=x.device)
    for c in (1, 3, 5, 7, 0, 2, 4, 6):          # of two equally near codes the even one stays
        code = torch.where(d[..., c] == near[..., 0], torch.full_like(code, c), code)
    return code | (torch.signbit(m).long() << 3), byte


def mx_values64(codes, byte, cols):
    mag = torch.tensor(GRID, dtype=torch.float64, device=codes.device)[codes & 7]
    v = torch.where(codes >= 8, -mag, mag) * pow2(byte - 127).unsqueeze(2)
    v = torch.where((byte == 255).unsqueeze(2), torch.full_like(v, math.nan), v)
    return v.reshape(codes.shape[0], -1)[:, :cols]


def mx_unpack(packed, rows, cols):
    """(codes [rows, blocks of cols_pad, 32], scale bytes) out of the packed form as the header documents it."""
    kp = -(-cols // 128) * 128
    raw = packed.long()
    b = raw[: rows * kp // 2].view(rows, kp // 2)
    codes = torch.stack([b & 15, b >> 4], dim=2).view(rows, kp // 32, 32)
    at = -(-(rows * kp // 2) // 512) * 512
    r = torch.arange(rows, device=raw.device)[:, None]
    k = torch.arange(kp // 32, device=raw.device)[None, :]
    return codes, raw[at + (r // 128 * (kp // 128) + k // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + k % 4]
