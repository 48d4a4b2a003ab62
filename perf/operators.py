"""Measured cases of the operators around the attention of a diffusion-transformer block.

  block_norm  x' = a x + gate N2(y),  h = N1(x') (1 + scale) + shift, and its gradients
  rope        rotary positions with several axes on q and k, and the inverse rotation (its gradient)
  mx_round    microscaled 4-bit floating point: quantise and read back
  mx_linear   activations quantised in the call, product with 4-bit weights, bias

``own`` False: plain forms in elementary torch operations; True: the library's entry points.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
NORMS = {"none": 0, "layer": 1, "rms": 2}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------------- the cases
def _norm(op, n, c, per_mod, x="bf16", io="bf16", residual=True, gate=True, post="none", norm="layer", affine=False,
          mod=True, alpha=1.0):
    return {"op": op, "n": n, "c": c, "per_mod": per_mod, "x": x, "io": io, "residual": residual, "gate": gate,
            "post": post, "norm": norm, "affine": affine, "mod": mod, "alpha": alpha}


def _rope(n, hq, hk, d, widths, layout="adjacent", ladder="axis", dtype="bf16", pos="int", offset=0, inverse=False):
    return {"op": "rope", "n": n, "hq": hq, "hk": hk, "d": d, "w0": widths[0], "w1": widths[1], "w2": widths[2],
            "layout": layout, "ladder": ladder, "type": dtype, "pos": pos, "offset": offset, "inverse": inverse}


def _round(rows, cols, dtype="bf16"):
    return {"op": "mx_round", "rows": rows, "cols": cols, "type": dtype}


def _linear(n, k, f, dtype="bf16", bias=True):
    return {"op": "mx_linear", "n": n, "k": k, "f": f, "type": dtype, "bias": bias}


def listed():
    named = {
        # the norm in front of the modulation of a single embedding row: pure latency
        "norm_one_row": _norm("norm", 1, 1536, 1, residual=False, gate=False),
        # behind the self-attention of a 480x832 window: gated residual, then the modulated norm
        "norm_window": _norm("norm", 10920, 1536, 10920),
        # 77-frame clip, fp32 residual stream, one modulation row per latent frame, norms on both sides of the block
        "norm_clip_fp32_sandwich": _norm("norm", 31200, 5120, 1560, x="fp32", post="rms", norm="rms", affine=True),
        # gradients of the same step at the window, one modulation row per latent frame
        "norm_back_window": _norm("norm_back", 10920, 1536, 1560),
        # gradients at the 40-head window with norms on both sides and the affine norm in front of cross-attention
        "norm_back_large_sandwich": _norm("norm_back", 12480, 5120, 12480, x="fp32", post="rms", affine=True),
        # rotation of q and k of the 77-frame clip by explicit (t, y, x) positions
        "rope_clip": _rope(31200, 40, 40, 128, (44, 42, 42)),
        # gradient of the rotation with shared key heads, half pairs and frame times in seconds; odd token count
        "rope_back_shared_heads": _rope(4097, 40, 8, 128, (32, 48, 48), "halves", "whole", "fp16", "float", 0, True),
        # a projection's weights taken to 4 bits and read back
        "mx_round_weights": _round(4608, 1536),
        # fp32 weights with a ragged inner extent
        "mx_round_ragged": _round(5120, 13825, "fp32"),
        # the modulation row of a denoising step: one row against 4-bit weights, six vectors of 1536 features
        "mx_linear_one_row": _linear(1, 1536, 9216),
        # QKV projection of a 480x832 window
        "mx_linear_window": _linear(10920, 1536, 4608),
        # QKV projection of the 77-frame clip
        "mx_linear_clip": _linear(31200, 5120, 15360),
    }
    return [dict(c, name=name) for name, c in named.items()]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_back", "rope", "mx_round", "mx_linear", "mx_linear"])
    if op in ("norm", "norm_back"):
        n = _log(rng, 1, 31200)
        c = 128 * rng.randint(1, 40) if rng.random() < 0.7 else rng.randint(8, 5120)
        io = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        x = "fp32" if rng.random() < 0.4 else io
        residual = rng.random() < 0.8
        return _norm(op, n, c, rng.choice([n, n, max(1, n // rng.randint(2, 20)), 1 if n <= 4096 else n]), x, io,
                     residual, residual and rng.random() < 0.7, rng.choice(["none", "rms", "layer"]) if residual else "none",
                     rng.choice(["layer", "rms"]), rng.random() < 0.5, rng.random() < 0.7,
                     rng.choice([1.0, 0.5]) if residual else 1.0)
    if op == "rope":
        d = rng.choice([64, 80, 96, 128, 128, 128, 256])
        hk = rng.randint(1, 16)
        hq = hk * rng.randint(1, max(1, 40 // hk))
        w0 = 2 * rng.randint(1, d // 4)
        w1 = 2 * rng.randint(0, (d - w0) // 2)
        w2 = 2 * rng.randint(0, (d - w0 - w1) // 2) if w1 else 0
        if rng.random() < 0.5:
            w2 = d - w0 - w1 if w1 else 0
        n = min(_log(rng, 1, 31200), 31200 * 40 * 128 // (hq * d))
        return _rope(n, hq, hk, d, (w0, w1, w2), rng.choice(["adjacent", "halves"]), rng.choice(["axis", "whole"]),
                     rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.choice(["int", "float"]),
                     rng.choice([0, 0, 1000003]), rng.random() < 0.4)
    if op == "mx_round":
        cols = _log(rng, 1, 16384)
        return _round(min(_log(rng, 1, 16384), (1 << 26) // cols + 1), cols, rng.choice(["bf16", "bf16", "fp16", "fp32"]))
    k = 128 * rng.randint(1, 80) if rng.random() < 0.6 else rng.randint(8, 10240)
    f = 8 * rng.randint(1, 1920)
    n = min(_log(rng, 1, 31200), int(31200 * 5120 * 15360 // (k * f)))
    return _linear(n, k, f, rng.choice(["bf16", "bf16", "fp16", "fp32"]), rng.random() < 0.7)


# --------------------------------------------------------------------------------------------------------- the inputs
def _mods(c):
    return -(-c["n"] // c["per_mod"])


def _rng(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) + 1)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32)


def _prepare_norm(c, seed):
    g, n, ch = _rng(seed), c["n"], c["c"]
    tx, tio = TYPES[c["x"]], TYPES[c["io"]]
    # a residual stream: some channels much larger than the others, and a mean that is not zero
    wide = 1.0 + 4.0 * torch.rand(ch, generator=g, device=DEV) ** 4
    s = {"x": (_randn(g, n, ch) * wide + 0.5).to(tx)}
    s["y"] = _randn(g, n, ch).to(tio) if c["residual"] else None
    # modulation rows as a block holds them: six vectors of c features side by side
    six = _randn(g, _mods(c), 6, ch) * 0.3
    s["shift"], s["scale"] = (six[:, 0], six[:, 1]) if c["mod"] else (None, None)
    s["gate"] = six[:, 2] if c["gate"] else None
    s["weight"] = 1.0 + 0.2 * _randn(g, ch) if c["affine"] else None
    s["bias"] = 0.2 * _randn(g, ch) if c["affine"] else None
    s["post_weight"] = 1.0 + 0.2 * _randn(g, ch) if c["post"] != "none" else None
    if c["op"] == "norm_back":   # `x` stands for the saved x'; gradients of h and of x'
        s["dh"] = _randn(g, n, ch).to(tio)
        s["dx_out"] = _randn(g, n, ch).to(tx) if c["residual"] else None
    return s


def _prepare_rope(c, seed):
    g, n = _rng(seed), c["n"]
    t = TYPES[c["type"]]
    s = {"q": _randn(g, n, c["hq"], c["d"]).to(t), "k": _randn(g, n, c["hk"], c["d"]).to(t)}
    side = max(1, int(math.sqrt(n / 8.0)))        # a grid of frames, rows and columns that holds n tokens
    i = torch.arange(n, device=DEV)
    axes = torch.stack([i // (side * side), i // side % side, i % side])[:_axes(c)] + c["offset"]
    axes = axes + torch.randint(0, 7, (_axes(c), 1), generator=g, device=DEV)
    s["positions"] = (axes.to(torch.float32) * 0.25 if c["pos"] == "float" else axes.to(torch.int32)).contiguous()
    return s


def _axes(c):
    return 1 + (c["w1"] > 0) + (c["w2"] > 0)


def _widths(c):
    return [c["w0"], c["w1"], c["w2"]][:_axes(c)]


def _heavy(g, rows, cols):
    """Activations and weights: normal, with columns of larger values as transformer layers have them."""
    return _randn(g, rows, cols) * (1.0 + 7.0 * torch.rand(cols, generator=g, device=DEV) ** 6)


def _packed(values):
    """The documented packed form of a 4-bit matrix (codes, then scales in tiles of 128 rows x 4 blocks), built with
    torch as a program would from its checkpoint."""
    rows, cols = values.shape
    kp = -(-cols // 128) * 128
    v = torch.nn.functional.pad(values, (0, kp - cols)).view(rows, kp // 32, 32)
    amax = v.abs().amax(dim=2)
    e = (torch.frexp(amax)[1] - 3).clamp(-127, 127)
    e = torch.where(amax > 0, e, torch.full_like(e, -127))
    m = torch.ldexp(v.abs(), -e.unsqueeze(2))
    code = torch.zeros_like(m, dtype=torch.uint8)
    for i, edge in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):   # halfway points; ties to the even code
        code += (m > edge) if i % 2 == 0 else (m >= edge)
    code |= torch.signbit(v).to(torch.uint8) << 3
    code = code.view(rows, kp // 2, 2)
    codes = (code[..., 0] | code[..., 1] << 4).reshape(-1)
    sc = torch.zeros((-(-rows // 128) * 128, kp // 32), dtype=torch.uint8, device=values.device)
    sc[:rows] = (e + 127).to(torch.uint8)
    sc = sc.view(-1, 4, 32, kp // 128, 4).permute(0, 3, 2, 1, 4).reshape(-1)
    at = -(-codes.numel() // 512) * 512
    out = torch.zeros(at + sc.numel(), dtype=torch.uint8, device=values.device)
    out[:codes.numel()] = codes
    out[at:] = sc
    return out


def prepare(case, seed):
    c = case
    if c["op"] in ("norm", "norm_back"):
        s = _prepare_norm(c, seed)
    elif c["op"] == "rope":
        s = _prepare_rope(c, seed)
    elif c["op"] == "mx_round":
        s = {"x": (_heavy(_rng(seed), c["rows"], c["cols"]) / math.sqrt(c["cols"])).to(TYPES[c["type"]])}
    else:
        g = _rng(seed)
        s = {"x": _heavy(g, c["n"], c["k"]).to(TYPES[c["type"]]),
             "w": _packed(_heavy(g, c["f"], c["k"]) / math.sqrt(c["k"])),
             "bias": 0.1 * _randn(g, c["f"]) if c["bias"] else None}
    s["case"] = c
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms
def _rows(m, c):
    """A modulation vector per token (broadcast where all tokens share one)."""
    if m is None:
        return None
    return m if m.shape[0] == 1 else m.repeat_interleave(c["per_mod"], dim=0)[: c["n"]]


def _stat(x, kind):
    """xhat and 1 / its deviation."""
    d = x - x.mean(dim=1, keepdim=True) if kind == "layer" else x
    r = torch.rsqrt((d * d).mean(dim=1, keepdim=True) + EPS)
    return d * r, r


def _plain_norm(s, c):
    x = s["x"].float()
    if c["residual"]:
        z = s["y"].float()
        if c["post"] != "none":
            z = _stat(z, c["post"])[0] * s["post_weight"]
        if c["gate"]:
            z = z * _rows(s["gate"], c)
        x = c["alpha"] * x + z
    h = _stat(x, c["norm"])[0]
    if c["affine"]:
        h = h * s["weight"] + s["bias"]
    if c["mod"]:
        h = h * (1.0 + _rows(s["scale"], c)) + _rows(s["shift"], c)
    return {"x_out": x.to(s["x"].dtype) if c["residual"] else None, "h": h.to(TYPES[c["io"]])}


def _per_mod(v, c):
    """Sums of the rows of every modulation row's tokens (in 64 bits: up to 31200 terms)."""
    v = v.double()
    if _mods(c) == 1:
        return v.sum(dim=0, keepdim=True)
    whole = c["n"] // c["per_mod"]
    parts = [v[: whole * c["per_mod"]].view(whole, c["per_mod"], -1).sum(dim=1)]
    if c["n"] % c["per_mod"]:
        parts.append(v[whole * c["per_mod"]:].sum(dim=0, keepdim=True))
    return torch.cat(parts)


def _norm_grad(g, xhat, r, kind):
    g = g - xhat * (g * xhat).mean(dim=1, keepdim=True) - (g.mean(dim=1, keepdim=True) if kind == "layer" else 0.0)
    return g * r


def _plain_norm_back(s, c):
    xhat, r = _stat(s["x"].float(), c["norm"])
    dn, out = s["dh"].float(), {}
    n = xhat * s["weight"] + s["bias"] if c["affine"] else xhat
    if c["mod"]:
        out["dscale"], out["dshift"] = _per_mod(dn * n, c).float(), _per_mod(dn, c).float()
        dn = dn * (1.0 + _rows(s["scale"], c))
    if c["affine"]:
        out["dweight"], out["dbias"] = (dn * xhat).double().sum(dim=0).float(), dn.double().sum(dim=0).float()
        dn = dn * s["weight"]
    dx = _norm_grad(dn, xhat, r, c["norm"])
    if c["residual"]:
        dx = dx + s["dx_out"].float()
        y = s["y"].float()
        if c["post"] != "none":
            yhat, ry = _stat(y, c["post"])
            y = yhat * s["post_weight"]
        if c["gate"]:
            out["dgate"] = _per_mod(dx * y, c).float()
        dz = dx * _rows(s["gate"], c) if c["gate"] else dx
        if c["post"] != "none":
            out["dpost_weight"] = (dz * yhat).double().sum(dim=0).float()
            dz = _norm_grad(dz * s["post_weight"], yhat, ry, c["post"])
        out["dy"] = dz.to(s["y"].dtype)
        dx = c["alpha"] * dx
    out["dx"] = dx.to(s["x"].dtype)
    return out


def _plain_rope(s, c):
    widths, total = _widths(c), sum(_widths(c))
    ang = []
    done = 0
    for a, w in enumerate(widths):
        i = torch.arange(w // 2, device=DEV, dtype=torch.float64)
        power = i / (w // 2) if c["ladder"] == "axis" else (i + done) / (total // 2)
        done += w // 2
        ang.append(s["positions"][a].double()[:, None] * torch.pow(10000.0, -power)[None, :])
    ang = torch.cat(ang, dim=1)[:, None, :]
    cos, sin = ang.cos().float(), ang.sin().float()
    if c["inverse"]:
        sin = -sin
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        y = x.clone()
        lo, hi = ((slice(0, total, 2), slice(1, total, 2)) if c["layout"] == "adjacent"
                  else (slice(0, total // 2), slice(total // 2, total)))
        y[..., lo] = x[..., lo] * cos - x[..., hi] * sin
        y[..., hi] = x[..., hi] * cos + x[..., lo] * sin
        out[name] = y.to(s[name].dtype)
    return out


def _to_mx(x):
    """Values that the 4-bit form of fp32 rows stands for, in fp32."""
    rows, cols = x.shape
    v = torch.nn.functional.pad(x, (0, -cols % 32)).view(rows, -1, 32)
    e = (torch.frexp(v.abs().amax(dim=2, keepdim=True))[1] - 3).clamp(-127, 127)
    m = torch.ldexp(v, -e)
    step = torch.where(m.abs() < 2, 0.5, torch.where(m.abs() < 4, 1.0, 2.0))
    m = (torch.round(m / step) * step).clamp(-6, 6)
    return torch.ldexp(m, e).view(rows, -1)[:, :cols]


def _from_packed(p, rows, cols):
    """fp32 values of a packed 4-bit matrix."""
    kp = -(-cols // 128) * 128
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=p.device)
    grid = torch.cat([grid, -grid])
    codes = p[: rows * kp // 2].view(rows, kp // 2).int()
    v = torch.stack([grid[codes & 15], grid[codes >> 4]], dim=2).view(rows, kp // 32, 32)
    at = -(-(rows * kp // 2) // 512) * 512
    sc = p[at:].view(-1, kp // 128, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, kp // 32)[:rows]
    return torch.ldexp(v, (sc.int() - 127).unsqueeze(2)).view(rows, kp)[:, :cols]


def _plain_mx_linear(s, c):
    y = _to_mx(s["x"].float()) @ _from_packed(s["w"], c["f"], c["k"]).t()
    if c["bias"]:
        y = y + s["bias"]
    return {"y": y.to(torch.bfloat16)}


# ------------------------------------------------------------------------------------------------------- the operators
def _own(s, c):
    from paper_2607_28144_b200 import binding

    if c["op"] == "norm":
        x_out, h = binding.regenvc_block_norm_forward(
            s["x"], s["y"], gate=s["gate"], post_norm=NORMS[c["post"]], post_weight=s["post_weight"], post_eps=EPS,
            residual_scale=c["alpha"], norm=NORMS[c["norm"]], weight=s["weight"], bias=s["bias"], eps=EPS,
            scale=s["scale"], shift=s["shift"], tokens_per_mod=c["per_mod"], h_dtype=TYPES[c["io"]])
        return {"x_out": x_out, "h": h}
    if c["op"] == "norm_back":
        g = binding.regenvc_block_norm_backward(
            s["dh"], s["x"], dx_out=s["dx_out"], y=s["y"], gate=s["gate"], post_norm=NORMS[c["post"]],
            post_weight=s["post_weight"], post_eps=EPS, residual_scale=c["alpha"], norm=NORMS[c["norm"]],
            weight=s["weight"], bias=s["bias"], eps=EPS, scale=s["scale"], shift=s["shift"],
            tokens_per_mod=c["per_mod"])
        return {k: v for k, v in g.items() if v is not None}
    if c["op"] == "rope":
        q, k = binding.regenvc_rope_axes(s["q"], s["k"], s["positions"], _widths(c), rope_theta=10000.0,
                                         halves=c["layout"] == "halves", whole_ladder=c["ladder"] == "whole",
                                         inverse=c["inverse"])
        return {"q": q, "k": k}
    if c["op"] == "mx_round":
        packed = binding.regenvc_mxfp4_quantize(s["x"])
        return {"x": binding.regenvc_mxfp4_dequantize(packed, c["rows"], c["cols"], s["x"].dtype)}
    return {"y": binding.regenvc_mxfp4_linear(s["x"], s["w"], c["f"], s["bias"])}


def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c)
    if c["op"] == "norm":
        return _plain_norm(s, c)
    if c["op"] == "norm_back":
        return _plain_norm_back(s, c)
    if c["op"] == "rope":
        return _plain_rope(s, c)
    if c["op"] == "mx_round":
        return {"x": _to_mx(s["x"].float()).to(s["x"].dtype)}
    return _plain_mx_linear(s, c)


# ------------------------------------------------------------------------------------------------------------ the work
def work(case):
    c = case
    if c["op"] in ("norm", "norm_back"):
        e, sx, si, m = c["n"] * c["c"], SIZE[c["x"]], SIZE[c["io"]], _mods(c) * c["c"] * 4
        res, vec = c["residual"], 2 * c["affine"] + (c["post"] != "none")
        if c["op"] == "norm":     # x, y in; x', h out
            return {"bytes": e * (sx + si + res * (si + sx)) + m * (2 * c["mod"] + c["gate"]) + vec * c["c"] * 4,
                    "flops": e * (8 + 4 * res)}
        # x', dh in, dx out; dx', y in, dy out; parameters and modulation rows in, their gradients out
        return {"bytes": e * (2 * sx + si + res * (sx + 2 * si)) + m * (3 * c["mod"] + 2 * c["gate"]) + 2 * vec * c["c"] * 4,
                "flops": e * (16 + 12 * res)}
    if c["op"] == "rope":
        e = c["n"] * (c["hq"] + c["hk"]) * c["d"]
        return {"bytes": 2 * e * SIZE[c["type"]] + 4 * _axes(c) * c["n"], "flops": 3 * e}
    if c["op"] == "mx_round":     # values in, 4-bit form out and in again, values out
        e = c["rows"] * c["cols"]
        return {"bytes": e * 2 * SIZE[c["type"]] + 2 * (e // 2 + e // 32), "flops": 4 * e}
    n, k, f = c["n"], c["k"], c["f"]
    return {"bytes": n * k * SIZE[c["type"]] + f * k * 17 / 32 + 2 * n * f + 4 * f * c["bias"], "flops": 2.0 * n * k * f}


# ------------------------------------------------------------------------------------------- the definitions, in 64 bits
def _exact_norm(s, c):
    """Token by token from the definitions: the gradients are those that automatic differentiation gives in 64 bits."""
    wants = c["op"] == "norm_back"
    p = {k: s[k].double() for k in ("weight", "bias", "post_weight", "scale", "shift", "gate") if s[k] is not None}
    for v in p.values():
        v.requires_grad_(wants)
    row = torch.arange(c["n"], device=DEV) // c["per_mod"]
    out_x, out_h, dx, dy = [], [], [], []
    step = max(1, (1 << 25) // c["c"])
    for a in range(0, c["n"], step):
        at = slice(a, min(c["n"], a + step))
        x = s["x"][at].double().requires_grad_(wants)

        def norm(t, kind):
            if kind == "layer":
                t = t - t.sum(1, keepdim=True) / c["c"]
            return t / ((t ** 2).sum(1, keepdim=True) / c["c"] + EPS).sqrt()

        if c["residual"]:
            y = s["y"][at].double().requires_grad_(wants)
            z = norm(y, c["post"]) * p["post_weight"] if c["post"] != "none" else y
            z = z * p["gate"][row[at]] if c["gate"] else z
        if not wants:
            t = c["alpha"] * x + z if c["residual"] else x
        else:
            t = x
        h = norm(t, c["norm"])
        if c["affine"]:
            h = h * p["weight"] + p["bias"]
        if c["mod"]:
            h = h * (1 + p["scale"][row[at]]) + p["shift"][row[at]]
        if not wants:
            out_x.append(t)
            out_h.append(h)
            continue
        # the saved x' is where the norm in front is differentiated; its gradient then goes on to x and y
        (h * s["dh"][at].double()).sum().backward()
        d = x.grad
        if c["residual"]:
            d = d + s["dx_out"][at].double()
            (z * d).sum().backward()
            dy.append(y.grad)
            d = c["alpha"] * d
        dx.append(d)
    if not wants:
        return {"x_out": torch.cat(out_x) if c["residual"] else None, "h": torch.cat(out_h)}
    g = {"dx": torch.cat(dx)}
    if c["residual"]:
        g["dy"] = torch.cat(dy)
    g.update({"d" + k: v.grad for k, v in p.items()})
    return g


def _exact_rope(s, c):
    widths, total = _widths(c), sum(_widths(c))
    turn, j = [], 0
    for a, w in enumerate(widths):
        for i in range(w // 2):
            f = 10000.0 ** (-2.0 * i / w) if c["ladder"] == "axis" else 10000.0 ** (-2.0 * j / total)
            turn.append(s["positions"][a].double() * f)
            j += 1
    z = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), torch.stack(turn, dim=1))[:, None, :]
    z = z.conj() if c["inverse"] else z
    out = {}
    for name in ("q", "k"):
        x = s[name].double()
        r, rest = x[..., :total], x[..., total:]
        if c["layout"] == "adjacent":
            r = torch.view_as_real(torch.view_as_complex(r.unflatten(-1, (-1, 2)).contiguous()) * z).flatten(-2)
        else:
            r = torch.complex(r[..., : total // 2], r[..., total // 2:]) * z
            r = torch.cat([r.real, r.imag], dim=-1)
        out[name] = torch.cat([r, rest], dim=-1)
    return out


def _exact_mx(x):
    rows, cols = x.shape
    v = torch.zeros((rows, -(-cols // 32) * 32), dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, -1, 32)
    top = v.abs().max(dim=2, keepdim=True)[0]
    # powers of two by the exponent fields of 64-bit floats (a logarithm may land just below a whole number)
    e = ((top.view(torch.int64) >> 52) - 1023 - 2).clamp_min(-127)
    scale = torch.where(top > 0, ((e + 1023) << 52).view(torch.float64), torch.ones_like(top))
    m = v.abs() / scale
    # distance to each of the eight magnitudes; of two equally near ones the one with the even code
    best, at = torch.full_like(m, math.inf), torch.zeros_like(m)
    for code in (0, 2, 4, 6, 1, 3, 5, 7):
        value = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)[code]
        near = (m - value).abs() < best
        best, at = torch.where(near, (m - value).abs(), best), torch.where(near, torch.full_like(m, value), at)
    return (torch.sign(v) * at * scale).view(rows, -1)[:, :cols]


def _exact_unpack(p, rows, cols):
    """Byte by byte as the layout is documented, on the host."""
    kp = -(-cols // 128) * 128
    raw = p.cpu().numpy()
    r, b = np.arange(rows)[:, None], np.arange(kp // 32)[None, :]
    at = -(-(rows * (kp // 2)) // 512) * 512
    sc = raw[at + (r // 128 * (kp // 128) + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4]
    codes = raw[: rows * (kp // 2)].reshape(rows, kp // 2)
    nib = np.empty((rows, kp), dtype=np.uint8)
    nib[:, 0::2], nib[:, 1::2] = codes & 15, codes >> 4
    mag = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    return torch.from_numpy(mag[:, :cols] * np.repeat(np.exp2(sc.astype(np.float64) - 127), 32, axis=1)[:, :cols]).to(p.device)


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] in ("norm", "norm_back"):
        return _exact_norm(s, c)
    if c["op"] == "rope":
        return _exact_rope(s, c)
    if c["op"] == "mx_round":
        return {"x": _exact_mx(s["x"].double())}
    x, w = _exact_mx(s["x"].double()), _exact_unpack(s["w"], c["f"], c["k"])
    y = x @ w.t()
    return {"y": y + s["bias"].double() if c["bias"] else y}
