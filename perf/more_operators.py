"""Measured cases of the operators that attend over cached windows.

  norm_rope       q and k of every head normalised (RMS, with gains) and rotated by positions on several axes, one pass
  norm_rope_back  its gradients
  append          new tokens' keys (normalised, rotated) and values into a paged cache, their queries beside them
  attend          attention of chunks of new tokens over the paged cache, ragged, with masks by groups of tokens

``own`` False: plain forms in elementary torch operations; True: the library's entry points.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-6
THETA = 10000.0


# ---------------------------------------------------------------------------------------------------------- the cases
def _heads(op, n, hq, hk, d=128, dtype="bf16", layout="adjacent", ladder="axis", pos="int", gains=True):
    return {"op": op, "n": n, "hq": hq, "hk": hk, "d": d, "type": dtype, "layout": layout, "ladder": ladder, "pos": pos,
            "gains": gains}


def _append(seqs, new, cached, hq, hk, d=128, page=64, dtype="bf16", layout="adjacent", ladder="axis", pos="int",
            gains=True, ragged=True, order="tokens"):
    return {"op": "append", "seqs": seqs, "new": new, "cached": cached, "hq": hq, "hk": hk, "d": d, "page": page,
            "type": dtype, "layout": layout, "ladder": ladder, "pos": pos, "gains": gains, "ragged": ragged, "order": order}


def _attend(seqs, new, cached, hq, hk, d=128, page=64, dtype="bf16", group=0, window=0, ragged=True, order="tokens"):
    return {"op": "attend", "seqs": seqs, "new": new, "cached": cached, "hq": hq, "hk": hk, "d": d, "page": page,
            "type": dtype, "group": group, "window": window, "ragged": ragged, "order": order}


def listed():
    named = {
        # one token of one stream: pure latency
        "norm_rope_one_token": _heads("norm_rope", 1, 12, 12),
        # q and k of a 480x832 window
        "norm_rope_window": _heads("norm_rope", 10920, 12, 12),
        # gradients at the same window
        "norm_rope_back_window": _heads("norm_rope_back", 10920, 12, 12),
        # fp32 gradients with shared key heads, half pairs and frame times in seconds; odd token count
        "norm_rope_back_shared_fp32": _heads("norm_rope_back", 4097, 40, 8, 128, "fp32", "halves", "whole", "float"),
        # one new token for each of 64 streams
        "append_tokens": _append(64, 1, 4000, 40, 8, page=16, layout="halves", ladder="whole"),
        # a whole window of 7 latent frames, a page per latent frame
        "append_window": _append(1, 10920, 10920, 12, 12, page=1560, ragged=False),
        # one token of one stream over a short cache: pure latency
        "attend_one_token": _attend(1, 1, 300, 12, 12),
        # single tokens of 64 streams over ragged caches, shared key heads
        "attend_tokens": _attend(64, 1, 16384, 40, 8, page=16, group=1),
        # a new latent frame over the window before it and itself
        "attend_frame": _attend(1, 1560, 10920, 12, 12, page=1560, ragged=False),
        # a new window, causal by latent frames, over the last 14 frames of a 77-frame clip; 40 heads
        "attend_window": _attend(1, 10920, 20280, 40, 40, page=1560, group=1560, window=14, ragged=False),
        # chunks and single tokens of several streams in one call, causal, fp16, narrow heads, odd lengths
        "attend_mixed_fp16": _attend(9, 1500, 6000, 24, 8, 64, 48, "fp16", 1, order="heads"),
    }
    return [dict(c, name=name) for name, c in named.items()]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["norm_rope", "norm_rope_back", "append", "attend", "attend", "attend"])
    hk = rng.randint(1, 16)
    hq = hk * rng.choice([1, 1, 2, 3, 4, 5, 7, 8])
    layout, ladder, pos = rng.choice(["adjacent", "halves"]), rng.choice(["axis", "whole"]), rng.choice(["int", "float"])
    gains = rng.random() < 0.7
    if op in ("norm_rope", "norm_rope_back"):
        d = rng.choice([64, 80, 96, 128, 128, 128, 256])
        n = min(_log(rng, 1, 31200), 31200 * 40 * 128 // (hq * d))
        return _heads(op, n, hq, hk, d, rng.choice(["bf16", "bf16", "fp16", "fp32"]), layout, ladder, pos, gains)
    d = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 48, 64, 128, 256, 1560])
    order = rng.choice(["tokens", "heads"])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    seqs = _log(rng, 1, 128)
    new = 1 if rng.random() < 0.4 else _log(rng, 1, 10920)
    cached = _log(rng, 1, 32768) - 1
    while seqs * (new + cached) * hk * d > 31200 * 40 * 128:     # the caches of the largest listed case
        seqs, cached, new = max(1, seqs // 2), cached * 3 // 4, max(1, new * 3 // 4)
    if op == "append":
        return _append(seqs, new, cached, hq if rng.random() < 0.8 else 0, hk, d, page, dtype, layout, ladder, pos, gains,
                       True, order)
    group = rng.choice([0, 1, 1, rng.randint(2, 1560)])
    window = rng.randint(1, max(1, 8192 // group)) if group and rng.random() < 0.3 else 0
    return _attend(seqs, new, cached, hq, hk, d, page, dtype, group, window, True, order)


# --------------------------------------------------------------------------------------------------------- the inputs
def lengths(c):
    """New and cached tokens of every sequence (the first has the most)."""
    rng = random.Random(c["seqs"] * 1000003 + c["new"] * 101 + c["cached"])
    new, cached = [c["new"]], [c["cached"]]
    for _ in range(c["seqs"] - 1):
        if c["ragged"]:
            new.append(1 if rng.random() < 0.5 else rng.randint(1, c["new"]))
            cached.append(rng.randint(c["cached"] // 4, c["cached"]))
        else:
            new.append(c["new"])
            cached.append(c["cached"])
    return new, cached


def _rng(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) + 1)


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV, dtype=dtype)


def _widths(c):
    """Elements of a head that turn with the frame, the row and the column."""
    d = c["d"]
    rest = d // 3 // 2 * 2
    return [d - 2 * rest, rest, rest]


def _positions(c, n, g):
    """(frame, row, column) of n tokens on a grid that holds them."""
    side = max(1, int(math.sqrt(n / 8.0)))
    i = torch.arange(n, device=DEV)
    axes = torch.stack([i // (side * side), i // side % side, i % side])
    axes = axes + torch.randint(0, 7, (3, 1), generator=g, device=DEV)
    return (axes.to(torch.float32) * 0.25 if c["pos"] == "float" else axes.to(torch.int32)).contiguous()


def _gains(c, g):
    return [1.0 + 0.2 * _randn(g, c["d"]) if c["gains"] else None for _ in range(2)]


def _cache(c, pages, g):
    shape = (pages, c["page"], c["hk"], c["d"]) if c["order"] == "tokens" else (pages, c["hk"], c["page"], c["d"])
    t = _randn(g, *shape, dtype=TYPES[c["type"]])
    return t if c["order"] == "tokens" else t.transpose(1, 2)      # [pages, tokens of a page, heads, d] either way


def prepare(case, seed):
    c, g = case, _rng(seed)
    s = {"case": c}
    if c["op"] in ("norm_rope", "norm_rope_back"):
        n, t = c["n"], TYPES[c["type"]]
        wide = 1.0 + 4.0 * torch.rand(c["d"], generator=g, device=DEV) ** 4      # some features larger than the others
        s["q"], s["k"] = ((_randn(g, n, h, c["d"]) * wide).to(t) for h in (c["hq"], c["hk"]))
        s["positions"] = _positions(c, n, g)
        s["q_weight"], s["k_weight"] = _gains(c, g)
        if c["op"] == "norm_rope_back":
            s["dq"], s["dk"] = (_randn(g, n, h, c["d"]).to(t) for h in (c["hq"], c["hk"]))
        return s
    t = TYPES[c["type"]]
    new, cached = lengths(c)
    n, total = sum(new), [a + b for a, b in zip(new, cached)]
    need = [-(-m // c["page"]) for m in total]
    pages, wide = sum(need) + 3, max(need)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table, at = torch.zeros((c["seqs"], wide), dtype=torch.int32, device=DEV), 0
    for i, m in enumerate(need):
        table[i, :m] = order[at:at + m]
        at += m
    starts = [0]
    for m in new:
        starts.append(starts[-1] + m)
    s["table"] = table
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s["lengths"] = torch.tensor(total, dtype=torch.int32, device=DEV)
    s["k_cache"], s["v_cache"] = _cache(c, pages, g), _cache(c, pages, g)
    if c["op"] == "append":
        # a projection's rows: queries, keys and values of a token side by side
        rows = _randn(g, n, c["hq"] + 2 * c["hk"], c["d"]).to(t)
        s["q"] = rows[:, : c["hq"]] if c["hq"] else None
        s["k"], s["v"] = rows[:, c["hq"]: c["hq"] + c["hk"]], rows[:, c["hq"] + c["hk"]:]
        s["positions"] = _positions(c, n, g)
        s["q_weight"], s["k_weight"] = _gains(c, g)
    else:
        heat = 0.5 + 2.0 * torch.rand((c["hq"], 1), generator=g, device=DEV)     # some heads look more closely than others
        s["q"] = (_randn(g, n, c["hq"], c["d"]) * heat).to(t)
        if own:
            from paper_2607_28144_b200 import binding

            size = binding.regenvc_paged_attn_workspace_bytes(c["hq"], c["hk"], c["d"])
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms
def _turns(s, c):
    """cos and sin [tokens, 1, pairs] in 32 bits, from angles in 64."""
    parts, total, j = [], sum(_widths(c)), 0
    for a, w in enumerate(_widths(c)):
        i = torch.arange(w // 2, device=DEV, dtype=torch.float64)
        f = THETA ** (-2.0 * i / w) if c["ladder"] == "axis" else THETA ** (-2.0 * (i + j) / total)
        parts.append(s["positions"][a].double()[:, None] * f)
        j += w // 2
    ang = torch.cat(parts, dim=1)[:, None, :]
    return ang.cos().float(), ang.sin().float()


def _turn(x, cos, sin, c):
    half = c["d"] // 2
    lo, hi = (slice(0, None, 2), slice(1, None, 2)) if c["layout"] == "adjacent" else (slice(0, half), slice(half, None))
    y = torch.empty_like(x)
    y[..., lo] = x[..., lo] * cos - x[..., hi] * sin
    y[..., hi] = x[..., hi] * cos + x[..., lo] * sin
    return y


def _norm_turn(x, w, cos, sin, c):
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    return _turn(x if w is None else x * w, cos, sin, c)


def _plain_back(s, c):
    cos, sin = _turns(s, c)
    out = {}
    for name in ("q", "k"):
        x, w = s[name].float(), s[name + "_weight"]
        r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
        n = x * r
        g = _turn(s["d" + name].float(), cos, -sin, c)
        if w is not None:
            out["d" + name + "_weight"] = (g * n).sum(dim=(0, 1), dtype=torch.float64).float()
            g = g * w
        out["d" + name] = (r * (g - n * (g * n).mean(dim=-1, keepdim=True))).to(s[name].dtype)
    return _in_order(out)


def _in_order(grads):
    return {k: grads[k] for k in ("dq", "dk", "dq_weight", "dk_weight") if grads.get(k) is not None}


def _plain_append(s, c):
    cos, sin = _turns(s, c)
    t = TYPES[c["type"]]
    k = _norm_turn(s["k"], s["k_weight"], cos, sin, c).to(t)
    starts, counts = s["starts"][:-1].long(), (s["starts"][1:] - s["starts"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(c["seqs"], device=DEV), counts, output_size=k.shape[0])
    at = torch.arange(k.shape[0], device=DEV) - starts[seq] + (s["lengths"].long() - counts)[seq]
    page = s["table"][seq, at // c["page"]].long()
    s["k_cache"][page, at % c["page"]] = k
    s["v_cache"][page, at % c["page"]] = s["v"]
    q = _norm_turn(s["q"], s["q_weight"], cos, sin, c).to(t) if c["hq"] else None
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _limits(c, new, total):
    """First and one past the last cached token that each new token of a sequence sees."""
    p = torch.arange(total - new, total, device=DEV)
    if not c["group"]:
        return torch.zeros_like(p), torch.full_like(p, total)
    block = p // c["group"]
    hi = ((block + 1) * c["group"]).clamp(max=total)
    lo = ((block - c["window"] + 1) * c["group"]).clamp(min=0) if c["window"] else torch.zeros_like(p)
    return lo, hi


def _plain_attend(s, c):
    new, cached = lengths(c)
    out, at, share = torch.empty_like(s["q"]), 0, c["hq"] // c["hk"]
    for i, (m, old) in enumerate(zip(new, cached)):
        total = m + old
        pages = s["table"][i, : -(-total // c["page"])].long()
        lo, hi = _limits(c, m, total)
        j = torch.arange(total, device=DEV)
        hide = (j < lo[:, None]) | (j >= hi[:, None])
        heads = max(1, (1 << 30) // (m * total * share))     # heads of the cache in hand at a time
        for h in range(0, c["hk"], heads):
            e = min(c["hk"], h + heads)
            k = s["k_cache"][pages, :, h:e].flatten(0, 1)[:total].float()
            v = s["v_cache"][pages, :, h:e].flatten(0, 1)[:total].float()
            q = s["q"][at:at + m, h * share:e * share].float().unflatten(1, (e - h, share))
            x = q.permute(1, 2, 0, 3).flatten(1, 2) @ k.permute(1, 2, 0)            # [heads, share * m, total]
            x = (x * (1.0 / math.sqrt(c["d"]))).unflatten(1, (share, m)).masked_fill_(hide, -math.inf)
            x = torch.exp(x - x.amax(dim=-1, keepdim=True))
            norm = x.sum(dim=-1, keepdim=True)
            y = (x.flatten(1, 2) @ v.permute(1, 0, 2)).unflatten(1, (share, m)) / norm
            out[at:at + m, h * share:e * share] = y.permute(2, 0, 1, 3).flatten(1, 2).to(out.dtype)
        at += m
    return {"out": out}


# ------------------------------------------------------------------------------------------------------- the operators
def _own(s, c):
    from paper_2607_28144_b200 import binding

    if c["op"] != "attend":
        how = dict(rope_theta=THETA, halves=c["layout"] == "halves", whole_ladder=c["ladder"] == "whole", eps=EPS,
                   q_weight=s["q_weight"], k_weight=s["k_weight"])
    if c["op"] == "norm_rope":
        q, k = binding.regenvc_qk_norm_rope_forward(s["q"], s["k"], s["positions"], _widths(c), **how)
        return {"q": q, "k": k}
    if c["op"] == "norm_rope_back":
        g = binding.regenvc_qk_norm_rope_backward(s["dq"], s["dk"], s["q"], s["k"], s["positions"], _widths(c), **how)
        return _in_order(g)
    if c["op"] == "append":
        if not c["hq"]:
            how["q_weight"] = None
        q = binding.regenvc_paged_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["starts"],
                                         q=s["q"], positions=s["positions"], widths=_widths(c), norm=binding.NORM_RMS, **how)
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    out, _ = binding.regenvc_paged_attn_forward(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], s["starts"],
                                                group=c["group"], window=c["window"], workspace=s["workspace"])
    return {"out": out}


def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c)
    if c["op"] == "norm_rope":
        cos, sin = _turns(s, c)
        return {n: _norm_turn(s[n], s[n + "_weight"], cos, sin, c).to(s[n].dtype) for n in ("q", "k")}
    if c["op"] == "norm_rope_back":
        return _plain_back(s, c)
    return _plain_append(s, c) if c["op"] == "append" else _plain_attend(s, c)


# ------------------------------------------------------------------------------------------------------------ the work
def _seen(c):
    """(query, key) pairs that attend, and cached tokens that any query sees, over all sequences."""
    pairs = keys = 0
    for m, old in zip(*lengths(c)):
        total, b, w = m + old, c["group"], c["window"]
        if not b:
            pairs, keys = pairs + m * total, keys + total
            continue
        p = old
        while p < total:                         # the new tokens of one group see the same keys
            end = min(total, (p // b + 1) * b)
            lo = max(0, (p // b - w + 1) * b) if w else 0
            pairs += (end - p) * (end - lo)
            p = end
        keys += total - (max(0, (old // b - w + 1) * b) if w else 0)
    return pairs, keys


def work(case):
    c, size = case, SIZE[case["type"]]
    if c["op"] in ("norm_rope", "norm_rope_back"):
        e = c["n"] * (c["hq"] + c["hk"]) * c["d"]
        if c["op"] == "norm_rope":
            return {"bytes": 2 * e * size + 12 * c["n"] + 8 * c["d"] * c["gains"], "flops": 7 * e}
        return {"bytes": 3 * e * size + 12 * c["n"] + 16 * c["d"] * c["gains"], "flops": 14 * e}
    n = sum(lengths(c)[0])
    lists = 4 * n + 8 * c["seqs"]
    if c["op"] == "append":     # q, k, v in; q out; k, v into the cache
        e = n * (c["hq"] + 2 * c["hk"]) * c["d"]
        return {"bytes": 2 * e * size + 12 * n + lists, "flops": 7 * n * (c["hq"] + c["hk"]) * c["d"]}
    pairs, keys = _seen(c)
    return {"bytes": 2 * n * c["hq"] * c["d"] * size + 2 * keys * c["hk"] * c["d"] * size + 4 * keys // c["page"] + lists,
            "flops": 4.0 * pairs * c["hq"] * c["d"]}


# ------------------------------------------------------------------------------------------- the definitions, in 64 bits
def _phase(s, c):
    """e^(i angle) [tokens, 1, pairs]."""
    widths, turn, j = _widths(c), [], 0
    for a, w in enumerate(widths):
        for i in range(w // 2):
            f = THETA ** (-2.0 * i / w) if c["ladder"] == "axis" else THETA ** (-2.0 * j / sum(widths))
            turn.append(s["positions"][a].double() * f)
            j += 1
    return torch.polar(torch.ones((), dtype=torch.float64, device=DEV), torch.stack(turn, dim=1))[:, None, :]


def _exact_head(x, w, z, c):
    x = x / ((x ** 2).sum(-1, keepdim=True) / c["d"] + EPS).sqrt()
    x = x if w is None else x * w
    if c["layout"] == "adjacent":
        return torch.view_as_real(torch.view_as_complex(x.unflatten(-1, (-1, 2)).contiguous()) * z).flatten(-2)
    r = torch.complex(x[..., : c["d"] // 2], x[..., c["d"] // 2:]) * z
    return torch.cat([r.real, r.imag], dim=-1)


def _exact_back(s, c):
    """What automatic differentiation of the definition gives in 64 bits, some tokens at a time."""
    out, step = {}, max(1, (1 << 24) // (c["hq"] * c["d"]))
    z = _phase(s, c)
    for name in ("q", "k"):
        w = s[name + "_weight"]
        w = None if w is None else w.double().requires_grad_()
        parts = []
        for a in range(0, c["n"], step):
            at = slice(a, a + step)
            x = s[name][at].double().requires_grad_()
            (_exact_head(x, w, z[at], c) * s["d" + name][at].double()).sum().backward()
            parts.append(x.grad)
        out["d" + name] = torch.cat(parts)
        if w is not None:
            out["d" + name + "_weight"] = w.grad
    return _in_order(out)


def _exact_append(s, c):
    """Token by token into copies of the caches."""
    z = _phase(s, c)
    wk, wq = (None if s[n] is None else s[n].double() for n in ("k_weight", "q_weight"))
    k = _exact_head(s["k"].double(), wk, z, c)
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    row, table = 0, s["table"].tolist()
    for i, (m, old) in enumerate(zip(*lengths(c))):
        p = old
        while p < old + m:                       # the part of a sequence's new tokens that lies on one page
            e = min(old + m, (p // c["page"] + 1) * c["page"])
            page, a = table[i][p // c["page"]], p % c["page"]
            kc[page, a:a + e - p] = k[row:row + e - p]
            vc[page, a:a + e - p] = s["v"][row:row + e - p].double()
            row, p = row + e - p, e
    q = _exact_head(s["q"].double(), wq, z, c) if c["hq"] else None
    return {"q": q, "k_cache": kc, "v_cache": vc}


def _exact_attend(s, c):
    """Head by head and some queries at a time: softmax weights through the logarithm of their sum."""
    share, row = c["hq"] // c["hk"], 0
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    for i, (m, old) in enumerate(zip(*lengths(c))):
        total = m + old
        j = torch.arange(total, device=DEV)
        where = s["table"][i].long()[j // c["page"]], j % c["page"]
        step = max(1, (1 << 27) // total)
        for h in range(c["hk"]):
            k, v = (s[n][where[0], where[1], h].double() for n in ("k_cache", "v_cache"))
            for a in range(0, m, step):
                e = min(m, a + step)
                p = torch.arange(old + a, old + e, device=DEV)[:, None]
                see = torch.ones((e - a, total), dtype=torch.bool, device=DEV)
                if c["group"]:
                    see = j // c["group"] <= p // c["group"]
                    if c["window"]:
                        see &= j // c["group"] > p // c["group"] - c["window"]
                for b in range(h * share, (h + 1) * share):
                    x = s["q"][row + a:row + e, b].double() @ k.t() / c["d"] ** 0.5
                    x = torch.where(see, x, -math.inf)
                    out[row + a:row + e, b] = torch.exp(x - torch.logsumexp(x, dim=1, keepdim=True)) @ v
        row += m
    return {"out": out}


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "norm_rope":
        z = _phase(s, c)
        return {n: _exact_head(s[n].double(), None if s[n + "_weight"] is None else s[n + "_weight"].double(), z, c)
                for n in ("q", "k")}
    if c["op"] == "norm_rope_back":
        return _exact_back(s, c)
    return _exact_append(s, c) if c["op"] == "append" else _exact_attend(s, c)
