"""The operators around the attention in the order a block runs them: modulated norm, 4-bit QKV projection, rotation by
explicit positions, the library's attention, 4-bit output projection, gated residual step with the next norm.  Each step is
compared with its 64-bit form on the step's own input (the 4-bit rounding of a later step would otherwise turn a last-bit
difference into a whole code)."""
import pytest
import torch

import oracle
from block_ops_util import half_step, mx_codes64, mx_values64, block_norm64, rope64
from paper_2607_28144_b200 import binding as B
from paper_2607_28144_b200 import synth
from parity_util import assert_parity

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


def _block(s):
    """One pass; every intermediate result is returned."""
    n, c, h = s["n"], s["c"], s["h"]
    _, a = B.regenvc_block_norm_forward(s["x"], norm=B.NORM_LAYER, scale=s["scale"], shift=s["shift"], eps=EPS, tokens_per_mod=s["per"])
    qkv = B.regenvc_mxfp4_linear(a, s["w_qkv"], 3 * c, s["b_qkv"])
    q, k, v = (qkv[:, i * c:(i + 1) * c].view(n, h, 128) for i in range(3))
    qr, kr = B.regenvc_rope_axes(q, k, s["positions"], [44, 42, 42])
    o = torch.empty_like(qr)
    B.regenvc_cross_attn_forward(qr, kr, v.contiguous(), o)
    y = B.regenvc_mxfp4_linear(o.view(n, c), s["w_o"], c, s["b_o"])
    x2, h2 = B.regenvc_block_norm_forward(s["x"], y, gate=s["gate"], norm=B.NORM_RMS, weight=s["weight"], eps=EPS,
                                          tokens_per_mod=s["per"])
    return {"a": a, "qkv": qkv, "q": qr, "k": kr, "o": o, "y": y, "x2": x2, "h2": h2}


def _inputs(n, h, per):
    g = torch.Generator(device=DEV).manual_seed(n + h)
    r = lambda *sh: torch.randn(*sh, generator=g, device=DEV)  # noqa: E731
    c = 128 * h
    mods = 0.3 * r(-(-n // per), 6, c)
    s = {"n": n, "c": c, "h": h, "per": per, "x": (r(n, c) + 0.2).bfloat16(), "shift": mods[:, 0], "scale": mods[:, 1],
         "gate": mods[:, 2], "weight": 1 + 0.1 * r(c), "b_qkv": 0.1 * r(3 * c), "b_o": 0.1 * r(c)}
    s["wq64"], s["wo64"] = r(3 * c, c) / c ** 0.5, r(c, c) / c ** 0.5
    s["w_qkv"], s["w_o"] = B.regenvc_mxfp4_quantize(s["wq64"]), B.regenvc_mxfp4_quantize(s["wo64"])
    i = torch.arange(n, device=DEV)
    s["positions"] = torch.stack([i // 35, i // 7 % 5, i % 7]).to(torch.int32)
    return s


def _q64(x):
    codes, byte = mx_codes64(x.double())
    return mx_values64(codes, byte, x.shape[1])


def _near(got, ref, slack):
    err = (got.double() - ref).abs()
    assert torch.isfinite(got).all() and (err <= half_step(got.dtype) * ref.abs() + slack).all(), float((err - slack).max())


@pytest.mark.parametrize("n,h,per", [(1, 2, 1), (35, 2, 35), (301, 4, 100), (1000, 12, 250)])
def test_a_block_step_by_step(n, h, per):
    s = _inputs(n, h, per)
    c = s["c"]
    d = _block(s)
    assert B.regenvc_device_status() == 0
    # fp32 steps on values below 32: 2^-15 covers (64 + 70) 2^-24 32 of the norm; products: K 2^-23 of |terms|
    _, a = block_norm64(s["x"].double(), None, {"scale": s["scale"].double(), "shift": s["shift"].double()}, 1, 0, 1.0, per, EPS)
    _near(d["a"], a, 2.0 ** -11)
    for x, w, b, y in (("a", "wq64", "b_qkv", "qkv"), ("o", "wo64", "b_o", "y")):
        x64, w64 = _q64(d[x].reshape(n, c)), _q64(s[w])
        _near(d[y], x64 @ w64.t() + s[b].double(), c * 2.0 ** -23 * (x64.abs() @ w64.abs().t()) + 2.0 ** -22)
    for i, name in enumerate("qk"):
        ref, mag = rope64(d["qkv"][:, i * c:(i + 1) * c].view(n, h, 128).double(), s["positions"], [44, 42, 42], 1e4, False, False, False)
        _near(d[name], ref, 2.0 ** -21 * mag)
    v = d["qkv"][:, 2 * c:].view(n, h, 128).contiguous().cpu()
    ref = oracle.cross_attention(synth.bits(d["q"].cpu()), synth.bits(d["k"].cpu()), synth.bits(v))
    assert_parity(d["o"].cpu().double().numpy(), ref, float(v.float().abs().max()), "attention on rotated q and k")
    x2, h2 = block_norm64(s["x"].double(), d["y"].double(), {"gate": s["gate"].double(), "weight": s["weight"].double()}, 2, 0, 1.0,
                          per, EPS)
    _near(d["x2"], x2, 2.0 ** -18)
    _near(d["h2"], h2, 2.0 ** -11)


def test_the_rotation_agrees_with_the_attention_that_rotates_itself():
    """On a whole grid in order, rotating by explicit positions and attending without rotation is the library's
    self-attention, up to the rounding of rotated q and k to bf16 (2^-9 of a score's terms) instead of fp16."""
    T_, H, W, h = 3, 6, 11, 2
    n = T_ * H * W
    w = synth.Workload("grid", 41, T_, H, W, h, layers=1)
    q, k, v = (t.to(DEV) for t in synth.self_inputs(w))
    i = torch.arange(n, device=DEV)
    pos = torch.stack([i // (H * W), i // W % H, i % W]).to(torch.int32)
    qr, kr = B.regenvc_rope_axes(q, k, pos, [44, 42, 42])
    a, b = torch.empty_like(q), torch.empty_like(q)
    B.regenvc_cross_attn_forward(qr, kr, v, a)
    B.regenvc_attn_forward(q, k, v, b, T_, H, W)
    assert B.regenvc_device_status() == 0
    assert (a.float() - b.float()).abs().max() <= 2e-2 * v.float().abs().max()


def test_the_block_in_a_graph_replays_on_new_values():
    s = _inputs(210, 4, 70)
    want = _block(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _block(s)
    graph.replay()
    for k in want:
        assert torch.equal(got[k], want[k]), k
    s["x"].copy_(torch.randn(s["x"].shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(99)))
    graph.replay()
    again = _block(s)
    for k in again:
        assert torch.equal(got[k], again[k]), k
    assert B.regenvc_device_status() == 0
