"""Rotation by explicit positions against complex multiplication in 64 bits.  Bound: the angle's fraction is rounded to
fp32 as a multiple of a half turn (|value| <= 1, so pi 2^-25 < 2^-23 of the angle), sine and cosine are within 2 ulp
(2^-23), products and sum round three times: (2^-23 + 2^-23 + 3 2^-24)(|a| + |b|) < 2^-21 (|a| + |b|), and half a step of the
result's type."""
import pytest
import torch

from block_ops_util import floor_step, half_step, rope64
from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _positions(n, axes, seed, kind="int", offset=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    if kind == "int":
        return (torch.randint(-20, 2000, (axes, n), generator=g, device=DEV) + offset).to(torch.int32)
    return (torch.rand((axes, n), generator=g, device=DEV) * 300 + offset).contiguous()


def _randn(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


def _check(got, x, pos, widths, theta=1e4, halves=False, whole=False, inverse=False):
    ref, mag = rope64(x.double(), pos, widths, theta, halves, whole, inverse)
    err = (got.double() - ref).abs()
    bound = half_step(got.dtype) * ref.abs() + 2.0 ** -21 * mag + floor_step(got.dtype)
    assert torch.isfinite(got).all() and (err <= bound).all(), f"{(err / bound.clamp_min(1e-300)).max().item():.3g} times the bound"
    total = sum(widths)
    assert torch.equal(got[..., total:], x[..., total:]), "elements behind the rotated part are copied"


CASES = [  # n, q heads, k heads, head_dim, widths
    (1, 1, 0, 2, [2]), (1, 12, 12, 128, [44, 42, 42]), (7, 3, 1, 80, [20, 28, 32]), (300, 12, 12, 128, [44, 42, 42]),
    (1000, 40, 8, 128, [32, 48, 48]), (333, 5, 5, 64, [16, 24, 24]), (50, 4, 2, 256, [64, 64, 64, 64]), (65, 2, 1, 66, [2, 4, 6]),
    (129, 6, 3, 96, [32, 16, 16]), (40, 1, 1, 250, [250]), (2500, 16, 2, 64, [64])]


@pytest.mark.parametrize("n,hq,hk,d,widths", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_rotation(n, hq, hk, d, widths, dtype):
    q = _randn(n + d, n, hq, d).to(T[dtype])
    k = _randn(n + d + 1, n, hk, d).to(T[dtype]) if hk else None
    for i, (halves, whole, inverse, kind) in enumerate([(False, False, False, "int"), (True, True, False, "float"),
                                                        (True, False, True, "int"), (False, True, True, "float")]):
        pos = _positions(n, len(widths), n + i, kind)
        qo, ko = B.regenvc_rope_axes(q, k, pos, widths, halves=halves, whole_ladder=whole, inverse=inverse)
        _check(qo, q, pos, widths, 1e4, halves, whole, inverse)
        if hk:
            _check(ko, k, pos, widths, 1e4, halves, whole, inverse)
        else:
            assert ko is None


def test_far_positions_keep_their_angles():
    """2^-53 * 2^31 turns is 2^-22 of a turn; at a position near 10^7 it is below 2^-29 and the bound above holds."""
    n, d = 64, 64
    q = _randn(1, n, 2, d)
    for kind, offset in (("int", 10_000_019), ("float", 1_000_000.0)):
        pos = _positions(n, 2, 3, kind, offset)
        qo, _ = B.regenvc_rope_axes(q, None, pos, [32, 32], rope_theta=123.0)
        _check(qo, q, pos, [32, 32], 123.0)
    edge = torch.tensor([[2 ** 31 - 1, -2 ** 31, 0, 1]], dtype=torch.int32, device=DEV)
    q = _randn(2, 4, 1, 4)
    qo, _ = B.regenvc_rope_axes(q, None, edge, [4])
    ref, mag = rope64(q.double(), edge, [4], 1e4, False, False, False)
    assert ((qo.double() - ref).abs() <= (2.0 ** -21 + 7 * 2.0 ** -21) * mag).all()   # + 2 pi 2^-22 twice (both sides round)
    assert torch.equal(qo[2], q[2])


def test_views_of_a_fused_projection_in_place_and_other_layouts():
    n, h, hk, d = 200, 6, 2, 128
    w = [44, 42, 42]
    pos = _positions(n, 3, 8)
    for dtype in T.values():
        fused = _randn(5, n, (h + 2 * hk) * d).to(dtype)
        q, k = fused[:, : h * d].view(n, h, d), fused[:, h * d: (h + hk) * d].view(n, hk, d)
        qo, ko = B.regenvc_rope_axes(q, k, pos, w)
        _check(qo, q, pos, w)
        _check(ko, k, pos, w)
        both = fused.clone()
        q2, k2 = both[:, : h * d].view(n, h, d), both[:, h * d: (h + hk) * d].view(n, hk, d)
        a, b = B.regenvc_rope_axes(q2, k2, pos, w, q_out=q2, k_out=k2)
        assert torch.equal(q2, qo) and torch.equal(k2, ko) and a is q2 and b is k2
        assert torch.equal(both[:, (h + hk) * d:], fused[:, (h + hk) * d:]), "the values beside them were written"
        # heads first
        heads = q.permute(1, 0, 2).contiguous().permute(1, 0, 2)
        out = torch.empty((h, n, d), dtype=dtype, device=DEV).permute(1, 0, 2)
        B.regenvc_rope_axes(heads, None, pos, w, q_out=out)
        assert torch.equal(out, qo)
        # rows and heads at odd distances, and an address off the 16-byte grid
        buf = torch.full((n * (h * (d + 3) + 5) + 1,), float("nan"), dtype=dtype, device=DEV)
        odd = torch.as_strided(buf, (n, h, d), (h * (d + 3) + 5, d + 3, 1), 1)
        odd.copy_(q)
        written = ~torch.isnan(buf)
        B.regenvc_rope_axes(odd, None, pos, w, q_out=odd)
        assert torch.equal(odd, qo) and torch.equal(~torch.isnan(buf), written)


def test_the_inverse_is_the_gradient_and_agrees_with_differences():
    n, h, d, w = 50, 3, 64, [16, 24, 24]
    pos = _positions(n, 3, 21)
    g = _randn(6, n, h, d)
    for halves in (False, True):
        back, _ = B.regenvc_rope_axes(g, None, pos, w, halves=halves, inverse=True)
        x = _randn(7, n, h, d).double().requires_grad_()
        y, _ = rope64(x, pos, w, 1e4, halves, False, False)
        (y * g.double()).sum().backward()
        mag = rope64(g.double(), pos, w, 1e4, halves, False, True)[1]
        assert ((back.double() - x.grad).abs() <= 2.0 ** -24 * x.grad.abs() + 2.0 ** -21 * mag).all()
        # the rotation is linear: its difference quotient along v is exactly <g, rotation of v>
        v = _randn(8, n, h, d)
        step, _ = rope64(v.double(), pos, w, 1e4, halves, False, False)
        want = float((g.double() * step).sum())
        assert abs(float((back.double() * v.double()).sum()) - want) <= 2.0 ** -20 * float((mag * v.double().abs()).sum())


def test_streams_graphs_nan_and_refusals():
    n, h, d, w = 100, 4, 128, [44, 42, 42]
    pos = _positions(n, 3, 2)
    q, k = _randn(1, n, h, d).bfloat16(), _randn(2, n, h, d).bfloat16()
    want = B.regenvc_rope_axes(q, k, pos, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = B.regenvc_rope_axes(q, k, pos, w, stream=s)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = B.regenvc_rope_axes(q, k, pos, w)
    q2, pos2 = _randn(3, n, h, d).bfloat16(), _positions(n, 3, 4)
    want2 = B.regenvc_rope_axes(q2, k, pos2, w)
    q.copy_(q2)
    pos.copy_(pos2)
    graph.replay()
    assert torch.equal(res[0], want2[0]) and torch.equal(res[1], want2[1])
    bad = q.clone()
    bad[5, 1, 6] = float("nan")
    out, _ = B.regenvc_rope_axes(bad, None, pos, w)
    hit = torch.isnan(out)
    assert hit[5, 1, 6] and hit[5, 1, 7] and hit.sum() == 2
    with pytest.raises(TypeError):
        B.regenvc_rope_axes(q, k.float(), pos, w)
    with pytest.raises(TypeError):
        B.regenvc_rope_axes(q, k, pos.long(), w)
    with pytest.raises(TypeError):
        B.regenvc_rope_axes(q, k, pos[:2], w)
    with pytest.raises(ValueError):
        B.regenvc_rope_axes(q, k[:, :1].expand(n, h, d), pos, w)
    with pytest.raises(B.RegenvcError) as e:
        B.regenvc_rope_axes(q, k, pos, [44, 42, 44])
    assert e.value.code == B.ERR_BAD_SHAPE
    with pytest.raises(B.RegenvcError) as e:
        B.regenvc_rope_axes(q, k, pos, w, q_out=k)
    assert e.value.code == B.ERR_ALIASING
