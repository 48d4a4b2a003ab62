"""Infinities and sums past fp32's range in the norm and rotation of queries and keys: what they reach and what not."""
import math

import pytest
import torch

from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32

# head_dim, widths of the rotation (adjacent pairs: the elements behind it do not turn)
PARTIAL = [(128, (32,)), (128, (44, 20)), (64, (24, 20, 2)), (256, (6,)), (80, (20, 12)), (48, (46,)), (32, (16,)), (16, (2,))]


def turned(x, widths, pos, theta=1e4, back=False):
    """x [tokens, heads, d] in 64 bits with its leading pairs turned and all else as it is."""
    y, at = x.clone(), 0
    for a, w in enumerate(widths):
        angle = pos[a].double()[:, None] * theta ** (-2.0 * torch.arange(w // 2, device=DEV, dtype=torch.float64) / w)
        c, s = angle.cos()[:, None], angle.sin()[:, None] * (-1 if back else 1)
        u, v = x[..., at:at + w:2], x[..., at + 1:at + w:2]
        y[..., at:at + w:2], y[..., at + 1:at + w:2] = u * c - v * s, v * c + u * s
        at += w
    return y


def same(got, want, tolerance):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    assert torch.equal(got[torch.isinf(got)].sign(), want[torch.isinf(want)].sign())
    fine = torch.isfinite(want)
    assert ((got - want).abs()[fine] <= tolerance * want.abs()[fine] + 1e-5).all()


@pytest.mark.parametrize("dtype", [BF, FP, F32])
@pytest.mark.parametrize("d,widths", PARTIAL)
def test_infinities_behind_the_rotation_stay_in_their_element(dtype, d, widths):
    """An append without a norm: keys with infinite elements in the part that does not turn, in rows of either alignment."""
    g = torch.Generator().manual_seed(d)
    n, first = 12, sum(widths)
    x = torch.randn(n, 3, d, generator=g).to(dtype).to(DEV)
    for i in range(n):
        x[i, i % 3, first + (5 * i) % (d - first)] = math.inf if i % 2 else -math.inf
    pos = torch.randint(1, 50, (len(widths), n), generator=g, dtype=torch.int32).to(DEV)
    want = turned(x.double(), widths, pos)
    lists = (torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.tensor([n], dtype=torch.int32, device=DEV),
             torch.tensor([0, n], dtype=torch.int32, device=DEV))
    for off in (0, 1):
        room = torch.zeros(x.numel() + 1, dtype=dtype, device=DEV)
        rows = room[off:off + x.numel()].view(x.shape)
        rows.copy_(x)
        kc, vc = (torch.zeros(1, 16, 3, d, dtype=dtype, device=DEV) for _ in range(2))
        q = B.regenvc_paged_append(rows, rows, kc, vc, *lists, q=rows, positions=pos, widths=list(widths))
        assert B.regenvc_device_status() == B.OK
        same(q, want, 2 * torch.finfo(dtype).eps)
        same(kc[0, :n], want, 2 * torch.finfo(dtype).eps)
        assert torch.equal(vc[0, :n], rows)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("d,widths", PARTIAL)
def test_an_infinite_element_of_a_normalised_row(dtype, d, widths):
    """x / sqrt(mean(x^2)): the infinite element is not a number, the others are zeros, turned or not."""
    first = sum(widths)
    x = torch.ones(4, 1, d, dtype=dtype, device=DEV)
    for i in range(4):
        x[i, 0, first + i * (d - first - 1) // 3] = math.inf
    pos = torch.full((len(widths), 4), 3, dtype=torch.int32, device=DEV)
    want = torch.where(torch.isinf(x), math.nan, 0.0).double()
    for off in (0, 1):
        room = torch.zeros(x.numel() + 1, dtype=dtype, device=DEV)
        rows = room[off:off + x.numel()].view(x.shape)
        rows.copy_(x)
        same(B.regenvc_qk_norm_rope_forward(rows, None, pos, list(widths))[0], want, 0.0)


@pytest.mark.parametrize("d,widths", PARTIAL)
def test_an_infinite_gradient_behind_the_rotation(d, widths):
    """dw of its neighbours, which no other row's infinity belongs to, stays finite."""
    g = torch.Generator().manual_seed(d)
    first, n = sum(widths), 40
    x, dy = (torch.randn(n, 2, d, generator=g).to(DEV) for _ in range(2))
    at = first + (d - first) // 2
    dy[7, 1, at] = math.inf
    w = torch.ones(d, device=DEV)
    pos = torch.randint(1, 50, (len(widths), n), generator=g, dtype=torch.int32).to(DEV)
    x64 = x.double()
    norm = x64 / torch.sqrt((x64 * x64).mean(-1, keepdim=True) + 1e-6)
    want = (turned(dy.double(), widths, pos, back=True) * norm).sum((0, 1))
    for off in (0, 1):
        room = torch.zeros(x.numel() + 1, device=DEV)
        rows = room[off:off + x.numel()].view(x.shape)
        rows.copy_(x)
        got = B.regenvc_qk_norm_rope_backward(dy, None, rows, None, pos, list(widths), q_weight=w)
        same(got["dq_weight"], want, 1e-4)
        assert torch.isfinite(got["dq"][:7]).all() and torch.isfinite(got["dq"][8:]).all() and torch.isfinite(got["dq"][7, 0]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("d", [64, 128, 250])
def test_gradients_of_a_row_past_the_range_are_zeros(dtype, halves, d):
    """Its sum of squares passes fp32's range, so it normalises to 0: so do its gradients, and other rows' are as without it."""
    g = torch.Generator().manual_seed(d)
    x, dy = (torch.randn(6, 2, d, generator=g).to(dtype).to(DEV) for _ in range(2))
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(DEV)
    pos = torch.arange(6, dtype=torch.int32, device=DEV).view(1, -1)
    how = dict(halves=halves, q_weight=w)
    x[2, 1] = 0
    dy[2, 1] = dy[2, 1].abs() + 1                                    # the sum of dy x passes the range too
    base = B.regenvc_qk_norm_rope_backward(dy, None, x, None, pos, [d], **how)
    zero_row = dict(q_weight=w, halves=halves)
    for big in (2e19, 1e30, 3e38):
        y = x.clone()
        y[2, 1] = torch.where(torch.arange(d, device=DEV) % 2 == 0, big, 0.5 * big)
        assert (B.regenvc_qk_norm_rope_forward(y, None, pos, [d], **zero_row)[0][2, 1] == 0).all()
        got = B.regenvc_qk_norm_rope_backward(dy, None, y, None, pos, [d], **how)
        assert (got["dq"][2, 1] == 0).all()
        keep = torch.ones(6, 2, dtype=torch.bool, device=DEV)
        keep[2, 1] = False
        assert torch.equal(got["dq"][keep], base["dq"][keep])
        assert torch.isfinite(got["dq_weight"]).all() and torch.equal(got["dq_weight"], base["dq_weight"])


@pytest.mark.parametrize("d", [64, 128, 250])
def test_gradients_of_an_infinite_element(d):
    """As in the forward pass: not a number in its place, zeros beside it, and the other rows as ever."""
    g = torch.Generator().manual_seed(d)
    x, dy = (torch.randn(6, 2, d, generator=g).to(DEV) for _ in range(2))
    w = torch.ones(d, device=DEV)
    base = B.regenvc_qk_norm_rope_backward(dy, None, x, None, q_weight=w)
    x[2, 1, 5] = math.inf
    got = B.regenvc_qk_norm_rope_backward(dy, None, x, None, q_weight=w)
    place = torch.zeros(6, 2, d, dtype=torch.bool, device=DEV)
    place[2, 1, 5] = True
    assert torch.equal(torch.isnan(got["dq"]), place) and torch.equal(torch.isnan(got["dq_weight"]), place[2, 1])
    row = got["dq"][2, 1].nan_to_num()
    assert (row == 0).all()
    keep = ~place.any(-1)
    assert torch.equal(got["dq"][keep], base["dq"][keep])
