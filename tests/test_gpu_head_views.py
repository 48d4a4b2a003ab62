"""Norm and rotation of queries and keys that are views of one tensor, in place, in any order of its axes."""
import itertools

import pytest
import torch

from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def views(order, n, heads, d, dtype):
    """Three operands [n, heads, d] in one tensor whose axes (n, 3, h) lie in the given order, d last; and the tensor."""
    size = {"n": n, "3": 3, "h": heads}
    all3 = torch.randn(*(size[a] for a in order), d, generator=torch.Generator().manual_seed(n)).to(dtype).to(DEV)
    return all3.permute(*(order.index(a) for a in "3nh"), 3), all3


@pytest.mark.parametrize("order", ["".join(o) for o in itertools.permutations("n3h")])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("n,heads", [(37, 4), (37, 1), (1, 4)])
def test_in_place_among_the_others(order, dtype, n, heads):
    d = 64
    x, room = views(order, n, heads, d, dtype)
    kept = [t.clone(memory_format=torch.contiguous_format) for t in x]
    w = torch.linspace(0.5, 1.5, d, device=DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV).view(1, -1)
    how = dict(q_weight=w, k_weight=w)
    want = B.regenvc_qk_norm_rope_forward(kept[0], kept[1], pos, [d], **how)
    grads = B.regenvc_qk_norm_rope_backward(kept[0], kept[1], *want, pos, [d], **how)
    B.regenvc_qk_norm_rope_forward(x[0], x[1], pos, [d], q_out=x[0], k_out=x[1], **how)
    assert torch.equal(x[0], want[0]) and torch.equal(x[1], want[1]) and torch.equal(x[2], kept[2])
    x[0].copy_(kept[0]), x[1].copy_(kept[1])
    got = B.regenvc_qk_norm_rope_backward(x[0], x[1], *want, pos, [d], dq=x[0], dk=x[1], **how)
    assert torch.equal(x[0], grads["dq"]) and torch.equal(x[1], grads["dk"]) and torch.equal(x[2], kept[2])
    assert torch.equal(got["dq_weight"], grads["dq_weight"]) and torch.equal(got["dk_weight"], grads["dk_weight"])


@pytest.mark.parametrize("order", ["".join(o) for o in itertools.permutations("n3h")])
def test_appending_with_the_queries_in_place(order):
    n, heads, d = 20, 3, 64
    x, _ = views(order, n, heads, d, BF)
    kept = [t.clone(memory_format=torch.contiguous_format) for t in x]
    pos = torch.arange(n, dtype=torch.int32, device=DEV).view(1, -1)
    lists = (torch.tensor([[1, 0]], dtype=torch.int32, device=DEV), torch.tensor([n], dtype=torch.int32, device=DEV),
             torch.tensor([0, n], dtype=torch.int32, device=DEV))
    results = []
    for (q, k, v), place in ((kept, None), (x, x[0])):
        caches = [torch.zeros(2, 16, heads, d, dtype=BF, device=DEV) for _ in range(2)]
        out = B.regenvc_paged_append(k, v, *caches, *lists, q=q, positions=pos, widths=[d], norm=B.NORM_RMS, q_out=place)
        results.append((out.contiguous(), *caches))
    assert all(torch.equal(a, b) for a, b in zip(*results)) and B.regenvc_device_status() == B.OK
    assert torch.equal(x[1], kept[1]) and torch.equal(x[2], kept[2])


@pytest.mark.parametrize("heads,far", [(3, (1 << 30) + 64), (2, 1 << 31)])
def test_one_token_of_heads_that_lie_far_apart(heads, far):
    """A [heads, tokens, d] buffer of more than 2^31 elements, one token of it."""
    d = 64
    room = torch.empty((heads - 1) * far + d, dtype=BF, device=DEV)
    x = room.as_strided((1, heads, d), (d, far, 1))
    x.copy_(torch.randn(1, heads, d, generator=torch.Generator().manual_seed(1)).to(BF))
    near, pos = x.contiguous(), torch.full((1, 1), 9, dtype=torch.int32, device=DEV)
    want = B.regenvc_qk_norm_rope_forward(near, None, pos, [d])[0]

    def close(a, b):     # (vectors more than 2 GB apart take the form without 16-byte accesses, which sums in another order)
        return ((a.double() - b.double()).abs() <= 2.0 ** -7 * b.double().abs() + 1e-5).all()

    assert close(B.regenvc_qk_norm_rope_forward(x, None, pos, [d])[0], want)
    caches = [torch.zeros(1, 16, heads, d, dtype=BF, device=DEV) for _ in range(4)]
    lists = (torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV),
             torch.tensor([0, 1], dtype=torch.int32, device=DEV))
    q = B.regenvc_paged_append(x, x, *caches[:2], *lists, q=x, positions=pos, widths=[d], norm=B.NORM_RMS)
    p = B.regenvc_paged_append(near, near, *caches[2:], *lists, q=near, positions=pos, widths=[d], norm=B.NORM_RMS)
    assert close(q, p) and close(caches[0], caches[2]) and torch.equal(caches[1], caches[3])
    outs = [B.regenvc_paged_attn_forward(t, *caches[2:], *lists, lse=True) for t in (x, near)]
    assert all(torch.equal(a, b) for a, b in zip(*outs)) and B.regenvc_device_status() == B.OK
