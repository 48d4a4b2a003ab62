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
