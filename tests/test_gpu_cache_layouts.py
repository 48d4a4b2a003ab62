"""Caches as views of one tensor, of any size and order of the axes."""
import pytest
import torch

from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def lists(table, lengths, starts):
    return tuple(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (table, lengths, starts))


def test_one_head_in_a_cache_of_more_than_2_31_elements():
    pages, d = 524288 + 9, 128
    both = torch.empty((pages, 2, 16, 1, d), dtype=BF, device=DEV)
    g = torch.Generator().manual_seed(2)
    k, v, q = (torch.randn(20, h, d, generator=g).to(BF).to(DEV) for h in (1, 1, 4))
    far = lists([[pages - 1, pages - 4]], [20], [0, 20])
    near, at = [torch.zeros(2, 16, 1, d, dtype=BF, device=DEV) for _ in range(2)], lists([[1, 0]], [20], [0, 20])
    outs = []
    for caches, where in (((both[:, 0], both[:, 1]), far), (near, at)):
        B.regenvc_paged_append(k, v, *caches, *where)
        outs.append(B.regenvc_paged_attn_forward(q, *caches, *where, group=1)[0])
    assert torch.equal(*outs) and B.regenvc_device_status() == B.OK
    assert torch.equal(both[pages - 1, 0, :, 0], k[:16, 0]) and torch.equal(both[pages - 4, 1, :4, 0], v[16:, 0])


def test_one_slot_in_a_cache_of_more_than_2_31_elements():
    pages, d = 524288 + 9, 128
    both = torch.empty((pages, 2, 1, 17, d), dtype=BF, device=DEV)
    k, v = (torch.randn(2, 17, d, generator=torch.Generator().manual_seed(s)).to(BF).to(DEV) for s in (3, 4))
    B.regenvc_paged_append(k, v, both[:, 0], both[:, 1], *lists([[pages - 1, 5]], [2], [0, 2]))
    assert B.regenvc_device_status() == B.OK
    assert torch.equal(both[pages - 1, :, 0], torch.stack([k[0], v[0]])) and torch.equal(both[5, :, 0], torch.stack([k[1], v[1]]))
