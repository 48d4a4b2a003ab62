"""Caches as views of one tensor: a page's, a slot's or a head's key beside its value in any order of the axes, axes with one
entry in tensors of more than 2^31 elements, and the longest sequences."""
import itertools

import pytest
import torch

from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def lists(table, lengths, starts):
    return tuple(torch.tensor(x, dtype=torch.int32, device=DEV) for x in (table, lengths, starts))


def views(order, pages, slots, heads, d):
    """K and V [pages, slots, heads, d] in one tensor whose axes (p, 2, s, h) lie in the given order, d last."""
    size = {"p": pages, "2": 2, "s": slots, "h": heads}
    both = torch.zeros(*(size[a] for a in order), d, dtype=BF, device=DEV)
    both = both.permute(*(order.index(a) for a in "2psh"), 4)
    return both[0], both[1]


@pytest.mark.parametrize("order", ["".join(o) for o in itertools.permutations("p2sh")])
@pytest.mark.parametrize("pages,slots,heads", [(7, 16, 3), (7, 16, 1), (1, 96, 2)])
def test_keys_beside_values(order, pages, slots, heads):
    g = torch.Generator().manual_seed(0)
    n, d = 90, 64
    q = torch.randn(n, 2 * heads, d, generator=g).to(BF).to(DEV)
    k, v = (torch.randn(n, heads, d, generator=g).to(BF).to(DEV) for _ in range(2))
    where = lists([[(5 * i + 2) % pages for i in range(-(-n // slots))]], [n], [0, n])
    apart = [torch.zeros(pages, slots, heads, d, dtype=BF, device=DEV) for _ in range(2)]
    beside = views(order, pages, slots, heads, d)
    for caches in (apart, beside):
        B.regenvc_paged_append(k, v, *caches, *where, norm=B.NORM_RMS)
    assert torch.equal(apart[0], beside[0]) and torch.equal(apart[1], beside[1])
    outs = [B.regenvc_paged_attn_forward(q, *caches, *where, group=1)[0] for caches in (apart, beside)]
    assert torch.equal(*outs) and B.regenvc_device_status() == B.OK


def test_a_slots_values_behind_its_keys_with_another_step_from_head_to_head():
    n, heads, d = 40, 3, 64
    k, v = (torch.randn(n, heads, d, generator=torch.Generator().manual_seed(s)).to(BF).to(DEV) for s in (5, 6))
    both = torch.zeros(3, 16, heads * (d + d + 8), dtype=BF, device=DEV)
    kc, vc = both[..., :heads * d].unflatten(2, (heads, d)), both[..., heads * d:].unflatten(2, (heads, d + 8))[..., :d]
    B.regenvc_paged_append(k, v, kc, vc, *lists([[2, 0, 1]], [n], [0, n]))
    assert B.regenvc_device_status() == B.OK
    for c, t in ((kc, k), (vc, v)):
        assert torch.equal(c[[2, 0, 1]].flatten(0, 1)[:n], t)
    assert (both.view(48, -1)[:, heads * d:].unflatten(1, (heads, d + 8))[..., d:] == 0).all()


def test_one_slot_and_one_page():
    """Axes with one entry, whose strides mean nothing."""
    g = torch.Generator().manual_seed(1)
    for order in ("p2sh", "ps2h", "psh2", "2psh", "h2ps"):
        for pages, slots in ((8, 1), (1, 8), (1, 1)):
            n = pages * slots
            k, v = (torch.randn(n, 2, 64, generator=g).to(BF).to(DEV) for _ in range(2))
            kc, vc = views(order, pages, slots, 2, 64)
            B.regenvc_paged_append(k, v, kc, vc, *lists([list(range(pages))], [n], [0, n]))
            assert B.regenvc_device_status() == B.OK
            assert torch.equal(kc.reshape(n, 2, 64), k) and torch.equal(vc.reshape(n, 2, 64), v)


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


def test_sequences_of_more_than_2_30_tokens_are_reported():
    """A table may name a page again and again; positions are held as far as 2^30."""
    slots = 1 << 20
    kc, vc = (torch.zeros(2, slots, 1, 64, dtype=BF, device=DEV) for _ in range(2))
    x = torch.ones(1, 1, 64, dtype=BF, device=DEV)
    table = [[0] * 1024 + [1]]
    B.regenvc_paged_append(x, x, kc, vc, *lists(table, [1 << 30], [0, 1]))
    assert B.regenvc_device_status() == B.OK and (kc[0, -1] == 1).all() and kc.sum() == 64
    B.regenvc_paged_append(x, x, kc, vc, *lists(table, [(1 << 30) + 1], [0, 1]))
    assert B.regenvc_device_status() == B.ERR_RANGE and kc.sum() == 64
    B.regenvc_paged_attn_forward(x, kc, vc, *lists(table, [(1 << 30) + 1], [0, 1]))
    assert B.regenvc_device_status() == B.ERR_RANGE
