"""A streaming decoder's steps with every element held to its bound: what the append wrote is read back and is what the attention
is compared on, so that nothing rounds differently on the two sides."""
import math

import pytest
import torch

from block_ops_util import U, floor_step, half_step, rope64
from paper_2607_28144_b200 import binding as B
from test_gpu_paged_attn_weights import definition

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, FP = torch.bfloat16, torch.float16


class Cache:
    """One layer's cache for several sequences, its unused slots not numbers."""

    def __init__(self, seqs, hk, d, page, pages, dtype, g):
        self.k, self.v = (torch.full((pages, page, hk, d), math.nan, dtype=dtype, device=DEV) for _ in range(2))
        self.table = torch.randperm(pages, generator=g).to(torch.int32)[: seqs * (pages // seqs)].view(seqs, -1).to(DEV)
        self.lengths = [0] * seqs
        self.page = page

    def lists(self, new):
        self.lengths = [a + b for a, b in zip(self.lengths, new)]
        starts = [sum(new[:i]) for i in range(len(new) + 1)]
        return self.table, torch.tensor(self.lengths, dtype=torch.int32, device=DEV), torch.tensor(starts, dtype=torch.int32, device=DEV)

    def read(self, s):
        t = torch.arange(self.lengths[s], device=DEV)
        at = self.table[s, t // self.page].long(), t % self.page
        return self.k[at], self.v[at]


def attended(cache, new, q, out, lse, group):
    at = 0
    for s, m in enumerate(new):
        part = slice(at, at + m)
        at += m
        if not m:
            continue
        ref, ref_lse, bound, lse_bound = definition(q[part], *cache.read(s), group, 1 / math.sqrt(q.shape[2]))
        err, lse_err = (out[part].double() - ref).abs(), (lse[part].double() - ref_lse).abs()
        assert (err <= bound).all() and (lse_err <= lse_bound).all(), (s, m, float((err / bound).max()), float((lse_err / lse_bound).max()))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq,hk,d,group,norm,layout", [(6, 2, 128, 60, True, False), (4, 4, 64, 1, True, True), (5, 1, 128, 0, False, False)])
def test_frames_of_two_streams_then_single_tokens(dtype, hq, hk, d, group, norm, layout):
    g = torch.Generator().manual_seed(0)
    gains = [(1 + 0.2 * torch.randn(d, generator=g)).to(DEV) if norm else None for _ in range(2)]
    cache = Cache(2, hk, d, 48, 40, dtype, g)
    widths = [d - 2 * (d // 3 // 2 * 2), d // 3 // 2 * 2, d // 3 // 2 * 2]
    for new in ([60, 60], [60, 0], [60, 120], [1, 1], [1, 0], [0, 1], [58, 7], [300, 2]):
        n = sum(new)
        rows = torch.randn(n, hq + 2 * hk, d, generator=g).to(dtype).to(DEV)
        pos = torch.randint(0, 64, (3, n), generator=g, dtype=torch.int32).to(DEV)
        lists = cache.lists(new)
        how = dict(norm=B.NORM_RMS, q_weight=gains[0], k_weight=gains[1]) if norm else {}
        q = B.regenvc_paged_append(rows[:, hq:hq + hk], rows[:, hq + hk:], cache.k, cache.v, *lists, q=rows[:, :hq], positions=pos,
                                   widths=widths, halves=layout, **how)
        out, lse = B.regenvc_paged_attn_forward(q, cache.k, cache.v, *lists, group=group, lse=True)
        assert B.regenvc_device_status() == B.OK
        attended(cache, new, q, out, lse, group)


def test_a_window_normalised_over_all_features():
    """The model's own order: the norm over all heads' features, then an append that only rotates."""
    T, H, W, h, d = 3, 10, 16, 4, 128
    n = T * H * W
    g = torch.Generator().manual_seed(1)
    rows = [torch.randn(n, h * d, generator=g).to(BF).to(DEV) for _ in range(3)]
    gains = [(1 + 0.2 * torch.randn(h * d, generator=g)).to(DEV) for _ in range(2)]
    q, k = (B.regenvc_block_norm_forward(x, weight=w, norm=B.NORM_RMS)[1].view(n, h, d) for x, w in zip(rows, gains))
    v = rows[2].view(n, h, d)
    i = torch.arange(n, device=DEV)
    pos = torch.stack([i // (H * W), i // W % H, i % W]).to(torch.int32)
    cache = Cache(1, h, d, 64, 10, BF, g)
    lists = cache.lists([n])
    turned = B.regenvc_paged_append(k, v, cache.k, cache.v, *lists, q=q, positions=pos, widths=[44, 42, 42])
    out, lse = B.regenvc_paged_attn_forward(turned, cache.k, cache.v, *lists, lse=True)
    assert B.regenvc_device_status() == B.OK
    for x, y in ((q, turned), (k, cache.read(0)[0])):
        ref, mag = rope64(x.double(), pos, [44, 42, 42], 10000.0, False, False, False)
        # products and sums in fp32 with sines and cosines off by a few steps, and one rounding
        assert ((y.double() - ref).abs() <= half_step(BF) * ref.abs() + 16 * U * mag + floor_step(BF)).all()
    assert torch.equal(cache.read(0)[1], v)
    attended(cache, [n], turned, out, lse, 0)
