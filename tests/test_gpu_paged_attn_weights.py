"""Weights of distant keys and large values in the attention over a paged cache, and its results against bounds that count
what the kernel does and no more."""
import math

import pytest
import torch

from block_ops_util import U, floor_step, half_step
from cache_ops_util import sees
from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, FP = torch.bfloat16, torch.float16
POWER = 2.0 ** -21            # relative error of a probability's power of two (the special-function unit: 2^-22), twice


def one_sequence(q, k, v, page=64):
    """The call's arguments for one sequence whose keys and values lie in pages in reverse order."""
    pages = -(-k.shape[0] // page)
    caches = []
    for t in (k, v):
        c = torch.zeros((pages * page, *t.shape[1:]), dtype=t.dtype, device=DEV)
        c[: t.shape[0]] = t
        caches.append(c.view(pages, page, *t.shape[1:]).flip(0).contiguous())
    table = torch.arange(pages - 1, -1, -1, dtype=torch.int32, device=DEV).view(1, -1)
    return (q, *caches, table, torch.tensor([k.shape[0]], dtype=torch.int32, device=DEV),
            torch.tensor([0, q.shape[0]], dtype=torch.int32, device=DEV))


def definition(q, k, v, group, scale):
    """(out, lse, bound of |out - kernel|, bound of |lse - kernel|) in 64 bits, from the definition."""
    dtype, d, keys = q.dtype, q.shape[2], k.shape[0]
    see = sees(q.shape[0], keys, group, 0).to(DEV)
    share = q.shape[1] // k.shape[1]
    outs, lses, bounds, lse_bounds = [], [], [], []
    for a in range(q.shape[1]):
        x, kk, vv = q[:, a].double(), k[:, a // share].double(), v[:, a // share].double()
        s = (scale * (x @ kk.t())).masked_fill(~see, -math.inf)
        lse = torch.logsumexp(s, dim=1)
        w = torch.exp(s - lse[:, None])
        out, size = w @ vv, w @ vv.abs()
        # a score: d products and sums in fp32; its scale, the reference's product and their difference, which the reference's
        # distance from the maximum (32 powers of two at most) makes larger
        score = (d + 8) * U * (scale * (x.abs() @ kk.abs().t())).masked_fill(~see, 0.0).amax(dim=1) + \
            6 * U * (s.abs().masked_fill(~see, 0.0).amax(dim=1) + 32)
        # sums in fp32: 64 terms one after another in a tile, the tiles, the pieces of thread blocks; P V takes 16 keys at a time
        weight = POWER + 2 * score + (keys / 16 + 256) * 2 * U
        bounds.append((half_step(dtype) + 2 * weight)[:, None] * size + half_step(dtype) * out.abs() + floor_step(dtype))
        if dtype == FP:
            # fp16 probabilities are 2^8 at the largest of the reference's tile and 2^-24 apart below 2^-14
            bounds[-1] += 2.0 ** -33 * (see.double() @ vv.abs())
        outs.append(out)
        lses.append(lse)
        lse_bounds.append(weight + 4 * U * (lse.abs() + 32))
    return [torch.stack(t, dim=1) for t in (outs, lses, bounds, lse_bounds)]


def check(q, k, v, group=1, scale=None):
    out, lse = B.regenvc_paged_attn_forward(*one_sequence(q, k, v), group=group, scale=scale, lse=True)
    assert B.regenvc_device_status() == B.OK
    ref, ref_lse, bound, lse_bound = definition(q, k, v, group, scale or 1 / math.sqrt(q.shape[2]))
    err, lse_err = (out.double() - ref).abs(), (lse.double() - ref_lse).abs()
    assert (err <= bound).all(), float((err / bound).max())
    assert (lse_err <= lse_bound).all(), float((lse_err / lse_bound).max())
    return out, lse


def randn(*shape, dtype, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("new,keys,hq,hk,d", [(1, 1, 1, 1, 128), (1, 300, 12, 12, 128), (3, 4000, 8, 2, 64), (200, 1000, 4, 2, 128),
                                              (300, 700, 3, 1, 64), (16, 9000, 2, 2, 128)])
def test_against_the_definition(dtype, new, keys, hq, hk, d):
    heat = 3.0                                                      # some keys weigh much more than others
    check(randn(new, hq, d, dtype=dtype, seed=1) * heat, randn(keys, hk, d, dtype=dtype, seed=2), randn(keys, hk, d, dtype=dtype, seed=3))


@pytest.mark.parametrize("dtype", [FP, BF])
@pytest.mark.parametrize("gap", [10.0, 16.0, 20.0, 24.5, 25.25, 27.0])
@pytest.mark.parametrize("new,d", [(1, 128), (1, 64), (130, 128)])
def test_a_strong_first_key_over_a_long_weak_tail(dtype, gap, new, d):
    """One key `gap` powers of two above 32767 others alike: together they weigh up to 3 %, each less than fp16's smallest value
    of the first key's."""
    keys = 32768
    q, k = torch.zeros(new, 1, d, dtype=dtype, device=DEV), torch.zeros(keys, 1, d, dtype=dtype, device=DEV)
    q[..., 0], k[0, :, 0] = 1.0, gap
    for first, rest in ((0.0, 1.0), (1.0, 1.0), (1.0, -1.0)):
        v = torch.full((keys, 1, d), rest, dtype=dtype, device=DEV)
        v[0] = first
        check(q, k, v, group=0, scale=math.log(2.0))


@pytest.mark.parametrize("dtype", [FP, BF])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gap", [22.0, 24.5, 25.25, 27.0])
def test_a_weak_tail_that_one_thread_block_walks_over(dtype, d, gap):
    """Whole items, as long calls have them: no piece of the tail has a reference of its own."""
    new, keys = 148 * 256 + 60, 32768
    q, k = torch.zeros(new, 1, d, dtype=dtype, device=DEV), torch.zeros(keys, 1, d, dtype=dtype, device=DEV)
    q[..., 0], k[0, :, 0] = 1.0, gap
    v = torch.ones(keys, 1, d, dtype=dtype, device=DEV)
    v[0] = 0.0
    out, lse = B.regenvc_paged_attn_forward(*one_sequence(q, k, v), scale=math.log(2.0), lse=True)
    assert B.regenvc_device_status() == B.OK
    ref, ref_lse, bound, lse_bound = definition(q[:1], k, v, 0, math.log(2.0))     # all rows are alike
    assert ((out.double() - ref).abs() <= bound).all(), float(((out.double() - ref).abs() / bound).max())
    assert ((lse.double() - ref_lse).abs() <= lse_bound).all()


@pytest.mark.parametrize("dtype", [FP, BF])
@pytest.mark.parametrize("at", [0, 127, 128, 5000, 8191])
def test_a_strong_key_anywhere(dtype, at):
    keys, d = 8192, 128
    q, k = torch.zeros(2, 2, d, dtype=dtype, device=DEV), torch.zeros(keys, 1, d, dtype=dtype, device=DEV)
    q[..., 0] = 1.0
    for gap in (7.0, 9.0, 15.0, 17.0, 24.0, 33.0, 60.0):
        k[at, 0, 0] = gap
        check(q, k, randn(keys, 1, d, dtype=dtype, seed=4), group=0, scale=math.log(2.0))


@pytest.mark.parametrize("step", [0.5, 3.0, 7.0, 12.0, 20.0, 30.0])
@pytest.mark.parametrize("new,d", [(1, 128), (140, 128), (140, 64)])
def test_large_values_under_rising_scores(step, new, d):
    """bf16 values of 10^38: the result is a mean of them and finite, whatever the sums on the way there are."""
    keys = 2000
    q, k = torch.zeros(new, 1, d, dtype=BF, device=DEV), torch.zeros(keys, 1, d, dtype=BF, device=DEV)
    q[..., 0], k[:, 0, 0] = 1.0, (torch.arange(keys, device=DEV) // 200 * step).to(BF)
    v = (1 + randn(keys, 1, d, dtype=torch.float32, seed=5).abs().clamp(max=1.9)) * 1e38
    out, _ = check(q, k, v.to(BF), group=0, scale=math.log(2.0))
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("new,d", [(1, 128), (140, 128), (140, 64)])
def test_small_values(new, d):
    """bf16 values of 2^-80: their products with probabilities are in fp32's range."""
    keys = 2000
    v = (randn(keys, 1, d, dtype=torch.float32, seed=5) * 2.0 ** -80).to(BF)
    check(randn(new, 1, d, dtype=BF, seed=6) * 2, randn(keys, 1, d, dtype=BF, seed=7), v, group=0)


@pytest.mark.parametrize("new,keys,hq,hk,d", [([256], [40000], 1, 1, 128), ([129], [38000], 1, 1, 128), ([16], [80000], 1, 1, 64),
                                              ([200, 1], [25000, 19000], 2, 1, 64)])
def test_items_cut_over_every_thread_block(new, keys, hq, hk, d):
    """One item's pieces lie in all the blocks; every row of the join against the definition."""
    q = randn(sum(new), hq, d, dtype=BF, seed=6)
    k, v = (randn(sum(keys), hk, d, dtype=BF, seed=s) for s in (7, 8))
    page = 8
    need = [-(-m // page) for m in keys]
    caches = [torch.full((sum(need), page, hk, d), math.nan, dtype=BF, device=DEV) for _ in range(2)]
    table, at, row = torch.zeros((len(new), max(need)), dtype=torch.int32, device=DEV), 0, 0
    for s, (m, n) in enumerate(zip(keys, need)):
        table[s, :n] = torch.arange(at, at + n, device=DEV)
        for c, t in zip(caches, (k, v)):
            c[at:at + n].view(-1, hk, d)[:m] = t[row:row + m]
        at, row = at + n, row + m
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    out, lse = B.regenvc_paged_attn_forward(q, *caches, table, torch.tensor(keys, dtype=torch.int32, device=DEV),
                                            torch.tensor(starts, dtype=torch.int32, device=DEV), group=1, lse=True)
    assert B.regenvc_device_status() == B.OK
    row = 0
    for s, (m, n) in enumerate(zip(new, keys)):
        part = slice(starts[s], starts[s] + m)
        ref, ref_lse, bound, lse_bound = definition(q[part], k[row:row + n], v[row:row + n], 1, 1 / math.sqrt(d))
        assert ((out[part].double() - ref).abs() <= bound).all()
        assert ((lse[part].double() - ref_lse).abs() <= lse_bound).all()
        row += n
