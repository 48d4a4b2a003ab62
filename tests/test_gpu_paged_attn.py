"""Attention over a paged cache against its 64-bit form: ragged batches, shared heads, masks by groups and windows, pages that
end inside a tile, orders and strides, what lies in unseen slots, splits over the key axis."""
import math

import pytest
import torch

from cache_ops_util import attend64, scatter_pages, sees, slots_of
from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, FP = torch.bfloat16, torch.float16


def make(new, keys, hq, hk, d, page, dtype, order="tokens", seed=0, heat=1.0, junk=math.nan, pad=0):
    """Caches whose unused slots hold `junk`, and the call's arguments."""
    g = torch.Generator().manual_seed(seed)
    table, pages = scatter_pages(keys, page, order, g)
    shape = (pages, page, hk, d) if order == "tokens" else (pages, hk, page, d)
    kc, vc = torch.full(shape, junk, dtype=dtype), torch.full(shape, junk, dtype=dtype)
    if order == "heads":
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    k64, v64 = [], []
    for s, m in enumerate(keys):
        k, v = torch.randn(m, hk, d, generator=g).to(dtype), torch.randn(m, hk, d, generator=g).to(dtype)
        if m:
            at = slots_of(table, s, m, page)
            kc[at], vc[at] = k, v
        k64.append(k.double())
        v64.append(v.double())
    n = sum(new) + pad
    q = (heat * torch.randn(n, hq, d, generator=g)).to(dtype)
    starts = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32)
    kd = torch.empty(shape, dtype=dtype, device=DEV) if order == "tokens" else torch.empty(shape, dtype=dtype, device=DEV).transpose(1, 2)
    vd = torch.empty_like(kd) if order == "tokens" else torch.empty(shape, dtype=dtype, device=DEV).transpose(1, 2)
    kd.copy_(kc)
    vd.copy_(vc)
    return {"q": q, "k64": k64, "v64": v64, "args": (q.to(DEV), kd, vd, table.to(DEV), torch.tensor(keys, dtype=torch.int32).to(DEV),
                                                    starts.to(DEV)), "table": table}


def check(c, new, keys, out, lse, group, window, scale=None):
    at = 0
    d, dtype = c["q"].shape[2], c["q"].dtype
    for s, (m, n) in enumerate(zip(new, keys)):
        if m:
            see = sees(m, n, group, window)
            ref, ref_lse, bound, lse_bound = attend64(c["q"][at:at + m].double().to(DEV), c["k64"][s].to(DEV), c["v64"][s].to(DEV), see,
                                                      scale or 1 / math.sqrt(d), dtype)
            err = (out[at:at + m].double() - ref).abs()
            assert (err <= bound).all(), (s, m, n, float((err - bound).max()), float(err.max()))
            if lse is not None:
                got = lse[at:at + m].double()
                none = torch.isinf(ref_lse)
                assert torch.equal(none, torch.isinf(got)) and (got[none] < 0).all()
                assert ((got - ref_lse).abs()[~none] <= lse_bound[~none]).all()
        at += m


CASES = [
    # new tokens, cached tokens with them, hq, hk, d, page, type, group, window, order
    ([1], [1], 1, 1, 128, 16, BF, 0, 0, "tokens"),
    ([1], [301], 12, 12, 128, 64, BF, 0, 0, "tokens"),
    ([1, 1, 1], [1, 128, 129], 8, 2, 128, 16, BF, 1, 0, "tokens"),
    ([1] * 7, [17, 500, 1, 2049, 64, 63, 4100], 40, 8, 128, 32, FP, 1, 0, "heads"),
    ([5], [5], 3, 1, 64, 8, BF, 1, 0, "tokens"),
    ([128], [128], 1, 1, 128, 128, FP, 1, 0, "tokens"),
    ([129], [1000], 1, 1, 128, 48, BF, 1, 0, "tokens"),
    ([256], [300], 2, 2, 128, 256, BF, 0, 0, "heads"),
    ([257, 3, 0, 40], [257, 777, 90, 41], 6, 2, 64, 24, FP, 1, 0, "tokens"),
    ([700], [1500], 4, 4, 128, 1560, BF, 156, 0, "tokens"),
    ([700, 13], [1500, 3200], 4, 2, 128, 200, BF, 100, 5, "heads"),
    ([300], [2300], 5, 5, 64, 40, BF, 1, 130, "tokens"),
    ([1, 1], [9000, 400], 7, 1, 128, 64, BF, 1, 1000, "tokens"),
    ([33, 2, 190], [40, 2000, 1111], 24, 8, 64, 48, FP, 1, 0, "heads"),
    ([2000], [2000], 3, 3, 128, 104, BF, 1, 0, "tokens"),
]


@pytest.mark.parametrize("new,keys,hq,hk,d,page,dtype,group,window,order", CASES)
def test_against_the_64_bit_form(new, keys, hq, hk, d, page, dtype, group, window, order):
    c = make(new, keys, hq, hk, d, page, dtype, order, seed=len(new) + page)
    out, lse = B.regenvc_paged_attn_forward(*c["args"], group=group, window=window, lse=True)
    assert B.regenvc_device_status() == B.OK
    check(c, new, keys, out, lse, group, window)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("new,group", [(1, 0), (200, 0), (300, 1), (129, 40)])
def test_scores_that_rise_along_the_keys(dtype, new, group):
    """Every 40 keys the scores rise by some 20 nats: references are raised in either half of a tile, again and again."""
    keys, d = 900, 128
    c = make([new], [keys], 2, 1, d, 64, dtype, seed=3)
    k = c["k64"][0]
    k += (torch.arange(keys) // 40).double()[:, None, None] * 20 / math.sqrt(d)    # q . (1, .., 1) is about d here, below
    k = k.to(dtype).double()
    q = (1 + 0.2 * c["q"].double()).to(dtype)
    c["q"], c["k64"] = q, [k]
    args = list(c["args"])
    args[0] = q.to(DEV)
    at = slots_of(c["table"], 0, keys, 64)
    args[1][at[0].to(DEV), at[1].to(DEV)] = k.to(dtype).to(DEV)
    out, lse = B.regenvc_paged_attn_forward(*args, group=group, lse=True)
    assert B.regenvc_device_status() == B.OK
    check(c, [new], [keys], out, lse, group, 0)
