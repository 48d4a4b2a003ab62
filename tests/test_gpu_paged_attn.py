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


@pytest.mark.parametrize("group,window,page", [(1, 0, 16), (0, 0, 16), (3, 1, 16), (1, 0, 1560), (0, 0, 256)])
def test_rows_that_see_nothing(group, window, page):
    """Sequences with fewer cached tokens than rows, none at all, and none of either."""
    new, keys = [5, 4, 0, 200, 2], [3, 0, 0, 150, 9]
    c = make(new, keys, 4, 2, 128, page, BF, seed=5)
    out, lse = B.regenvc_paged_attn_forward(*c["args"], group=group, window=window, lse=True)
    assert B.regenvc_device_status() == B.OK
    check(c, new, keys, out, lse, group, window)
    assert (out[5:9] == 0).all() and torch.isinf(lse[5:9]).all()
    if group:
        assert (out[:2] == 0).all() and torch.isinf(lse[:2]).all()


def test_strided_operands_padded_rows_and_a_scale():
    new, keys = [3, 130], [40, 300]
    c = make(new, keys, 6, 3, 64, 16, FP, seed=6, pad=7)
    q, kc, vc, table, lengths, starts = c["args"]
    rows = torch.randn(140, 12, 64, device=DEV).to(FP)                # a projection's rows: q, k, v side by side
    rows[:, :6] = q
    both = torch.full((kc.shape[0], 2, *kc.shape[1:]), math.nan, dtype=FP, device=DEV)   # keys and values in one tensor
    both[:, 0], both[:, 1] = kc, vc
    wide = torch.zeros((2, table.shape[1] + 3), dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    out = torch.full((140, 6, 80), 7.0, dtype=FP, device=DEV)
    lse = torch.full((140, 6), 7.0, device=DEV)
    B.regenvc_paged_attn_forward(rows[:, :6], both[:, 0], both[:, 1], wide[:, :table.shape[1]], lengths, starts, group=1, scale=0.21,
                                 out=out[..., :64], lse=lse)
    assert B.regenvc_device_status() == B.OK
    check(c, new, keys, out[..., :64], lse, 1, 0, 0.21)
    assert (out[133:] == 7).all() and (out[..., 64:] == 7).all() and (lse[133:] == 7).all()


def test_pages_before_the_window_need_not_exist():
    new, keys, page = [70, 1], [1000, 513], 32
    c = make(new, keys, 2, 1, 128, page, BF, seed=7)
    args = list(c["args"])
    group, window = 10, 7
    table = args[3].clone()
    for s, (m, n) in enumerate(zip(new, keys)):
        first = max(0, ((n - m) // group - window + 1) * group)       # the first token that any of them sees
        table[s, :first // page] = -1
        for t in range(first // page):
            args[1][c["table"][s, t]] = math.inf
            args[2][c["table"][s, t]] = math.nan
        args[1][c["table"][s, first // page], :first % page] = math.nan
        args[2][c["table"][s, first // page], :first % page] = math.inf
    args[3] = table
    out, lse = B.regenvc_paged_attn_forward(*args, group=group, window=window, lse=True)
    assert B.regenvc_device_status() == B.OK
    check(c, new, keys, out, lse, group, window)


@pytest.mark.parametrize("new,keys,hq,hk,d,group,window", [
    ([3000], [5000], 16, 16, 128, 500, 4),                            # whole items in rounds, then the rest of the line
    ([2600, 1, 700], [2600, 4000, 9000], 24, 12, 64, 1, 0),
    ([1] * 40, [700] * 40, 8, 8, 128, 0, 0),                          # more sequences than a warp has lanes
    ([1] * 3 + [260], [20000, 1, 64, 20000], 2, 1, 128, 1, 0)])       # items cut into many pieces
def test_splits_of_the_work(new, keys, hq, hk, d, group, window):
    c = make(new, keys, hq, hk, d, 64, BF, seed=8)
    out, lse = B.regenvc_paged_attn_forward(*c["args"], group=group, window=window, lse=True)
    again, lse2 = B.regenvc_paged_attn_forward(*c["args"], group=group, window=window, lse=True)
    assert B.regenvc_device_status() == B.OK
    check(c, new, keys, out, lse, group, window)
    assert torch.equal(out, again) and torch.equal(lse, lse2)         # the same split, the same sums


def test_a_thousand_sequences():
    g = torch.Generator().manual_seed(9)
    keys = torch.randint(1, 60, (1000,), generator=g).tolist()
    new = torch.randint(0, 3, (1000,), generator=g).tolist()
    keys = [max(k, n) for k, n in zip(keys, new)]
    c = make(new, keys, 2, 2, 64, 16, FP, seed=9)
    out, lse = B.regenvc_paged_attn_forward(*c["args"], group=1, lse=True)
    assert B.regenvc_device_status() == B.OK
    check(c, new, keys, out, lse, 1, 0)


def test_offsets_past_32_bits():
    """Caches of 2.3 10^9 elements each; the sequence lies at their end."""
    c = make([2], [130], 8, 8, 128, 16, BF, seed=10)
    q, kc, vc, table, lengths, starts = c["args"]
    pages = 140000
    big_k, big_v = (torch.empty((pages, 16, 8, 128), dtype=BF, device=DEV) for _ in range(2))
    shift = pages - kc.shape[0]
    big_k[shift:], big_v[shift:] = kc, vc
    out, lse = B.regenvc_paged_attn_forward(q, big_k, big_v, torch.where(table < 10 ** 6, table + shift, table), lengths, starts,
                                            group=1, lse=True)
    assert B.regenvc_device_status() == B.OK
    check(c, [2], [130], out, lse, 1, 0)


def test_contradictions_are_reported_and_nothing_else_is_read():
    c = make([1, 1], [40, 50], 2, 2, 128, 16, BF, seed=11)
    args = list(c["args"])
    bad = args[3].clone()
    bad[1, 1] = -5
    B.regenvc_paged_attn_forward(*args[:3], bad, *args[4:], group=1)
    assert B.regenvc_device_status() == B.ERR_RANGE
    bad[1, 1] = 10 ** 6
    B.regenvc_paged_attn_forward(*args[:3], bad, *args[4:], group=1)
    assert B.regenvc_device_status() == B.ERR_RANGE
    for lengths, starts in (([40, 10 ** 9], [0, 1, 2]), ([-1, 50], [0, 1, 2]), ([40, 50], [0, 2, 1]), ([40, 50], [0, 1, 900]),
                            ([40, 50], [-3, 1, 2])):
        B.regenvc_paged_attn_forward(*args[:4], torch.tensor(lengths, dtype=torch.int32, device=DEV),
                                     torch.tensor(starts, dtype=torch.int32, device=DEV), group=1)
        assert B.regenvc_device_status() == B.ERR_RANGE
    out, lse = B.regenvc_paged_attn_forward(*args, group=1, lse=True)     # and the next call is normal again
    assert B.regenvc_device_status() == B.OK
    check(c, [1, 1], [40, 50], out, lse, 1, 0)


def test_two_streams_at_once_and_a_graph_that_follows_the_lengths():
    new, keys = [1, 40, 3], [200, 600, 77]
    c = make(new, keys, 4, 2, 128, 16, BF, seed=12)
    args = list(c["args"])
    want, _ = B.regenvc_paged_attn_forward(*args, group=1)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                outs[i].append(B.regenvc_paged_attn_forward(*args, group=1)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for part in outs for o in part)
    assert B.regenvc_device_status() == B.OK
    size = B.regenvc_paged_attn_workspace_bytes(4, 2, 128)
    graphs, results = [], []
    for _ in range(2):                                                # a workspace each: they may be replayed at a time
        ws, out = torch.empty(size, dtype=torch.uint8, device=DEV), torch.zeros_like(args[0])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.regenvc_paged_attn_forward(*args, group=1, out=out, workspace=ws)
        graphs.append((g, ws))
        results.append(out)
    for lengths in (keys, [150, 555, 3], [1, 40, 50]):
        args[4].copy_(torch.tensor(lengths, dtype=torch.int32))
        torch.cuda.synchronize()
        for (g, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        want, _ = B.regenvc_paged_attn_forward(*args, group=1)
        assert torch.equal(results[0], want) and torch.equal(results[1], want)
    assert B.regenvc_device_status() == B.OK


def test_nothing_runs_while_a_status_is_set_and_all_does_afterwards():
    c = make([1], [40], 2, 2, 64, 16, FP, seed=13)
    B.regenvc_debug_expire_wait(200)
    B.regenvc_paged_attn_forward(*c["args"])                          # its waits fall through
    assert B.regenvc_device_status() == B.ERR_TIMEOUT
    out, lse = B.regenvc_paged_attn_forward(*c["args"], lse=True)
    assert B.regenvc_device_status() == B.OK
    check(c, [1], [40], out, lse, 0, 0)


@pytest.mark.parametrize("new,keys,group,d", [([300], [700], 1, 128), ([1, 1, 20], [9000, 40, 300], 1, 128), ([140, 3], [400, 90], 0, 64)])
def test_what_is_not_a_number_stays_in_the_rows_that_see_it(new, keys, group, d):
    hq, hk, page = 4, 2, 16
    c = make(new, keys, hq, hk, d, page, BF, seed=5)
    q, kc = c["args"][0], c["args"][1]
    for row, head in ((0, 1), (new[0] - 1, 3), (sum(new) - 1, 0)):
        c["q"][row, head] = math.nan
    q.copy_(c["q"])
    key = keys[-1] - 2                                       # of the last sequence, in one head of the cache
    page_at, slot_at = slots_of(c["table"], len(keys) - 1, keys[-1], page)
    kc[int(page_at[key]), int(slot_at[key]), 1, 3] = math.nan
    c["k64"][-1][key, 1, 3] = math.nan
    out, lse = B.regenvc_paged_attn_forward(*c["args"], group=group, lse=True)
    assert B.regenvc_device_status() == B.OK
    at = 0
    for s, (m, n) in enumerate(zip(new, keys)):
        ref, ref_lse, bound, lse_bound = attend64(c["q"][at:at + m].double().to(DEV), c["k64"][s].to(DEV), c["v64"][s].to(DEV),
                                                  sees(m, n, group, 0), 1 / math.sqrt(d), BF)
        got, got_lse = out[at:at + m].double(), lse[at:at + m].double()
        assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(torch.isnan(got_lse), torch.isnan(ref_lse))
        fine = ~torch.isnan(ref_lse)
        assert fine.any() or m == 1
        assert ((got - ref).abs() <= bound)[fine].all() and ((got_lse - ref_lse).abs() <= lse_bound)[fine].all()
        at += m


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq,hk", [(1, 1), (4, 1), (8, 2)])
def test_items_of_about_sixteen_rows(dtype, hq, hk):
    """Products of 64 and of 128 rows in turn in a thread block; a first call leaves NaN in lanes that are nobody's."""
    new, keys = [16, 17, 4, 5, 1, 40], [700, 300, 2000, 129, 5000, 41]
    hot = make([256], [256], hq, hk, 128, 16, dtype, seed=7)
    hot["args"][0].fill_(math.nan)
    B.regenvc_paged_attn_forward(*hot["args"], group=0)
    for heat, group in ((1.0, 1), (40.0, 0)):
        c = make(new, keys, hq, hk, 128, 16, dtype, seed=11, heat=heat)
        out, lse = B.regenvc_paged_attn_forward(*c["args"], group=group, lse=True)
        assert B.regenvc_device_status() == B.OK
        check(c, new, keys, out, lse, group, 0)
