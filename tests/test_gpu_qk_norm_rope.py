"""Queries and keys normalised per head and rotated, into rows and into a paged cache, and the gradients, against their 64-bit
forms."""
import pytest
import torch

from block_ops_util import U, floor_step, half_step
from cache_ops_util import head64, head_grads64, scatter_pages, slots_of
from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, FP, F32 = torch.bfloat16, torch.float16, torch.float32

CASES = [
    # tokens, hq, hk, d, type, widths, halves, whole ladder, float positions, gains
    (1, 12, 12, 128, BF, (44, 42, 42), False, False, False, True),
    (700, 12, 12, 128, BF, (44, 42, 42), False, False, False, True),
    (333, 8, 2, 128, FP, (32, 48, 48), True, True, True, True),
    (65, 5, 1, 64, F32, (24, 20, 20), True, False, False, True),
    (50, 3, 3, 256, BF, (256,), False, True, False, False),
    (40, 2, 4, 96, FP, (32, 32), True, False, True, True),
    (77, 7, 1, 80, BF, (20, 12), False, True, False, True),
    (31, 3, 0, 66, BF, (22, 22, 22), False, False, False, True),
    (29, 2, 2, 6, F32, (4,), True, False, False, True),
    (20, 2, 1, 250, FP, (100, 50), True, True, False, True),
    (90, 4, 4, 128, F32, (), False, False, False, True),
    (5000, 1, 1, 8, BF, (8,), True, True, False, True),
]


def operands(case, seed=0):
    n, hq, hk, d, dtype, widths, halves, whole, as_float, gains = case
    g = torch.Generator().manual_seed(seed)
    wide = 1 + 4 * torch.rand(d, generator=g) ** 4
    q, k = ((torch.randn(n, h, d, generator=g) * wide).to(dtype).to(DEV) if h else None for h in (hq, hk))
    pos = torch.randint(0, 5000, (len(widths), n), generator=g, dtype=torch.int32) if widths else None
    if pos is not None and as_float:
        pos = pos.float() * 0.125
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(DEV) if gains and h else None for h in (hq, hk)]
    how = dict(q_weight=w[0], k_weight=w[1], halves=halves, whole_ladder=whole)
    return q, k, None if pos is None else pos.to(DEV), list(widths) or None, how


def reference(x, w, pos, widths, how, eps=1e-6):
    return head64(x.double(), None if w is None else w.double(), pos, widths, 10000.0, how["halves"], how["whole_ladder"], eps)


def forward_bound(ref, mag, dtype, d):
    # sum of squares (d terms), rsqrt (2 steps), two products, cosine and sine of an angle rounded to a fraction of a turn
    # (its 32-bit fraction is off by up to pi 2^-24 of a turn's radians, cos and sin by two steps more), two products, a sum
    return half_step(dtype) * ref.abs() + (d / 2 + 24) * U * mag + floor_step(dtype)


@pytest.mark.parametrize("case", CASES)
def test_forward(case):
    q, k, pos, widths, how = operands(case)
    qo, ko = B.regenvc_qk_norm_rope_forward(q, k, pos, widths, **how)
    for x, y, w in ((q, qo, how["q_weight"]), (k, ko, how["k_weight"])):
        if x is None:
            assert y is None
            continue
        ref, mag = reference(x, w, pos, widths, how)
        assert ((y.double() - ref).abs() <= forward_bound(ref, mag, x.dtype, x.shape[2])).all()


@pytest.mark.parametrize("case", CASES)
def test_gradients_of_the_formula(case):
    q, k, pos, widths, how = operands(case)
    g = torch.Generator().manual_seed(9)
    dqo, dko = (None if x is None else torch.randn(x.shape, generator=g).to(x.dtype).to(DEV) for x in (q, k))
    got = B.regenvc_qk_norm_rope_backward(dqo, dko, q, k, pos, widths, **how)
    again = B.regenvc_qk_norm_rope_backward(dqo, dko, q, k, pos, widths, **how)
    for x, dy, name in ((q, dqo, "q"), (k, dko, "k")):
        if x is None:
            assert got["d" + name] is None
            continue
        w, d = how[name + "_weight"], x.shape[2]
        dx, mag, dw, dwm = head_grads64(x.double(), None if w is None else w.double(), dy.double(), pos, widths, 10000.0,
                                        how["halves"], how["whole_ladder"], 1e-6)
        err = (got["d" + name].double() - dx).abs()
        assert (err <= half_step(x.dtype) * dx.abs() + (2 * d + 48) * U * mag + floor_step(x.dtype)).all()
        assert torch.equal(got["d" + name], again["d" + name])
        if w is not None:
            # a thread adds up at most all tokens and heads; blocks and threads are joined in some dozen steps
            terms = x.shape[0] * x.shape[1]
            err = (got[f"d{name}_weight"].double() - dw).abs()
            assert (err <= (d + 64 + min(terms, 4096)) * U * dwm).all()
            assert torch.equal(got[f"d{name}_weight"], again[f"d{name}_weight"])


APPEND = [
    # new tokens, cached tokens with them, hq, hk, d, page, type, widths, halves, norm, order
    ([1], [1], 2, 2, 128, 16, BF, (44, 42, 42), False, True, "tokens"),
    ([1, 1, 0, 1], [17, 500, 33, 48], 8, 2, 128, 16, FP, (128,), True, True, "heads"),
    ([130, 7], [1000, 7], 12, 12, 128, 1560, BF, (44, 42, 42), False, True, "tokens"),
    ([64, 3, 20], [64, 900, 21], 0, 3, 64, 24, F32, (20, 20), True, True, "tokens"),
    ([9, 5], [9, 40], 3, 1, 66, 5, BF, (22, 22, 22), False, True, "heads"),
    ([40], [50], 2, 2, 80, 1, FP, (), False, False, "tokens"),
]


@pytest.mark.parametrize("new,keys,hq,hk,d,page,dtype,widths,halves,norm,order", APPEND)
def test_append(new, keys, hq, hk, d, page, dtype, widths, halves, norm, order):
    g = torch.Generator().manual_seed(page)
    table, pages = scatter_pages(keys, page, order, g)
    n = sum(new)
    rows = torch.randn(n + 4, hq + 2 * hk, d, generator=g).to(dtype).to(DEV)      # four rows behind the last sequence
    q, k, v = rows[:, :hq] if hq else None, rows[:, hq:hq + hk], rows[:, hq + hk:]
    shape = (pages, page, hk, d) if order == "tokens" else (pages, hk, page, d)
    kc, vc = (torch.randn(shape, generator=g).to(dtype).to(DEV) for _ in range(2))
    if order == "heads":
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    k_want, v_want = kc.double(), vc.double()
    k_bound = torch.zeros_like(k_want)
    pos = torch.randint(0, 9000, (len(widths), n + 4), generator=g, dtype=torch.int32).to(DEV) if widths else None
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(DEV) if norm else None for _ in range(2)]
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    q_out = torch.full((n + 4, hq, d), 7.0, dtype=dtype, device=DEV) if hq else None
    how = dict(halves=halves, whole_ladder=False)
    B.regenvc_paged_append(k, v, kc, vc, table.to(DEV), torch.tensor(keys, dtype=torch.int32, device=DEV),
                           torch.tensor(starts, dtype=torch.int32, device=DEV), q=q, positions=pos, widths=list(widths) or None,
                           norm=B.NORM_RMS if norm else B.NORM_NONE, q_weight=w[0] if hq else None, k_weight=w[1], q_out=q_out, **how)
    assert B.regenvc_device_status() == B.OK
    kr, km = head64(k.double(), None if w[1] is None else w[1].double(), pos, widths, 10000.0, halves, False, 1e-6, norm)
    for s, (m, total) in enumerate(zip(new, keys)):
        if not m:
            continue
        page_at, slot_at = slots_of(table, s, total, page)
        at = page_at[total - m:].to(DEV), slot_at[total - m:].to(DEV)
        part = slice(starts[s], starts[s] + m)
        k_want[at], v_want[at] = kr[part], v[part].double()
        k_bound[at] = forward_bound(kr[part], km[part], dtype, d)
    assert torch.equal(vc.double(), v_want)
    assert ((kc.double() - k_want).abs() <= k_bound).all()                        # other slots: as they were
    if hq:
        qr, qm = head64(q.double(), None if w[0] is None else w[0].double(), pos, widths, 10000.0, halves, False, 1e-6, norm)
        assert ((q_out.double() - qr).abs()[:n] <= forward_bound(qr, qm, dtype, d)[:n]).all()
        assert (q_out[n:] == 7.0).all()


def test_in_place_on_views_of_one_tensor():
    """q, k and v as a projection leaves them; forward, and the gradients over their own operands."""
    g = torch.Generator().manual_seed(3)
    for dtype, halves in ((BF, False), (F32, True)):
        rows = torch.randn(50, 6 + 2 + 2, 128, generator=g).to(dtype).to(DEV)
        pos = torch.arange(50, dtype=torch.int32, device=DEV).view(1, -1)
        w = (1 + 0.3 * torch.randn(128, generator=g)).to(DEV)
        how = dict(q_weight=w, k_weight=w, halves=halves)
        q, k = rows[:, :6], rows[:, 6:8]
        want = B.regenvc_qk_norm_rope_forward(q, k, pos, [128], **how)
        kept = rows.clone()
        grads = B.regenvc_qk_norm_rope_backward(want[0], want[1], q, k, pos, [128], **how)
        got = B.regenvc_qk_norm_rope_forward(q, k, pos, [128], q_out=q, k_out=k, **how)
        assert got[0].data_ptr() == rows.data_ptr()
        assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(rows[:, 8:], kept[:, 8:])
        again = B.regenvc_qk_norm_rope_backward(q, k, kept[:, :6], kept[:, 6:8], pos, [128], dq=q, dk=k, **how)
        assert torch.equal(q, grads["dq"]) and torch.equal(k, grads["dk"]) and torch.equal(rows[:, 8:], kept[:, 8:])
        assert torch.equal(again["dq_weight"], grads["dq_weight"]) and torch.equal(again["dk_weight"], grads["dk_weight"])


def test_values_are_copied_bit_by_bit_and_extremes_stay_in_their_row():
    v = torch.tensor([0x7FC1, 0x7F80, 0xFF80, 0x0001, 0x8000, 0x7F7F] + [0x3F80] * 122, dtype=torch.int32).to(torch.int16).view(BF)
    rows = torch.ones(3, 1, 128, dtype=BF, device=DEV)
    rows[1] = v.to(DEV)
    kc, vc = (torch.zeros(1, 8, 1, 128, dtype=BF, device=DEV) for _ in range(2))
    lists = (torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.tensor([5], dtype=torch.int32, device=DEV),
             torch.tensor([0, 3], dtype=torch.int32, device=DEV))
    B.regenvc_paged_append(rows, rows, kc, vc, *lists, norm=B.NORM_RMS)
    assert torch.equal(vc[0, 2:5].view(torch.int16), rows.view(torch.int16))
    assert (kc[0, 2] == 1).all() and (kc[0, 4] == 1).all() and (kc[0, :2] == 0).all()
    big = torch.full((2, 1, 128), 3e38, dtype=F32, device=DEV)
    big[1] = 0
    out, _ = B.regenvc_qk_norm_rope_forward(big, None)
    assert (out == 0).all()                                            # past fp32's range, and a row of zeros


def test_appending_to_places_that_do_not_exist_is_reported():
    rows = torch.ones(4, 1, 64, dtype=BF, device=DEV)
    starts = torch.tensor([0, 2, 4], dtype=torch.int32, device=DEV)
    for lengths, table in (([2, 2], [[0, 1], [-1, 1]]), ([2, 2], [[0, 1], [2, 1]]), ([2, 1], [[0, 0], [1, 0]]), ([2, 17], [[0, 0], [1, 1]])):
        kc, vc = (torch.zeros(2, 8, 1, 64, dtype=BF, device=DEV) for _ in range(2))
        B.regenvc_paged_append(rows, rows, kc, vc, torch.tensor(table, dtype=torch.int32, device=DEV),
                               torch.tensor(lengths, dtype=torch.int32, device=DEV), starts)
        assert B.regenvc_device_status() == B.ERR_RANGE
        assert (kc[0, :2] == 1).all() and (kc[0, 2:] == 0).all()       # the other sequence's tokens are there
    assert B.regenvc_device_status() == B.OK


def test_on_another_stream_and_in_a_graph():
    case = CASES[2]
    q, k, pos, widths, how = operands(case)
    want = B.regenvc_qk_norm_rope_forward(q, k, pos, widths, **how)
    grads = B.regenvc_qk_norm_rope_backward(*want, q, k, pos, widths, **how)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = B.regenvc_qk_norm_rope_forward(q, k, pos, widths, stream=s, **how)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q2 = q.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = B.regenvc_qk_norm_rope_forward(q2, k, pos, widths, **how)
        back = B.regenvc_qk_norm_rope_backward(*out, q2, k, pos, widths, **how)
    for scale in (1.0, 2.0):
        q2.copy_(scale * q)
        g.replay()
        torch.cuda.synchronize()
        ref = B.regenvc_qk_norm_rope_forward(q2, k, pos, widths, **how)
        rb = B.regenvc_qk_norm_rope_backward(*ref, q2, k, pos, widths, **how)
        assert torch.equal(out[0], ref[0]) and all(torch.equal(back[x], rb[x]) for x in rb)
    assert all(torch.equal(grads[x], B.regenvc_qk_norm_rope_backward(*want, q, k, pos, widths, **how)[x]) for x in grads)


def test_offsets_past_32_bits():
    pages = 140000                                                     # 2.3 10^9 elements
    kc, vc = (torch.empty((pages, 16, 8, 128), dtype=BF, device=DEV) for _ in range(2))
    rows = torch.randn(3, 8, 128, device=DEV).to(BF)
    table = torch.tensor([[pages - 1]], dtype=torch.int32, device=DEV)
    B.regenvc_paged_append(rows, rows, kc, vc, table, torch.tensor([16], dtype=torch.int32, device=DEV),
                           torch.tensor([0, 3], dtype=torch.int32, device=DEV))
    assert torch.equal(kc[-1, 13:], rows) and torch.equal(vc[-1, 13:], rows)


# blocks of 2, 4, 8 and 16 tokens, with a last one that is not full; heads that leave a part of the last round empty
MANY = [
    (2501, 2, 1, 128, BF, (44, 42, 42), False, False, False, True),
    (5003, 9, 4, 64, FP, (20, 12), True, True, False, True),
    (9999, 5, 2, 80, BF, (24, 20, 20), False, False, False, True),
    (19003, 3, 0, 32, F32, (16, 8), True, False, False, True),
    (30001, 1, 1, 16, BF, (16,), False, False, True, True),
]


@pytest.mark.parametrize("case", MANY)
def test_blocks_of_several_tokens(case):
    test_forward(case)
    test_gradients_of_the_formula(case)


def test_appending_blocks_of_several_tokens():
    new, keys, page, d = [4000, 1, 5501], [4100, 900, 5501], 24, 64
    g = torch.Generator().manual_seed(page)
    table, pages = scatter_pages(keys, page, "tokens", g)
    n = sum(new)
    q, k, v = (torch.randn(n, h, d, generator=g).to(BF).to(DEV) for h in (4, 1, 1))
    kc, vc = (torch.zeros(pages, page, 1, d, dtype=BF, device=DEV) for _ in range(2))
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    pos = torch.arange(n, dtype=torch.int32, device=DEV).view(1, -1)
    lists = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (keys, starts)]
    q_out = B.regenvc_paged_append(k, v, kc, vc, table.to(DEV), *lists, q=q, positions=pos, widths=[d], norm=B.NORM_RMS)
    qr, kr = B.regenvc_qk_norm_rope_forward(q, k, pos, [d])
    assert torch.equal(q_out, qr)
    for s, (m, total) in enumerate(zip(new, keys)):
        page_at, slot_at = slots_of(table, s, total, page)
        at = page_at[total - m:].to(DEV), slot_at[total - m:].to(DEV)
        part = slice(starts[s], starts[s] + m)
        assert torch.equal(kc[at], kr[part]) and torch.equal(vc[at], v[part])
    assert int((vc != 0).any(dim=3).sum()) <= n and B.regenvc_device_status() == B.OK


def test_vectors_more_than_two_gigabytes_apart():
    far = (1 << 30) + 64                                               # elements between the two heads: 2 GB and a little
    room = torch.empty(far + 64 * 3, dtype=BF, device=DEV)
    x = room.as_strided((3, 2, 64), (64, far, 1))
    x.copy_(torch.randn(3, 2, 64, generator=torch.Generator().manual_seed(1)).to(BF))
    near = x.contiguous()
    w = torch.ones(64, device=DEV)
    pos = torch.arange(3, dtype=torch.int32, device=DEV).view(1, -1)
    want, _ = B.regenvc_qk_norm_rope_forward(near, None, pos, [64], q_weight=w)
    ref, mag = reference(near, w, pos, (64,), dict(halves=False, whole_ladder=False))
    got, _ = B.regenvc_qk_norm_rope_forward(x, None, pos, [64], q_weight=w)
    for y in (want, got):
        assert ((y.double() - ref).abs() <= forward_bound(ref, mag, BF, 64)).all()
    back = B.regenvc_qk_norm_rope_backward(want, None, x, None, pos, [64], q_weight=w)
    dx, mag, dw, dwm = head_grads64(near.double(), w.double(), want.double(), pos, (64,), 10000.0, False, False, 1e-6)
    assert ((back["dq"].double() - dx).abs() <= half_step(BF) * dx.abs() + 176 * U * mag + floor_step(BF)).all()
    assert ((back["dq_weight"].double() - dw).abs() <= 134 * U * dwm).all()
