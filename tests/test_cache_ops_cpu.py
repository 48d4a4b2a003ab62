"""Host-side tests of the operators of attention over cached windows: sizes, every refusal before any CUDA call, the binding's
checks, and the 64-bit forms that the GPU tests compare with."""
import ctypes
import math

import pytest
import torch

from cache_ops_util import attend64, head64, head_grads64, sees
from paper_2607_28144_b200 import binding as B
from paper_2607_28144_b200 import build


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


A = [0x100000000 * (i + 1) for i in range(24)]   # far apart, never dereferenced: every call below must fail first


def _desc(kind, base, kw):
    d = dict(base)
    d.update(kw)
    if "widths" in d:
        d["widths"] = (ctypes.c_int * 4)(*d["widths"])
    return kind(**d)


def _norm(**kw):
    return _desc(B.QkNormRopeDesc, dict(n_tokens=5, n_q_heads=4, n_k_heads=2, head_dim=64, type=0, n_axes=3, widths=(20, 22, 22),
                                        rope_theta=1e4, eps=1e-6), kw)


def _forward(L, d, q=A[0], k=A[1], qw=A[2], kw=A[3], pos=A[4], qo=A[5], ko=A[6]):
    return L.regenvc_qk_norm_rope_forward(ctypes.byref(d) if d is not None else None, q, k, qw, kw, pos, qo, ko, None)


ROTATION_SHAPES = (dict(n_tokens=0), dict(n_tokens=(1 << 30) + 1), dict(n_q_heads=-1), dict(n_k_heads=65536), dict(head_dim=0),
                   dict(head_dim=258), dict(n_axes=5), dict(n_axes=-1), dict(widths=(20, 22, 24)), dict(widths=(20, 21, 22)),
                   dict(widths=(0, 22, 22)), dict(pos_stride=4))
ROTATION_KINDS = (dict(head_dim=63, widths=(20, 20, 20)), dict(type=3), dict(rope_theta=0.0), dict(rope_theta=float("nan")),
                  dict(halves=2), dict(whole_ladder=-1), dict(eps=-1.0), dict(eps=float("inf")))


def test_qk_norm_rope_refusals(L):
    d = _norm()
    assert _forward(L, None) == B.ERR_NULL_POINTER
    for bad in (dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(pos=None)):
        assert _forward(L, d, **bad) == B.ERR_NULL_POINTER, bad
    assert _forward(L, _norm(n_k_heads=0)) == B.ERR_NULL_POINTER                      # k without heads
    assert _forward(L, _norm(n_axes=0)) == B.ERR_NULL_POINTER                         # positions without axes
    assert _forward(L, _norm(n_q_heads=0), q=None, qo=None) == B.ERR_NULL_POINTER     # gains without q
    assert _forward(L, _norm(n_q_heads=0, n_k_heads=0), q=None, k=None, qo=None, ko=None, qw=None, kw=None) == B.ERR_NULL_POINTER
    for bad in ROTATION_SHAPES + (dict(q_head_stride=63), dict(q_token_stride=32), dict(k_out_token_stride=-1),
                                  dict(q_head_stride=100, q_token_stride=256)):
        assert _forward(L, _norm(**bad)) == B.ERR_BAD_SHAPE, bad
    for bad in ROTATION_KINDS:
        assert _forward(L, _norm(**bad)) == B.ERR_UNSUPPORTED, bad
    assert _forward(L, d, q=A[0] + 1) == B.ERR_MISALIGNED
    assert _forward(L, d, qw=A[2] + 2) == B.ERR_MISALIGNED
    assert _forward(L, d, pos=A[4] + 2) == B.ERR_MISALIGNED
    assert _forward(L, d, qo=A[0] + 16) == B.ERR_ALIASING
    assert _forward(L, _norm(q_out_token_stride=512), qo=A[0]) == B.ERR_ALIASING      # q's address, other strides
    assert _forward(L, d, qo=A[1]) == B.ERR_ALIASING
    assert _forward(L, d, ko=A[5]) == B.ERR_ALIASING
    assert _forward(L, d, qo=A[4]) == B.ERR_ALIASING
    assert _forward(L, d, ko=A[3]) == B.ERR_ALIASING
    fused = dict(q_token_stride=8 * 64, k_token_stride=8 * 64, q_out_token_stride=8 * 64, k_out_token_stride=8 * 64)
    near = A[0] + 2 * (4 * 64 - 8)                                                    # k eight elements into q's last head
    assert _forward(L, _norm(**fused), qo=A[0], k=near, ko=near) == B.ERR_ALIASING
    over = A[0] + 2 * 7 * 64                                                          # k runs into the next token's q
    assert _forward(L, _norm(**fused), qo=A[0], k=over, ko=over) == B.ERR_ALIASING


def _backward(L, d, dqo=A[0], dko=A[1], q=A[2], k=A[3], qw=A[4], kw=A[5], pos=A[6], dq=A[7], dk=A[8], dqw=A[9], dkw=A[10],
              ws=A[11], size=1 << 24):
    return L.regenvc_qk_norm_rope_backward(ctypes.byref(d), dqo, dko, q, k, qw, kw, pos, dq, dk, dqw, dkw, ws, size, None)


def test_qk_norm_rope_backward_refusals(L):
    d = _norm()
    need = B.regenvc_qk_norm_rope_workspace_bytes(64)
    assert need == 1184 * 2 * 64 * 4
    assert B.regenvc_qk_norm_rope_workspace_bytes(63) == B.regenvc_qk_norm_rope_workspace_bytes(258) == 0
    assert _backward(L, d, size=need - 1) == B.ERR_WORKSPACE
    assert _backward(L, d, ws=A[11] + 8) == B.ERR_WORKSPACE
    for bad in (dict(dqo=None), dict(dko=None), dict(q=None), dict(k=None), dict(dq=None), dict(dk=None), dict(qw=None), dict(kw=None),
                dict(ws=None), dict(pos=None)):
        assert _backward(L, d, **bad) == B.ERR_NULL_POINTER, bad
    for bad in ROTATION_SHAPES + (dict(dq_token_stride=32), dict(k_out_head_stride=1)):
        assert _backward(L, _norm(**bad)) == B.ERR_BAD_SHAPE, bad
    for bad in ROTATION_KINDS:
        assert _backward(L, _norm(**bad)) == B.ERR_UNSUPPORTED, bad
    for bad in (dict(dq=A[2]), dict(dq=A[0] + 32), dict(dk=A[7]), dict(dqw=A[0]), dict(dqw=A[4]), dict(dkw=A[9]), dict(ws=A[2]),
                dict(ws=A[7]), dict(dk=A[11]), dict(dq=A[6])):
        assert _backward(L, d, **bad) == B.ERR_ALIASING, bad


def _append_desc(**kw):
    return _desc(B.PagedAppendDesc, dict(n_tokens=5, n_q_heads=4, n_k_heads=2, head_dim=64, type=0, n_axes=3, widths=(20, 22, 22),
                                         rope_theta=1e4, eps=1e-6, norm=2, n_sequences=3, page_size=16, n_pages=10,
                                         pages_per_sequence=4), kw)


def _append(L, d, q=A[0], k=A[1], v=A[2], qw=A[3], kw=A[4], pos=A[5], starts=A[6], lengths=A[7], table=A[8], qo=A[9], kc=A[10], vc=A[11]):
    return L.regenvc_paged_append(ctypes.byref(d) if d is not None else None, q, k, v, qw, kw, pos, starts, lengths, table, qo, kc, vc, None)


LISTS = (dict(n_sequences=0), dict(n_sequences=4097), dict(page_size=0), dict(page_size=(1 << 20) + 8), dict(n_pages=0),
         dict(pages_per_sequence=0), dict(table_stride=3))


def test_paged_append_refusals(L):
    d = _append_desc()
    assert _append(L, None) == B.ERR_NULL_POINTER
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(pos=None), dict(starts=None), dict(lengths=None), dict(table=None),
                dict(qo=None), dict(kc=None), dict(vc=None)):
        assert _append(L, d, **bad) == B.ERR_NULL_POINTER, bad
    assert _append(L, _append_desc(norm=0)) == B.ERR_NULL_POINTER                     # gains without a norm
    assert _append(L, _append_desc(n_q_heads=0), q=None, qo=None) == B.ERR_NULL_POINTER
    assert _append(L, _append_desc(norm=1)) == B.ERR_UNSUPPORTED
    for bad in ROTATION_SHAPES + LISTS + (dict(n_k_heads=0), dict(k_slot_stride=63), dict(v_page_stride=64),
                                          dict(k_cache_head_stride=32), dict(v_token_stride=1)):
        assert _append(L, _append_desc(**bad)) == B.ERR_BAD_SHAPE, bad
    for bad in ROTATION_KINDS:
        assert _append(L, _append_desc(**bad)) == B.ERR_UNSUPPORTED, bad
    assert _append(L, d, kc=A[10] + 1) == B.ERR_MISALIGNED
    assert _append(L, d, starts=A[6] + 2) == B.ERR_MISALIGNED
    assert _append(L, d, table=A[8] + 1) == B.ERR_MISALIGNED
    for bad in (dict(kc=A[1]), dict(vc=A[2]), dict(kc=A[0]), dict(vc=A[10]), dict(kc=A[9]), dict(kc=A[8]), dict(vc=A[7]), dict(qo=A[1]),
                dict(qo=A[6]), dict(kc=A[5])):
        assert _append(L, d, **bad) == B.ERR_ALIASING, bad
    # one tensor with a page's values behind its keys is two caches; eight elements nearer they share memory
    page = 16 * 2 * 64
    halves = dict(k_page_stride=2 * page, v_page_stride=2 * page)
    assert _append(L, _append_desc(**halves), vc=A[10] + 2 * (page - 8)) == B.ERR_ALIASING


def _attn_desc(**kw):
    return _desc(B.PagedAttnDesc, dict(n_tokens=5, n_q_heads=4, n_k_heads=2, head_dim=64, type=0, n_sequences=3, page_size=16,
                                       n_pages=10, pages_per_sequence=4), kw)


def _attn(L, d, q=A[0], kc=A[1], vc=A[2], starts=A[3], lengths=A[4], table=A[5], out=A[6], lse=A[7], ws=A[8], size=1 << 30):
    return L.regenvc_paged_attn_forward(ctypes.byref(d) if d is not None else None, q, kc, vc, starts, lengths, table, out, lse, ws, size, None)


def test_paged_attn_refusals(L):
    d = _attn_desc()
    need = B.regenvc_paged_attn_workspace_bytes(4, 2, 64)
    assert need == 160 * 2 * (256 * (64 * 4 + 8) + 24)
    for bad in ((4, 3, 64), (4, 2, 96), (0, 2, 64), (4, 0, 128)):
        assert B.regenvc_paged_attn_workspace_bytes(*bad) == 0
    assert _attn(L, None) == B.ERR_NULL_POINTER
    for bad in (dict(q=None), dict(kc=None), dict(vc=None), dict(starts=None), dict(lengths=None), dict(table=None), dict(out=None),
                dict(ws=None)):
        assert _attn(L, d, **bad) == B.ERR_NULL_POINTER, bad
    for bad in LISTS + (dict(n_tokens=0), dict(n_q_heads=3), dict(n_k_heads=0), dict(group=-1), dict(window=-1), dict(window=2),
                        dict(n_tokens=1 << 30, n_q_heads=2), dict(q_head_stride=8), dict(out_token_stride=32), dict(k_slot_stride=64),
                        dict(v_page_stride=8)):
        assert _attn(L, _attn_desc(**bad)) == B.ERR_BAD_SHAPE, bad
    for bad in (dict(type=2), dict(type=-1), dict(head_dim=96), dict(head_dim=256), dict(page_size=12), dict(scale=-1.0),
                dict(scale=float("nan")), dict(scale=float("inf"))):
        assert _attn(L, _attn_desc(**bad)) == B.ERR_UNSUPPORTED, bad
    for bad in (dict(q=A[0] + 8), dict(kc=A[1] + 2), dict(out=A[6] + 8), dict(lse=A[7] + 2), dict(lengths=A[4] + 2)):
        assert _attn(L, d, **bad) == B.ERR_MISALIGNED, bad
    assert _attn(L, _attn_desc(q_token_stride=260)) == B.ERR_MISALIGNED
    assert _attn(L, _attn_desc(k_page_stride=16 * 128 + 4)) == B.ERR_MISALIGNED
    assert _attn(L, d, size=need - 1) == B.ERR_WORKSPACE
    assert _attn(L, d, ws=A[8] + 8) == B.ERR_WORKSPACE
    for bad in (dict(out=A[0]), dict(out=A[1] + 64), dict(out=A[2]), dict(lse=A[5]), dict(lse=A[6]), dict(ws=A[1]), dict(ws=A[6]),
                dict(out=A[4]), dict(ws=A[7])):
        assert _attn(L, d, **bad) == B.ERR_ALIASING, bad


def test_the_binding_refuses_what_the_library_cannot_see():
    q = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    cache = torch.zeros((4, 16, 2, 64), dtype=torch.bfloat16)
    table, lengths, starts = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        B.regenvc_qk_norm_rope_forward(q, None)                       # not on a GPU
    with pytest.raises(TypeError):
        B.regenvc_qk_norm_rope_forward(None, None)
    with pytest.raises(TypeError):
        B.regenvc_qk_norm_rope_forward(q, q.float())
    with pytest.raises(ValueError):
        B._rotation(None, [64], 3)
    with pytest.raises(TypeError):
        B._rotation(torch.zeros((2, 4)), [32, 32], 3)
    with pytest.raises(TypeError):
        B.regenvc_paged_attn_forward(q, cache, cache, table.long(), lengths, starts)
    with pytest.raises(TypeError):
        B.regenvc_paged_attn_forward(q, cache, cache, table, lengths, starts[:1])
    with pytest.raises(TypeError):
        B.regenvc_paged_attn_forward(q, cache, cache.half(), table, lengths, starts)
    with pytest.raises(TypeError):
        B.regenvc_paged_attn_forward(q, cache[..., :32], cache[..., :32], table, lengths, starts)
    with pytest.raises(ValueError):
        B._cache(cache[:, :1].expand(4, 16, 2, 64), "k_cache", torch.bfloat16)
    with pytest.raises(ValueError):
        B._head_strides(q[:, :1].expand(3, 2, 64), "q", torch.bfloat16, 3, 2, 64)
    # strides of axes with one entry are never used
    assert B._cache(cache.transpose(1, 2).contiguous().transpose(1, 2), "k_cache", torch.bfloat16) == (2048, 64, 1024)
    page, slot, head = B._cache(cache[:1, :, 1:], "k_cache", torch.bfloat16)
    assert slot == 128 and page >= 2048 and head >= 64 and page % 8 == head % 8 == 0


def test_the_64_bit_gradients_are_those_of_the_64_bit_norm():
    g = torch.Generator().manual_seed(0)
    for halves, widths, gains in ((False, (4, 6), True), (True, (8,), True), (True, (), False)):
        x = torch.randn(3, 2, 12, generator=g, dtype=torch.float64)
        w = 1 + 0.3 * torch.randn(12, generator=g, dtype=torch.float64) if gains else None
        dy = torch.randn(3, 2, 12, generator=g, dtype=torch.float64)
        pos = torch.randint(0, 50, (len(widths), 3), generator=g)

        def loss(x, w):
            return (head64(x, w, pos, widths, 100.0, halves, False, 1e-3)[0] * dy).sum()

        dx, _, dw, _ = head_grads64(x, w, dy, pos, widths, 100.0, halves, False, 1e-3)
        step = 1e-5                                                   # errors: step^2 of the third derivative, 2^-53 / step
        for i in range(0, x.numel(), 5):
            e = torch.zeros_like(x).view(-1)
            e[i] = step
            e = e.view_as(x)
            assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * step) - dx.view(-1)[i]) < 1e-7
        for i in range(12 if gains else 0):
            e = torch.zeros(12, dtype=torch.float64)
            e[i] = step
            assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * step) - dw[i]) < 1e-7


def test_the_64_bit_attention_by_loops():
    g = torch.Generator().manual_seed(1)
    for new, keys, group, window in ((3, 7, 1, 0), (4, 9, 2, 2), (2, 2, 0, 0), (5, 3, 1, 0)):
        q = torch.randn(new, 4, 8, generator=g, dtype=torch.float64)
        k, v = (torch.randn(keys, 2, 8, generator=g, dtype=torch.float64) for _ in range(2))
        out, lse, _, _ = attend64(q, k, v, sees(new, keys, group, window), 0.3, torch.float32)
        for i in range(new):
            p = keys - new + i
            seen = [t for t in range(keys) if group == 0 or (p >= 0 and t // group <= p // group and
                                                             (window == 0 or t // group > p // group - window))]
            for a in range(4):
                e = [math.exp(0.3 * float(q[i, a] @ k[t, a // 2])) for t in seen]
                want = sum((x * v[t, a // 2] for x, t in zip(e, seen)), torch.zeros(8, dtype=torch.float64)) / (sum(e) or 1.0)
                assert (out[i, a] - want).abs().max() < 1e-12
                assert (lse[i, a] == -math.inf) if not seen else abs(lse[i, a] - math.log(sum(e))) < 1e-12
