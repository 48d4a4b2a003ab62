"""Host-side checks of cache layouts, scales and status texts of the operators over cached windows.  Every call is refused."""
import ctypes

import pytest
import torch

from paper_2607_28144_b200 import binding as B
from paper_2607_28144_b200 import build


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


A = [0x100000000 * (i + 1) for i in range(24)]   # far apart, never dereferenced: every call below must fail


def append(L, kc, vc, q_out=A[9], **kw):
    d = dict(n_tokens=5, n_q_heads=4, n_k_heads=2, head_dim=64, type=0, n_sequences=3, page_size=16, n_pages=10, pages_per_sequence=4)
    d.update(kw)
    return L.regenvc_paged_append(ctypes.byref(B.PagedAppendDesc(**d)), A[0], A[1], A[2], None, None, None, A[6], A[7], A[8], q_out, kc, vc, None)


def caches(order, heads=2, slots=16, pages=10, d=64, near=0):
    """Strides and the distance of V (elements) of one tensor with axes (p, 2, s, h) in the given order."""
    size, stride, at = {"p": pages, "2": 2, "s": slots, "h": heads}, {}, d
    for a in reversed(order):
        stride[a] = at
        at *= size[a]
    return dict(k_page_stride=stride["p"], k_slot_stride=stride["s"], k_cache_head_stride=stride["h"], v_page_stride=stride["p"],
                v_slot_stride=stride["s"], v_cache_head_stride=stride["h"]), stride["2"] - near


@pytest.mark.parametrize("order", ["p2sh", "ps2h", "psh2", "ph2s", "phs2", "2psh", "hp2s", "h2ps", "s2ph", "sph2"])
def test_values_eight_elements_into_the_keys_are_refused(L, order):
    strides, apart = caches(order, near=8)
    assert append(L, A[10], A[10] + 2 * apart, **strides) == B.ERR_ALIASING
    assert append(L, A[10] + 2 * apart, A[10], **strides) == B.ERR_ALIASING


def test_values_among_the_keys_are_refused(L):
    # one slot on (the next slot's keys), one page on, one head on, and on the keys themselves
    strides, _ = caches("psh2")
    for far in (128, 256, 16 * 256, 0):
        assert append(L, A[10], A[10] + 2 * far, **strides) == B.ERR_ALIASING
    strides, _ = caches("ps2h")
    other = dict(strides, v_slot_stride=192)                         # the same pages, another step from slot to slot
    assert append(L, A[10], A[10] + 2 * 128, **other) == B.ERR_ALIASING


def test_strides_of_axes_with_one_entry_are_not_looked_at(L):
    """Refused for what comes later (keys given as the cache), not for a stride that no address uses."""
    for kw in (dict(n_k_heads=1, k_cache_head_stride=1 << 33, v_cache_head_stride=3), dict(page_size=1, k_slot_stride=1 << 33, v_slot_stride=8),
               dict(n_pages=1, k_page_stride=1 << 40, v_page_stride=1)):
        assert append(L, A[1], A[11], **kw) == B.ERR_ALIASING, kw
    for kw in (dict(k_cache_head_stride=1 << 33), dict(k_slot_stride=1 << 33), dict(k_page_stride=1 << 40)):
        assert append(L, A[1], A[11], **kw) == B.ERR_BAD_SHAPE, kw


def test_caches_whose_bytes_pass_64_bits_are_refused(L):
    assert append(L, A[1], A[11], n_pages=1 << 30, k_page_stride=1 << 38) == B.ERR_BAD_SHAPE
    assert append(L, A[11], A[1], n_pages=1 << 30, v_page_stride=1 << 36) == B.ERR_BAD_SHAPE
    assert append(L, A[1], A[11], n_pages=1 << 20, k_page_stride=1 << 38) == B.ERR_ALIASING      # 2^59 bytes: counted


def test_the_binding_names_short_strides_for_axes_with_one_entry():
    """Views of one tensor of 2^32 elements: (page, slot, head) strides that the library takes."""
    both = torch.empty((1 << 20, 2, 16, 1, 128), dtype=torch.bfloat16, device="meta")
    assert B._cache(both[:, 0], "k_cache", torch.bfloat16) == (4096, 128, 128)
    both = torch.empty((1 << 20, 2, 1, 16, 128), dtype=torch.bfloat16, device="meta")
    assert B._cache(both[:, 1], "v_cache", torch.bfloat16) == (4096, 128, 128)
    one = torch.empty((1, 2, 1 << 20, 16, 128), dtype=torch.bfloat16, device="meta")
    assert B._cache(one[:, :, :, :8][:, 1], "v_cache", torch.bfloat16)[1:] == (2048, 128)


def attend(L, scale, lse=A[7], **kw):
    d = B.PagedAttnDesc(n_tokens=5, n_q_heads=4, n_k_heads=2, head_dim=64, type=0, n_sequences=3, page_size=16, n_pages=10,
                        pages_per_sequence=4, scale=scale, **kw)
    return L.regenvc_paged_attn_forward(ctypes.byref(d), A[0], A[1], A[2], A[3], A[4], A[5], A[6], lse, A[8], 0, None)


def test_a_scale_whose_power_of_two_passes_the_range_is_refused(L):
    assert attend(L, 2.4e38) == B.ERR_UNSUPPORTED                     # times log2(e): past fp32
    assert attend(L, 1e38) == attend(L, 1e-45) == B.ERR_WORKSPACE     # in range; refused for the workspace of 0 bytes


def test_the_text_of_a_range_error_names_lists_and_operands():
    text = B.status_string(B.ERR_RANGE)
    assert "fp16" in text and "lists" in text
