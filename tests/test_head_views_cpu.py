"""Queries and keys that share memory, and strides as the library takes them, without a GPU: every call is refused."""
import ctypes

import pytest
import torch

from paper_2607_28144_b200 import binding as B
from paper_2607_28144_b200 import build


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


AT = 0x100000000                     # never dereferenced: every call below must fail


def in_place(L, token, head, far, n=5, hq=4, hk=4, k_token=None):
    """q at AT and k `far` elements on, both replaced in place."""
    d = B.QkNormRopeDesc(n_tokens=n, n_q_heads=hq, n_k_heads=hk, head_dim=64, type=0, eps=1e-6, q_token_stride=token, q_head_stride=head,
                         q_out_token_stride=token, q_out_head_stride=head, k_token_stride=k_token or token, k_head_stride=head,
                         k_out_token_stride=k_token or token, k_out_head_stride=head)
    k = AT + 2 * far
    return L.regenvc_qk_norm_rope_forward(ctypes.byref(d), AT, k, None, None, None, AT, k, None)


def test_vectors_that_meet_are_refused(L):
    # (tokens, heads, 3, 64), (tokens, 3, heads, 64), (heads, tokens, 3, 64), (heads, 3, tokens, 64), (3, ...): k too near or on
    # q's own vectors
    for token, head, apart in ((768, 192, 64), (768, 64, 256), (192, 960, 64), (64, 960, 320)):
        for far in (0, 8, apart - 8, head, token, head + 8, token + 56):
            assert in_place(L, token, head, far) == B.ERR_ALIASING, (token, head, far)
    assert in_place(L, 768, 192, 64, k_token=1536) == B.ERR_ALIASING     # another step from token to token
    assert in_place(L, 768, 192, 192, hq=4, hk=1) == B.ERR_ALIASING      # a key of q's second head
    assert in_place(L, 768, 192, 128 + 8, hq=4, hk=1) == B.ERR_ALIASING  # ... that runs into it


def test_one_token_of_heads_that_lie_far_apart():
    """[heads, tokens, d] buffers: the stride of a single token means nothing, whatever the heads' is."""
    for n, heads, strides, want in ((1, 3, (64, 1 << 30, 1), (192, 1 << 30)), (1, 1, (7, 9, 1), (0, 0)), (2, 1, (640, 5, 1), (640, 64)),
                                    (2, 3, (64, 1 << 30, 1), (64, 1 << 30))):
        t = torch.empty_strided((n, heads, 64), strides, dtype=torch.bfloat16, device="meta")
        assert B._own_strides(t, "q", n, heads, 64) == want
        assert B._head_strides(t, "q", torch.bfloat16, n, heads, 64) == want
