"""Host-side tests of the operators around a block's attention: sizes of their buffers, every refusal before any CUDA
call, the binding's checks, and the 64-bit forms that the GPU tests compare with."""
import ctypes

import pytest
import torch

from block_ops_util import block_norm64, mx_codes64, mx_values64, rope64
from paper_2607_28144_b200 import binding as B
from paper_2607_28144_b200 import build


@pytest.fixture(scope="module")
def L():
    build.build()
    return B.lib()


A = [0x10000000 * (i + 1) for i in range(24)]   # far apart, never dereferenced: every call below must fail first


def _norm_desc(**kw):
    d = dict(n_tokens=4, channels=64, tokens_per_mod=4, x_type=0, io_type=0, norm=1, post_norm=0, eps=1e-6, post_eps=1e-6,
             residual_scale=1.0)
    d.update(kw)
    return B.BlockNormDesc(**d)


def _forward(L, desc, x=A[0], y=A[1], gate=A[2], pw=None, w=A[3], b=A[4], s=A[5], t=A[6], xo=A[7], h=A[8]):
    return L.regenvc_block_norm_forward(ctypes.byref(desc) if desc is not None else None, x, y, gate, pw, w, b, s, t, xo, h, None)


def test_block_norm_forward_refusals(L):
    d = _norm_desc()
    assert _forward(L, None) == B.ERR_NULL_POINTER
    assert _forward(L, d, x=None) == B.ERR_NULL_POINTER
    assert _forward(L, d, h=None) == B.ERR_NULL_POINTER                  # a norm without h
    assert _forward(L, _norm_desc(norm=0)) == B.ERR_NULL_POINTER         # h without a norm
    assert _forward(L, _norm_desc(norm=0), h=None, xo=None) == B.ERR_NULL_POINTER
    assert _forward(L, d, y=None) == B.ERR_NULL_POINTER                  # x_out and gate without y
    assert _forward(L, _norm_desc(post_norm=2), y=None, xo=None, gate=None) == B.ERR_NULL_POINTER
    for bad in (dict(n_tokens=0), dict(n_tokens=(1 << 30) + 1), dict(channels=0), dict(channels=8193), dict(tokens_per_mod=0),
                dict(x_stride=63), dict(h_stride=-64), dict(mod_stride=1), dict(y_stride=(1 << 31) + 1)):
        assert _forward(L, _norm_desc(**bad)) == B.ERR_BAD_SHAPE, bad
    for bad in (dict(x_type=3), dict(io_type=-1), dict(x_type=0, io_type=1), dict(x_type=1, io_type=2), dict(norm=3),
                dict(post_norm=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(post_eps=float("inf")),
                dict(residual_scale=float("nan"))):
        assert _forward(L, _norm_desc(**bad)) == B.ERR_UNSUPPORTED, bad
    assert _forward(L, d, x=A[0] + 1) == B.ERR_MISALIGNED
    assert _forward(L, _norm_desc(x_type=2), x=A[0] + 2) == B.ERR_MISALIGNED
    assert _forward(L, d, s=A[5] + 2) == B.ERR_MISALIGNED
    assert _forward(L, d, xo=A[0] + 16) == B.ERR_ALIASING                # shifted onto x: not in place
    assert _forward(L, _norm_desc(x_out_stride=128), xo=A[0]) == B.ERR_ALIASING   # x's address, another stride
    assert _forward(L, d, h=A[0]) == B.ERR_ALIASING
    assert _forward(L, d, h=A[7]) == B.ERR_ALIASING
    assert _forward(L, d, xo=A[1]) == B.ERR_ALIASING
    assert _forward(L, d, h=A[5]) == B.ERR_ALIASING
    # the last element of a strided operand counts
    assert _forward(L, _norm_desc(x_stride=1000), h=A[0] + 2 * (3 * 1000 + 63)) == B.ERR_ALIASING


def _backward(L, desc, xo=A[0], y=A[1], gate=A[2], pw=None, w=A[3], b=A[4], s=A[5], dh=A[6], dxo=A[7], dx=A[8], dy=A[9],
              dg=A[10], dpw=None, dw=A[11], db=A[12], ds=A[13], dt=A[14], ws=A[15], size=1 << 20):
    return L.regenvc_block_norm_backward(ctypes.byref(desc), xo, y, gate, pw, w, b, s, dh, dxo, dx, dy, dg, dpw, dw, db, ds,
                                         dt, ws, size, None)


def test_block_norm_backward_refusals(L):
    d = _norm_desc()
    need = B.regenvc_block_norm_workspace_bytes(4, 64)
    assert need == 4 * 9 * 64 * 4
    assert B.regenvc_block_norm_workspace_bytes(10 ** 6, 64) == 760 * 9 * 64 * 4
    assert B.regenvc_block_norm_workspace_bytes(0, 64) == 0 and B.regenvc_block_norm_workspace_bytes(4, 8193) == 0
    assert _backward(L, d, size=need - 1) == B.ERR_WORKSPACE
    assert _backward(L, d, ws=A[15] + 8) == B.ERR_WORKSPACE
    for bad in (dict(ws=None), dict(xo=None), dict(dh=None), dict(y=None), dict(gate=None), dict(w=None), dict(s=None),
                dict(dpw=A[16])):
        assert _backward(L, d, **bad) == B.ERR_NULL_POINTER, bad
    n = _norm_desc(norm=0)
    assert _backward(L, n, dh=None) == B.ERR_NULL_POINTER                # dweight and its like without dh
    assert _backward(L, n, dh=None, dw=None, db=None, ds=None, dt=None, dxo=None) == B.ERR_NULL_POINTER
    none = dict(dx=None, dy=None, dg=None, dw=None, db=None, ds=None, dt=None)
    assert _backward(L, d, **none) == B.ERR_NULL_POINTER                 # nothing asked for
    assert _backward(L, d, dx=A[6]) == B.ERR_ALIASING
    assert _backward(L, d, dx=A[7] + 32) == B.ERR_ALIASING
    assert _backward(L, d, dw=A[11], db=A[11]) == B.ERR_ALIASING
    assert _backward(L, d, dg=A[15]) == B.ERR_ALIASING                   # the workspace is written too
    assert _backward(L, _norm_desc(dx_stride=10)) == B.ERR_BAD_SHAPE


def _rope_desc(**kw):
    d = dict(n_tokens=5, n_q_heads=4, n_k_heads=2, head_dim=64, type=0, n_axes=3, widths=(ctypes.c_int * 4)(20, 22, 22),
             rope_theta=1e4)
    if "widths" in kw:
        kw["widths"] = (ctypes.c_int * 4)(*kw["widths"])
    d.update(kw)
    return B.RopeAxesDesc(**d)


def _rope(L, desc, q=A[0], k=A[1], pos=A[2], qo=A[3], ko=A[4]):
    return L.regenvc_rope_axes(ctypes.byref(desc), q, k, pos, qo, ko, None)


def test_rope_axes_refusals(L):
    d = _rope_desc()
    assert L.regenvc_rope_axes(None, *A[:5], None) == B.ERR_NULL_POINTER
    for bad in (dict(q=None), dict(pos=None), dict(qo=None), dict(k=None), dict(ko=None), dict(k=None, ko=None)):
        assert _rope(L, d, **bad) == B.ERR_NULL_POINTER, bad
    assert _rope(L, _rope_desc(n_k_heads=0)) == B.ERR_NULL_POINTER
    for bad in (dict(n_tokens=0), dict(n_q_heads=0), dict(n_k_heads=-1), dict(head_dim=0), dict(head_dim=258), dict(n_axes=0),
                dict(n_axes=5), dict(widths=(20, 22, 24)), dict(widths=(20, 21, 22)), dict(widths=(0, 22, 22)),
                dict(pos_stride=4), dict(q_head_stride=63), dict(q_token_stride=32), dict(q_out_token_stride=-1),
                dict(q_head_stride=100, q_token_stride=256), dict(n_q_heads=65536)):
        assert _rope(L, _rope_desc(**bad)) == B.ERR_BAD_SHAPE, bad
    for bad in (dict(head_dim=63, widths=(20, 20, 20)), dict(type=3), dict(rope_theta=0.0), dict(rope_theta=float("nan")),
                dict(halves=2), dict(inverse=-1)):
        assert _rope(L, _rope_desc(**bad)) == B.ERR_UNSUPPORTED, bad
    assert _rope(L, d, q=A[0] + 1) == B.ERR_MISALIGNED
    assert _rope(L, _rope_desc(type=2), k=A[1] + 2) == B.ERR_MISALIGNED
    assert _rope(L, d, pos=A[2] + 2) == B.ERR_MISALIGNED
    assert _rope(L, d, qo=A[0] + 16) == B.ERR_ALIASING
    assert _rope(L, _rope_desc(q_out_token_stride=512), qo=A[0]) == B.ERR_ALIASING    # q's address, other strides
    assert _rope(L, d, qo=A[1]) == B.ERR_ALIASING
    assert _rope(L, d, ko=A[3]) == B.ERR_ALIASING
    assert _rope(L, d, qo=A[2]) == B.ERR_ALIASING
    fused = dict(q_token_stride=8 * 64, k_token_stride=8 * 64, q_out_token_stride=8 * 64, k_out_token_stride=8 * 64)
    # k one element too near to q inside the fused rows, and k running over the end of a row into the next one's q
    assert _rope(L, _rope_desc(**fused), q=A[0], qo=A[0], k=A[0] + 2 * (4 * 64 - 8), ko=A[0] + 2 * (4 * 64 - 8)) == B.ERR_ALIASING
    assert _rope(L, _rope_desc(**fused), q=A[0], qo=A[0], k=A[0] + 2 * 7 * 64, ko=A[0] + 2 * 7 * 64) == B.ERR_ALIASING


def test_mxfp4_sizes_and_refusals(L):
    assert B.regenvc_mxfp4_bytes(1, 1) == 512 + 512
    assert B.regenvc_mxfp4_bytes(129, 129) == (129 * 128 + 511) // 512 * 512 + 2 * 2 * 512
    assert B.regenvc_mxfp4_bytes(4608, 1536) == 4608 * 768 + 36 * 12 * 512
    assert B.regenvc_mxfp4_bytes(0, 5) == 0 and B.regenvc_mxfp4_bytes(5, 0) == 0 and B.regenvc_mxfp4_bytes(1, (1 << 24) + 1) == 0
    q = L.regenvc_mxfp4_quantize
    assert q(None, 0, 4, 4, 0, A[1], None) == B.ERR_NULL_POINTER
    assert q(A[0], 0, 4, 4, 0, None, None) == B.ERR_NULL_POINTER
    assert q(A[0], 0, 0, 4, 0, A[1], None) == B.ERR_BAD_SHAPE
    assert q(A[0], 0, 4, 4, 3, A[1], None) == B.ERR_BAD_SHAPE
    assert q(A[0], 3, 4, 4, 0, A[1], None) == B.ERR_UNSUPPORTED
    assert q(A[0] + 1, 0, 4, 4, 0, A[1], None) == B.ERR_MISALIGNED
    assert q(A[0], 0, 4, 4, 0, A[1] + 128, None) == B.ERR_MISALIGNED
    assert q(A[0], 0, 4, 4, 0, A[0], None) == B.ERR_ALIASING
    assert L.regenvc_mxfp4_dequantize(A[0], A[0] + 1022, 0, 4, 4, 0, None) == B.ERR_ALIASING
    p = L.regenvc_mxfp4_project
    assert p(None, A[1], None, A[2], 0, 4, 8, 32, None) == B.ERR_NULL_POINTER
    assert p(A[0], None, None, A[2], 0, 4, 8, 32, None) == B.ERR_NULL_POINTER
    assert p(A[0], A[1], None, None, 0, 4, 8, 32, None) == B.ERR_NULL_POINTER
    assert p(A[0], A[1], None, A[2], 0, 4, 0, 32, None) == B.ERR_BAD_SHAPE
    assert p(A[0], A[1], None, A[2], 0, 1 << 30, 1 << 24, 8, None) == B.ERR_BAD_SHAPE
    assert p(A[0], A[1], None, A[2], 0, 4, 12, 32, None) == B.ERR_UNSUPPORTED
    assert p(A[0], A[1], None, A[2], 2, 4, 8, 32, None) == B.ERR_UNSUPPORTED
    assert p(A[0], A[1] + 16, None, A[2], 0, 4, 8, 32, None) == B.ERR_MISALIGNED
    assert p(A[0] + 16, A[1], None, A[2], 0, 4, 8, 32, None) == B.ERR_MISALIGNED
    assert p(A[0], A[1], None, A[2] + 8, 0, 4, 8, 32, None) == B.ERR_MISALIGNED
    assert p(A[0], A[1], A[3] + 2, A[2], 0, 4, 8, 32, None) == B.ERR_MISALIGNED
    assert p(A[0], A[1], None, A[0], 0, 4, 8, 32, None) == B.ERR_ALIASING
    assert p(A[0], A[1], A[2] + 32, A[2], 0, 4, 8, 32, None) == B.ERR_ALIASING
    s = B.regenvc_mxfp4_linear_scratch_bytes
    assert s(1, 8, 80640) == 0 and s(1, 8, 80641) == B.regenvc_mxfp4_bytes(1, 80641)
    assert s(4, 8, 20096) == 0 and s(4, 8, 20097) == B.regenvc_mxfp4_bytes(4, 20097)
    assert s(1, 1 << 17, 4096) == 0 and s(2, 4096, 4096) == B.regenvc_mxfp4_bytes(2, 4096) and s(2, 4088, 4096) == 0
    assert s(5, 8, 32) == B.regenvc_mxfp4_bytes(5, 32) and s(0, 8, 32) == 0 and s(1, 0, 32) == 0
    f = L.regenvc_mxfp4_linear
    assert f(None, 0, 0, A[1], None, A[2], 0, 4, 8, 32, None, None) == B.ERR_NULL_POINTER
    assert f(A[0], 0, 0, A[1], None, A[2], 0, 5, 8, 32, None, None) == B.ERR_NULL_POINTER
    assert f(A[0], 5, 0, A[1], None, A[2], 0, 5, 8, 32, A[3], None) == B.ERR_UNSUPPORTED
    assert f(A[0], 0, 31, A[1], None, A[2], 0, 5, 8, 32, A[3], None) == B.ERR_BAD_SHAPE
    assert f(A[0], 0, 0, A[1], None, A[2], 0, 5, 8, 32, A[3] + 64, None) == B.ERR_MISALIGNED
    assert f(A[0], 0, 0, A[1], None, A[0], 0, 4, 8, 32, A[3], None) == B.ERR_ALIASING
    assert f(A[0], 0, 0, A[1], None, A[2], 0, 5, 8, 32, A[1], None) == B.ERR_ALIASING
    assert f(A[0], 0, 0, A[1], A[3] + 512, A[2], 0, 5, 8, 32, A[3], None) == B.ERR_ALIASING


def test_no_cpu_fallback(L):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    raw = (ctypes.c_uint8 * 65536)()
    a = (ctypes.addressof(raw) + 255) & ~255
    assert L.regenvc_mxfp4_quantize(a, 0, 4, 32, 0, a + 4096, None) in (B.ERR_CUDA, B.ERR_UNSUPPORTED)
    assert _forward(L, _norm_desc(), a, a + 4096, None, None, None, None, None, None, a + 8192, a + 16384) in (B.ERR_CUDA, B.ERR_UNSUPPORTED)


def test_binding_rejects_cpu_tensors_and_rows_that_share_memory():
    t = torch.zeros((4, 64), dtype=torch.bfloat16)
    for call in (lambda: B.regenvc_block_norm_forward(t), lambda: B.regenvc_block_norm_backward(t, t),
                 lambda: B.regenvc_rope_axes(t.view(4, 1, 64), None, torch.zeros((1, 4), dtype=torch.int32), [64]),
                 lambda: B.regenvc_mxfp4_quantize(t)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError):
        B._row_stride(torch.zeros((1, 64)).expand(4, 64))
    assert B._row_stride(torch.zeros((4, 64))[:, :32]) == 64 and B._row_stride(torch.zeros((1, 64))) == 0


def test_the_plain_norm_and_its_differences():
    """The automatic gradient that the GPU tests use, against differences of the plain form (64 bits: truncation
    ~ step^2, rounding ~ 1e-16 / step)."""
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    for norm, post in ((1, 0), (2, 2), (1, 1), (0, 2)):
        p = {k: r(2, 6).requires_grad_() for k in ("gate", "scale", "shift")}
        p.update({k: r(6).requires_grad_() for k in ("post_weight", "weight", "bias")})
        x, y = r(5, 6).requires_grad_(), r(5, 6).requires_grad_()
        cx, ch = r(5, 6), r(5, 6)

        def value():
            t, h = block_norm64(x, y, p, norm, post, 0.7, 3, 1e-6)
            return (t * cx).sum() + (0.0 if h is None else (h * ch).sum())

        value().backward()
        for leaf in [x, y, *p.values()]:
            if leaf.grad is None:
                continue
            d = r(*leaf.shape)
            with torch.no_grad():
                leaf += 1e-5 * d
                up = value()
                leaf -= 2e-5 * d
                down = value()
                leaf += 1e-5 * d
            want = float((leaf.grad * d).sum())
            assert abs(float(up - down) / 2e-5 - want) <= 1e-6 * (1 + abs(want)) * 10


def test_the_plain_rotation_keeps_lengths_and_turns_back():
    g = torch.Generator().manual_seed(2)
    x = torch.randn(7, 3, 20, generator=g, dtype=torch.float64)
    pos = torch.randint(-50, 1000, (2, 7), generator=g)
    for halves in (False, True):
        y, _ = rope64(x, pos, [6, 8], 1e4, halves, False, False)
        assert torch.allclose(y.norm(dim=2), x.norm(dim=2), rtol=1e-13) and torch.equal(y[..., 14:], x[..., 14:])
        assert torch.allclose(rope64(y, pos, [6, 8], 1e4, halves, False, True)[0], x, rtol=0, atol=1e-13)


def test_the_plain_4_bit_form():
    x = torch.tensor([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -5.0, 7.9, 0.0, -0.24] + [0.0] * 20], dtype=torch.float64)
    codes, byte = mx_codes64(x)
    assert byte.tolist() == [[127]]                # largest magnitude in [4, 8): scale 1
    assert mx_values64(codes, byte, 12)[0].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, -4.0, 6.0, 0.0, 0.0]
