"""The operators around a block's attention at the library's real sizes, where a thread block walks over more rows than its
ring or its batch of loads holds.  References, bounds and guards as in the operators' own tests."""
import pytest
import torch

from block_ops_util import half_step, mx_values64, rope64
from paper_2607_28144_b200 import binding as B
from test_gpu_block_norm import _backward_check, _forward_check, _grads, _guarded, _inputs
from test_gpu_mxfp4 import _check_packed, _product_check, _quantised64, _values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6
T = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}

# tokens, channels, tokens per modulation row, types, norm, post norm: the 480x832 window with a row per frame, a wide fp32
# stream, narrow and odd rows, rows that leave room for one or two stages only, a modulation row per token
NORMS = [(10920, 1536, 1560, "bf16", "bf16", 1, 0), (10920, 1536, 10920, "fp16", "fp16", 2, 1), (4000, 5120, 1560, "fp32", "bf16", 1, 2),
         (20000, 200, 20000, "bf16", "bf16", 1, 0), (10000, 1531, 4000, "bf16", "bf16", 1, 2), (6000, 777, 613, "fp32", "fp32", 1, 1),
         (2000, 8192, 999, "fp32", "fp32", 2, 2), (1500, 7001, 1500, "fp32", "fp16", 1, 1), (3000, 512, 1, "fp32", "bf16", 1, 2)]


@pytest.mark.parametrize("n,c,per,xt,iot,norm,post", NORMS)
def test_block_norm(n, c, per, xt, iot, norm, post):
    x, y, p, r = _inputs(n, c, per, n + c, T[xt], T[iot], True, True, post, True, True)
    xo, check_x = _guarded(n, c, T[xt])
    h, check_h = _guarded(n, c, T[iot])
    B.regenvc_block_norm_forward(x, y, **p, norm=norm, post_norm=post, residual_scale=0.5, eps=EPS, post_eps=EPS, tokens_per_mod=per,
                                 x_out=xo, h=h)
    check_x()
    check_h()
    _forward_check(x, y, p, norm, post, 0.5, per, xo, h)
    dh, more = r(n, c).to(T[iot]), r(n, c).to(T[xt])
    got = _grads(x, y, dh, more, p, norm, post, 0.5, per)
    _backward_check(x, y, dh, more, p, norm, post, 0.5, per, got)
    again = _grads(x, y, dh, more, p, norm, post, 0.5, per)
    assert all(got[k] is None or torch.equal(got[k], again[k]) for k in got), "two calls differ"


@pytest.mark.parametrize("rows,cols,dtype", [(10920, 1536, "bf16"), (9000, 5120, "fp16"), (4608, 1536, "bf16"), (4000, 4097, "fp32"),
                                             (3000, 8192, "fp32"), (20000, 130, "bf16")])
def test_to_4_bits_and_back(rows, cols, dtype):
    x = _values(rows + cols, rows, cols, T[dtype])
    need = B.regenvc_mxfp4_bytes(rows, cols)
    buf = torch.full((need + 512,), 0xA5, dtype=torch.uint8, device=DEV)
    B.regenvc_mxfp4_quantize(x, buf[:need])
    assert (buf[need:] == 0xA5).all(), "wrote past the packed form"
    codes, byte = _check_packed(buf[:need], x)
    want = mx_values64(codes, byte, cols)
    del codes
    for out in (torch.bfloat16, torch.float32):
        back, check = _guarded(rows, cols, out)
        B.regenvc_mxfp4_dequantize(buf[:need], rows, cols, out=back)
        check()
        assert torch.equal(back.double(), want.to(out).double())


@pytest.mark.parametrize("n,k,f", [(10920, 1536, 4608), (10920, 4608, 1536), (3000, 5120, 5120)])
def test_4_bit_linear(n, k, f):
    x, w = _values(n, n, k, torch.bfloat16, False), _values(f, f, k, torch.float32, False) / k ** 0.5
    y = B.regenvc_mxfp4_linear(x, B.regenvc_mxfp4_quantize(w), f)
    assert B.regenvc_device_status() == 0
    _product_check(y, _quantised64(x), _quantised64(w), None)


@pytest.mark.parametrize("n,hq,hk,halves,dtype", [(10920, 12, 12, False, "bf16"), (4097, 40, 8, True, "fp16"), (12480, 40, 40, False, "bf16")])
def test_rotation(n, hq, hk, halves, dtype):
    g = torch.Generator(device=DEV).manual_seed(n)
    q, k = (torch.randn(n, h, 128, generator=g, device=DEV).to(T[dtype]) for h in (hq, hk))
    i = torch.arange(n, device=DEV)
    pos = torch.stack([i // 1560, i // 52 % 30, i % 52]).int()
    for inverse in (False, True):
        got = B.regenvc_rope_axes(q, k, pos, [44, 42, 42] if not halves else [32, 48, 48], halves=halves, inverse=inverse)
        for x, y in zip((q, k), got):
            ref, mag = rope64(x.double(), pos, [44, 42, 42] if not halves else [32, 48, 48], 1e4, halves, False, inverse)
            assert ((y.double() - ref).abs() <= half_step(T[dtype]) * ref.abs() + 2.0 ** -21 * mag + 2.0 ** -25).all()


@pytest.mark.parametrize("norm", [0, 1, 2])
@pytest.mark.parametrize("post", [0, 1, 2])
@pytest.mark.parametrize("xt,iot", [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32")])
def test_gradients_of_every_pair_of_norms(norm, post, xt, iot):
    """Which sums share an exchange depends on both norms and on the types; rows of one warp, of several, and as images."""
    for n, c, per in ((700, 200, 300), (900, 1536, 900), (300, 5120, 77), (400, 1531, 133)):
        x, y, p, r = _inputs(n, c, per, n + c, T[xt], T[iot], True, True, post, norm > 0, norm > 0)
        dh, more = (r(n, c).to(T[iot]) if norm else None), r(n, c).to(T[xt])
        got = _grads(x, y, dh, more, p, norm, post, 0.5, per)
        _backward_check(x, y, dh, more, p, norm, post, 0.5, per, got)
        xo, h = B.regenvc_block_norm_forward(x, y, **p, norm=norm, post_norm=post, residual_scale=0.5, eps=EPS, post_eps=EPS,
                                             tokens_per_mod=per)
        _forward_check(x, y, p, norm, post, 0.5, per, xo, h)
