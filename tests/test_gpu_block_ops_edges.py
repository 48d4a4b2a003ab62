"""Calls of the operators around a block's attention that the documentation allows and the ordinary tests do not make:
addresses off every vector size, offsets past 32 bits, extreme scales and inner extents, streams named by number, two calls
at once.  References and bounds as in the operators' own tests."""
import pytest
import torch

from block_ops_util import block_norm64, floor_step, half_step, mx_codes64, mx_values64, rope64
from paper_2607_28144_b200 import binding as B
from test_gpu_block_norm import EPS, _backward_check, _forward_check, _grads, _inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _off(t, by):
    """A packed copy of t whose first element lies `by` elements behind a 512-byte boundary."""
    buf = torch.full((t.numel() + by + 8,), float("nan"), dtype=t.dtype, device=DEV)
    out = buf[by: by + t.numel()].view(t.shape)
    out.copy_(t)
    return out


@pytest.mark.parametrize("n,c,per", [(1, 3, 1), (7, 33, 2), (40, 1536, 10), (900, 129, 300), (33, 4099, 33)])
@pytest.mark.parametrize("xt,iot", [("bf16", "bf16"), ("fp32", "fp16"), ("fp32", "fp32")])
def test_block_norm_at_odd_addresses(n, c, per, xt, iot):
    for by in (1, 3, 8):
        x, y, p, r = _inputs(n, c, per, n + c + by, T[xt], T[iot], True, True, 2, True, True)
        x, y = _off(x, by), _off(y, by + 1)
        h = _off(torch.zeros((n, c), dtype=T[iot], device=DEV), by + 2)
        kw = dict(norm=1, post_norm=2, eps=EPS, post_eps=EPS, tokens_per_mod=per)
        xo, _ = B.regenvc_block_norm_forward(x, y, **p, **kw, h=h)
        _forward_check(x, y, p, 1, 2, 1.0, per, xo, h)
        dh, dxo = _off(r(n, c).to(T[iot]), by), _off(r(n, c).to(T[xt]), 2 * by)
        got = _grads(xo, y, dh, dxo, p, 1, 2, 1.0, per)
        _backward_check(xo, y, dh, dxo, p, 1, 2, 1.0, per, got)
        # in place at the odd address
        again, _ = B.regenvc_block_norm_forward(x, y, **p, **kw, x_out=x)
        assert again is x and torch.equal(x, xo)
        same = _grads(xo, y, dh, dxo, p, 1, 2, 1.0, per, dx=dxo)
        assert all(torch.equal(same[k], got[k]) for k in got)


def test_block_norm_wide_rows_of_every_type_in_one_stage():
    """Gradients of 8191 and 8192 fp32 channels: one row of the four tensors fills a thread block's shared memory."""
    for c in (8191, 8192, 7000):
        x, y, p, r = _inputs(5, c, 2, c, torch.float32, torch.float32, True, True, 1, True, True)
        dh, dxo = r(5, c), r(5, c)
        _backward_check(x, y, dh, dxo, p, 1, 1, 0.25, 2, _grads(x, y, dh, dxo, p, 1, 1, 0.25, 2))


@pytest.mark.parametrize("c", [256, 251])
def test_offsets_past_32_bits(c):
    n, far = 3, (1 << 30) + 8                      # rows 2 GiB of bf16 apart: the last begins past 2^31 elements, 2^32 bytes
    buf = torch.empty((2 * far + 4096,), dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(buf, (n, c), (far, 1), 8)
    g = torch.Generator(device=DEV).manual_seed(c)
    x.copy_(torch.randn(n, c, generator=g, device=DEV))
    _, h = B.regenvc_block_norm_forward(x, norm=1, eps=EPS)
    _forward_check(x, None, {}, 1, 0, 1.0, n, None, h)
    dh = torch.randn(n, c, generator=g, device=DEV).bfloat16()
    _backward_check(x, None, dh, None, {}, 1, 0, 1.0, n, B.regenvc_block_norm_backward(dh, x, eps=EPS))
    codes, byte = mx_codes64(x.double())
    packed = B.regenvc_mxfp4_quantize(x)
    assert torch.equal(B.regenvc_mxfp4_dequantize(packed, n, c, torch.float32).double(), mx_values64(codes, byte, c))
    out = torch.as_strided(buf, (n, c), (far, 1), 2048)
    B.regenvc_mxfp4_dequantize(packed, n, c, out=out)
    assert torch.equal(out.double(), mx_values64(codes, byte, c))
    d = c // 4 * 2 if c % 2 == 0 else 250
    q = x[:, :d].unsqueeze(1)
    pos = torch.tensor([[3, 1000, 7]], dtype=torch.int32, device=DEV)
    qo, _ = B.regenvc_rope_axes(q, None, pos, [d])
    ref, mag = rope64(q.double(), pos, [d], 1e4, False, False, False)
    assert ((qo.double() - ref).abs() <= half_step(torch.bfloat16) * ref.abs() + 2.0 ** -21 * mag).all()


def _linear_check(x, w, f, ydt=torch.bfloat16, spread=0.0):
    wp = B.regenvc_mxfp4_quantize(w)
    y = B.regenvc_mxfp4_linear(x, wp, f, y_dtype=ydt)
    assert B.regenvc_device_status() == 0
    a, b = (mx_values64(*mx_codes64(t.double()), t.shape[1]) for t in (x, w))
    ref, mag = a @ b.t(), a.abs() @ b.abs().t()
    bound = half_step(ydt) * ref.abs() + x.shape[1] * 2.0 ** -23 * mag + floor_step(ydt)
    assert torch.isfinite(y).all() and ((y.double() - ref).abs() <= bound).all()


@pytest.mark.parametrize("n,k,f", [(1, 40000, 64), (1, 80640, 16), (1, 80700, 16), (4, 20096, 16), (4, 20200, 16), (3, 4096, 4088),
                                   (3, 4096, 4104), (1, 1, 8), (2, 31, 8), (1, 257, 4744), (300, 40000, 72)])
def test_inner_extents_at_the_ends_of_the_one_kernel_form(n, k, f):
    g = torch.Generator(device=DEV).manual_seed(n + k + f)
    _linear_check(torch.randn(n, k, generator=g, device=DEV), torch.randn(f, k, generator=g, device=DEV) / k ** 0.5, f)


@pytest.mark.parametrize("n", [1, 3, 200])
def test_scales_at_both_ends(n):
    """Values of 2^100 against weights of 2^-100 and the other way round: each scale is near an end of its range, their
    product is not.  (All codes and the result's terms are as in the ordinary case, times a power of two.)"""
    g = torch.Generator(device=DEV).manual_seed(n)
    x, w = torch.randn(n, 256, generator=g, device=DEV), torch.randn(64, 256, generator=g, device=DEV)
    for e in (100, -100, 118):
        _linear_check(x * 2.0 ** e, w * 2.0 ** -e, 64)


def test_more_tokens_than_one_round_of_pairs_and_features_that_end_inside_a_block():
    g = torch.Generator(device=DEV).manual_seed(5)
    for n, k, f in ((9601, 300, 584), (2817, 1536, 4616), (12480, 264, 1544)):
        _linear_check(torch.randn(n, k, generator=g, device=DEV).bfloat16(), torch.randn(f, k, generator=g, device=DEV), f)


@pytest.mark.parametrize("n,k,f", [(100, 256, 20000), (6, 700, 20008), (128, 300, 15376), (70, 520, 60008), (17, 1300, 28424)])
def test_few_tokens_and_many_features(n, k, f):
    """One tile of tokens: wide items of single thread blocks, one or several per block, starting in the middle of 128
    features and ending inside a block of 64."""
    g = torch.Generator(device=DEV).manual_seed(n + f)
    _linear_check(torch.randn(n, k, generator=g, device=DEV).bfloat16(), torch.randn(f, k, generator=g, device=DEV), f, torch.float16)


def test_streams_by_number_and_two_calls_at_once():
    n, c = 600, 512
    g = torch.Generator(device=DEV).manual_seed(6)
    x = [torch.randn(n, c, generator=g, device=DEV).bfloat16() for _ in range(2)]
    w = B.regenvc_mxfp4_quantize(torch.randn(768, c, generator=g, device=DEV))
    dh = torch.randn(n, c, generator=g, device=DEV).bfloat16()
    sc = 0.1 * torch.randn(6, c, generator=g, device=DEV)

    def chain(i, stream=None):
        _, h = B.regenvc_block_norm_forward(x[i], scale=sc, tokens_per_mod=100, stream=stream)
        y = B.regenvc_mxfp4_linear(h, w, 768, stream=stream)
        d = B.regenvc_block_norm_backward(dh, x[i], scale=sc, tokens_per_mod=100, stream=stream)
        return h, y, d["dx"], d["dscale"]

    want = [chain(i) for i in range(2)]
    torch.cuda.synchronize()
    legacy = chain(0, stream=0)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(legacy, want[0]))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for _ in range(5):
        for i, s in enumerate(streams):
            got[i] = chain(i, stream=s.cuda_stream if i else s)
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i]))
    assert B.regenvc_device_status() == 0


def test_operands_on_the_host_or_of_another_kind_are_refused():
    x = torch.zeros((4, 64), device=DEV)
    with pytest.raises(ValueError):
        B.regenvc_block_norm_forward(x, weight=torch.ones(64))
    with pytest.raises(ValueError):
        B.regenvc_rope_axes(x.view(4, 1, 64), None, torch.zeros((1, 4), dtype=torch.int32), [64])
    with pytest.raises(TypeError):
        B.regenvc_block_norm_forward(x.double())
    with pytest.raises(TypeError):
        B.regenvc_block_norm_forward(x, weight=torch.ones(64, device=DEV).double())
    with pytest.raises(TypeError):
        B.regenvc_block_norm_backward(x[:3], x)
    with pytest.raises(ValueError):
        B.regenvc_block_norm_forward(x, h=x.clone(), norm=B.NORM_NONE)
    with pytest.raises(B.RegenvcError):
        B.regenvc_block_norm_forward(x, norm=B.NORM_NONE)
    with pytest.raises(B.RegenvcError):
        B.regenvc_block_norm_forward(torch.zeros((0, 64), device=DEV))
    with pytest.raises(B.RegenvcError):
        B.regenvc_mxfp4_quantize(torch.zeros((0, 64), device=DEV))


def test_the_library_set_up_again_after_a_shutdown():
    g = torch.Generator(device=DEV).manual_seed(8)
    x, w = torch.randn(300, 256, generator=g, device=DEV), torch.randn(64, 256, generator=g, device=DEV)
    want = B.regenvc_mxfp4_linear(x, B.regenvc_mxfp4_quantize(w), 64)
    torch.cuda.synchronize()
    B.regenvc_shutdown()
    assert torch.equal(B.regenvc_mxfp4_linear(x, B.regenvc_mxfp4_quantize(w), 64), want)
    assert B.regenvc_device_status() == 0


def test_norm_of_float64_reference_at_a_zero_epsilon():
    """eps = 0 and tiny rows: the powers of 1 / deviation in the gradient stay in range (rows of 1e-15: 1 / deviation 1e15,
    its cube past fp32)."""
    n, c = 6, 96
    g = torch.Generator(device=DEV).manual_seed(12)
    x = torch.randn(n, c, generator=g, device=DEV) * 1e-15
    dh = torch.randn(n, c, generator=g, device=DEV) * 1e-15
    got = B.regenvc_block_norm_backward(dh, x, norm=2, eps=0.0)["dx"]
    xd = x.double().requires_grad_()
    _, h = block_norm64(xd, None, {}, 2, 0, 1.0, n, 0.0)
    (h * dh.double()).sum().backward()
    # T < 10 for these rows: 64 u (2 + T)^2 of a row's largest |dh| / deviation
    r = torch.rsqrt((x.double() ** 2).mean(1, keepdim=True))
    bound = 64 * 2.0 ** -24 * 144 * dh.double().abs().amax(1, keepdim=True) * r
    assert torch.isfinite(got).all() and ((got.double() - xd.grad).abs() <= bound).all()
