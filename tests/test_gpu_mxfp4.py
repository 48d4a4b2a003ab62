"""Microscaled 4-bit matrices.  Quantisation is exact arithmetic and a search: the codes, the scales and their places in
the packed form have to be equal.  Product: 4-bit products with power-of-two scales are exact; the fp32 accumulation of K
terms is off by at most K 2^-23 of the sum of their magnitudes (the tensor core may truncate), then half a step of the
result's type."""
import pytest
import torch

from block_ops_util import floor_step, half_step, mx_codes64, mx_unpack, mx_values64
from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def _values(seed, rows, cols, dtype, spread=True):
    g = torch.Generator(device=DEV).manual_seed(seed)
    v = torch.randn(rows, cols, generator=g, device=DEV)
    if spread:
        v = v * torch.exp2(torch.randint(-6, 6, (rows, 1), generator=g, device=DEV).float())
    return v.to(dtype)


def _check_packed(packed, x):
    rows, cols = x.shape
    codes, byte = mx_codes64(x.double())
    got, got_byte = mx_unpack(packed, rows, cols)
    nb = byte.shape[1]
    assert torch.equal(got_byte[:, :nb], byte) and (got_byte[:, nb:] == 0).all(), "scales"
    assert torch.equal(got[:, :nb], codes), "codes"
    assert (got[:, nb:] == 0).all(), "padding codes"
    # scales of the rows that fill up the last tile
    kp = -(-cols // 128) * 128
    tiles = packed[-(-(rows * kp // 2) // 512) * 512:].view(-1, kp // 128, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, kp // 32)
    assert (tiles[rows:] == 0).all()
    return codes, byte


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (5, 128), (128, 256), (129, 1000), (300, 1536), (31, 129), (1000, 40),
                                       (2, 8200)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_quantise_and_read_back(rows, cols, dtype):
    x = _values(rows + cols, rows, cols, T[dtype])
    need = B.regenvc_mxfp4_bytes(rows, cols)
    buf = torch.full((need + 512,), 0xA5, dtype=torch.uint8, device=DEV)
    B.regenvc_mxfp4_quantize(x, buf[:need])
    assert (buf[need:] == 0xA5).all(), "wrote past the packed form"
    codes, byte = _check_packed(buf[:need], x)
    for out in T.values():
        if dtype == "fp32" and out == torch.float16:
            continue
        back = B.regenvc_mxfp4_dequantize(buf[:need], rows, cols, out)
        assert torch.equal(back.double(), mx_values64(codes, byte, cols).to(out).double())


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_ties_zeros_extremes_and_blocks_that_hold_nan(dtype):
    t = T[dtype]
    x = torch.zeros((6, 96), device=DEV, dtype=torch.float32)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, -0.25, -2.5, -5.0, 7.99], device=DEV)
    for r, s in enumerate((1.0, 2.0 ** -10, 2.0 ** 8)):
        x[r, :12] = ties * s
        x[r, 32:44] = -ties * s
    x[3, 5] = float("nan")
    x[3, 40] = float("inf")
    x[3, 70] = -1.0
    x[4, :] = -0.0
    tiny = {"bf16": 1.2e-38, "fp16": 6e-8, "fp32": 1e-45}[dtype]      # at or below the smallest normal values
    x[5, 0], x[5, 33], x[5, 64] = tiny, 3 * tiny, torch.finfo(t).max
    x = x.to(t)
    packed = B.regenvc_mxfp4_quantize(x)
    codes, byte = _check_packed(packed, x)
    assert byte[3].tolist()[:2] == [255, 255] and byte[3, 2] == 125
    back = B.regenvc_mxfp4_dequantize(packed, 6, 96, torch.float32)
    assert torch.isnan(back[3, :64]).all() and torch.isfinite(back[3, 64:]).all()
    assert torch.equal(back.double().nan_to_num(1.25), mx_values64(codes, byte, 96).nan_to_num(1.25))


def test_strided_rows_and_odd_addresses():
    buf = _values(3, 50, 400, torch.bfloat16)
    for a, b in ((0, 256), (8, 264), (1, 200), (3, 4)):
        x = buf[:, a:b]
        packed = B.regenvc_mxfp4_quantize(x)
        _check_packed(packed, x)
        out = torch.full((50, 401), 7.0, dtype=torch.float32, device=DEV)
        B.regenvc_mxfp4_dequantize(packed, 50, b - a, out=out[:, 1: 1 + b - a])
        assert torch.equal(out[:, 1: 1 + b - a], B.regenvc_mxfp4_dequantize(packed, 50, b - a, torch.float32))
        assert (out[:, 0] == 7).all() and (out[:, 1 + b - a:] == 7).all()


def _product_check(y, x64, w64, bias):
    ref, mag = x64 @ w64.t(), x64.abs() @ w64.abs().t()
    if bias is not None:
        ref, mag = ref + bias.double(), mag + bias.double().abs()
    bound = half_step(y.dtype) * ref.abs() + x64.shape[1] * 2.0 ** -23 * mag + floor_step(y.dtype)
    err = (y.double() - ref).abs()
    assert torch.isfinite(y).all() and (err <= bound).all(), f"{(err / bound).max().item():.3g} times the bound"


def _quantised64(x):
    codes, byte = mx_codes64(x.double())
    return mx_values64(codes, byte, x.shape[1])


# tokens, in_features, out_features: single tokens and features, half stages of K, tiles that begin in the middle of 128
# features, a thread block with several items (more items than SMs, more K stages than buffers), ragged everything
SHAPES = [(1, 32, 8), (1, 1536, 9216), (2, 1536, 1536), (3, 100, 200), (4, 5120, 1024), (5, 128, 64), (8, 640, 1000), (17, 130, 24),
          (100, 256, 192), (128, 384, 200), (129, 1536, 4608), (257, 2000, 1000), (1000, 1536, 2056), (130, 5120, 640),
          (6000, 128, 1536), (4500, 896, 1160), (20000, 200, 392)]


@pytest.mark.parametrize("n,k,f", SHAPES)
def test_product(n, k, f):
    x, w = _values(n + k, n, k, torch.bfloat16, False), _values(n + f, f, k, torch.float32, False) / k ** 0.5
    bias = torch.randn(f, device=DEV, generator=torch.Generator(device=DEV).manual_seed(f))
    xp, wp = B.regenvc_mxfp4_quantize(x), B.regenvc_mxfp4_quantize(w)
    x64, w64 = _quantised64(x), _quantised64(w)
    buf = torch.full(((n + 2) * f,), float("nan"), dtype=torch.bfloat16, device=DEV)
    y = buf[: n * f].view(n, f)
    B.regenvc_mxfp4_project(xp, wp, n, f, k, bias, y=y)
    assert B.regenvc_device_status() == 0
    assert torch.isnan(buf[n * f:]).all(), "wrote past y"
    _product_check(y, x64, w64, bias)
    assert torch.equal(B.regenvc_mxfp4_project(xp, wp, n, f, k, bias), y), "two calls differ"
    # the call that quantises inside, of each type of x, without bias, fp16 result
    for t in T.values():
        xt = x.to(t)
        y2 = B.regenvc_mxfp4_linear(xt, wp, f, None, y_dtype=torch.float16)
        assert B.regenvc_device_status() == 0
        _product_check(y2, _quantised64(xt), w64, None)


@pytest.mark.parametrize("n", [1, 4, 100, 300, 5000])
def test_small_whole_numbers_come_out_exactly(n):
    """Codes that are whole numbers, scales 1: every sum is a whole number below 2^8 = what bf16 holds exactly."""
    k, f = 192, 328
    g = torch.Generator(device=DEV).manual_seed(n)
    x = torch.randint(-1, 2, (n, k), generator=g, device=DEV).float()
    w = torch.randint(-1, 2, (f, k), generator=g, device=DEV).float()
    x[:, ::32], w[:, ::32] = 4.0, 0.0                # a 4 in each block fixes the scale at 1; it meets a zero
    w[:, 1::32], x[:, 1::32] = 4.0, 0.0
    y = B.regenvc_mxfp4_linear(x.bfloat16(), B.regenvc_mxfp4_quantize(w), f)
    assert (x.double() @ w.double().t()).abs().max() <= 256
    assert torch.equal(y.double(), x.double() @ w.double().t())


@pytest.mark.parametrize("n", [1, 3, 200])
def test_nan_and_infinity_stay_in_their_rows_and_columns(n):
    k, f = 200, 264
    x, w = _values(1, n, k, torch.float32, False), _values(2, f, k, torch.float32, False)
    w[7, 150] = float("nan")
    if n > 1:
        x[1, 3] = float("inf")
    y = B.regenvc_mxfp4_linear(x, B.regenvc_mxfp4_quantize(w), f)
    assert B.regenvc_device_status() == 0
    bad = torch.zeros((n, f), dtype=torch.bool, device=DEV)
    bad[:, 7] = True
    if n > 1:
        bad[1] = True
    assert torch.equal(torch.isnan(y), bad) and torch.isfinite(y[~bad]).all()


@pytest.mark.parametrize("n", [1, 2, 700])
def test_strided_activations_streams_graphs_and_launches(n):
    k, f = 320, 512
    big = _values(n, n, k + 40, torch.bfloat16, False)
    w = B.regenvc_mxfp4_quantize(_values(9, f, k, torch.float32, False))
    for a in (0, 8, 3):
        x = big[:, a: a + k]
        want = B.regenvc_mxfp4_linear(x.contiguous(), w, f)
        assert torch.equal(B.regenvc_mxfp4_linear(x, w, f), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = B.regenvc_mxfp4_linear(x, w, f, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    static = x.clone()
    with torch.cuda.graph(graph):
        y = B.regenvc_mxfp4_linear(static, w, f)
    other = _values(77, n, k, torch.bfloat16, False)
    want = B.regenvc_mxfp4_linear(other, w, f)
    static.copy_(other)
    for _ in range(3):
        graph.replay()
    assert torch.equal(y, want) and B.regenvc_device_status() == 0
    before = B.regenvc_kernel_launch_count()
    B.regenvc_mxfp4_linear(static, w, f)
    assert B.regenvc_kernel_launch_count() - before in (1, 2)


def test_a_set_status_word_skips_the_product_and_its_report_clears_it():
    n, k, f = 300, 256, 512
    x, w = _values(1, n, k, torch.bfloat16, False), B.regenvc_mxfp4_quantize(_values(2, f, k, torch.float32, False))
    want = B.regenvc_mxfp4_linear(x, w, f)
    assert B.regenvc_device_status() == 0
    B.regenvc_debug_expire_wait(200)
    B.regenvc_mxfp4_linear(x, w, f)
    assert B.regenvc_device_status() == B.ERR_TIMEOUT and B.regenvc_device_status() == 0
    assert torch.equal(B.regenvc_mxfp4_linear(x, w, f), want)


def test_refusals_of_the_binding():
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    w = B.regenvc_mxfp4_quantize(torch.zeros((16, 64), device=DEV))
    with pytest.raises(TypeError):
        B.regenvc_mxfp4_linear(x, w[:-1], 16)
    with pytest.raises(TypeError):
        B.regenvc_mxfp4_linear(x.t(), w, 16)
    with pytest.raises(ValueError):
        B.regenvc_mxfp4_quantize(x[:1].expand(4, 64))
    with pytest.raises(TypeError):
        B.regenvc_mxfp4_linear(x, w, 16, torch.zeros(15, device=DEV))
    with pytest.raises(B.RegenvcError) as e:
        B.regenvc_mxfp4_linear(x, w, 12)
    assert e.value.code == B.ERR_UNSUPPORTED


@pytest.mark.parametrize("n", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_values_of_few_tokens_one_by_one(n, dtype):
    """Weights with a single 1 per feature give back x as it was taken to 4 bits, exactly: every code, tie and sign, of each
    token, from x itself and from its packed form."""
    k = 160
    x = torch.zeros((n, k), device=DEV)
    steps = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.2, 0.3, 0.7, 0.8, 4.9, 5.1, 7.5], device=DEV)
    for b in range(k // 32):
        x[:, 32 * b] = 7.0                            # fixes the block's scale
        x[:, 32 * b + 1: 32 * b + 1 + 22] = steps * (-1.0) ** b * 2.0 ** (0 if b < 2 else -3 * b)
        x[:, 32 * b] *= 2.0 ** (0 if b < 2 else -3 * b)
    x = (x * torch.exp2(torch.arange(n, device=DEV))[:, None]).to(T[dtype])
    want = _quantised64(x)
    w = B.regenvc_mxfp4_quantize(torch.eye(k, device=DEV))
    assert torch.equal(B.regenvc_mxfp4_linear(x, w, k).double(), want)
    assert torch.equal(B.regenvc_mxfp4_project(B.regenvc_mxfp4_quantize(x), w, n, k, k).double(), want)
