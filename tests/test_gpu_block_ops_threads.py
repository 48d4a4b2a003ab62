"""Operators around a block's attention called from two host threads at a time, at sizes that share a build of a kernel but
want different amounts of shared memory.  The C entry points are called without the binding, so that the threads spend their
time inside the library."""
import ctypes
import threading

import pytest
import torch

from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
CALLS = 3000


def _norm_forward(c, xt, iot, stream, g):
    n = 300                                     # more rows than SMs: the grid comes from the occupancy
    x, y = torch.randn(n, c, generator=g, device=DEV).to(T[xt]), torch.randn(n, c, generator=g, device=DEV).to(T[iot])
    xo, h = torch.empty_like(x), torch.empty_like(y)
    d = B.BlockNormDesc(n, c, n, B.TYPES[T[xt]], B.TYPES[T[iot]], 1, 2, 1e-6, 1e-6, 1.0)
    args = (ctypes.byref(d), x.data_ptr(), y.data_ptr(), None, None, None, None, None, None, xo.data_ptr(), h.data_ptr(), stream)
    return B.lib().regenvc_block_norm_forward, args, (xo, h), (d, x, y)


def _norm_backward(c, xt, iot, stream, g):
    n = 300
    x, dx_out = (torch.randn(n, c, generator=g, device=DEV).to(T[xt]) for _ in range(2))
    y, dh = (torch.randn(n, c, generator=g, device=DEV).to(T[iot]) for _ in range(2))
    w = torch.ones(c, device=DEV)
    dx, dy, dw = torch.empty_like(x), torch.empty_like(y), torch.empty_like(w)
    size = B.regenvc_block_norm_workspace_bytes(n, c)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    d = B.BlockNormDesc(n, c, n, B.TYPES[T[xt]], B.TYPES[T[iot]], 1, 2, 1e-6, 1e-6, 1.0)
    args = (ctypes.byref(d), x.data_ptr(), y.data_ptr(), None, None, w.data_ptr(), None, None, dh.data_ptr(), dx_out.data_ptr(),
            dx.data_ptr(), dy.data_ptr(), None, None, dw.data_ptr(), None, None, None, ws.data_ptr(), size, stream)
    return B.lib().regenvc_block_norm_backward, args, (dx, dy, dw), (d, x, dx_out, y, dh, w, ws)


def _linear(cols, tokens, _, stream, g):
    f = 64
    x, w = torch.randn(tokens, cols, generator=g, device=DEV), torch.randn(f, cols, generator=g, device=DEV)
    wp = B.regenvc_mxfp4_quantize(w)
    y = torch.empty((tokens, f), dtype=torch.bfloat16, device=DEV)
    assert B.regenvc_mxfp4_linear_scratch_bytes(tokens, f, cols) == 0
    args = (x.data_ptr(), B.TYPES[x.dtype], 0, wp.data_ptr(), None, y.data_ptr(), 0, tokens, f, cols, None, stream)
    return B.lib().regenvc_mxfp4_linear, args, (y,), (x, wp)


def _two_threads(make, a, b, first, second):
    """Both calls alternate freely on a stream each: every call succeeds, and the results are those of the call alone."""
    jobs, want = [], []
    for i, size in enumerate((a, b)):
        stream = torch.cuda.Stream()
        call, args, out, keep = make(size, first, second, ctypes.c_void_p(stream.cuda_stream), torch.Generator(device=DEV).manual_seed(i))
        torch.cuda.synchronize()
        assert call(*args) == B.OK
        torch.cuda.synchronize()
        want.append([t.clone() for t in out])
        jobs.append((call, args, out, keep, stream))
    refused, start = [0, 0], threading.Barrier(2)

    def work(i):
        call, args = jobs[i][:2]
        start.wait()
        for k in range(CALLS):
            refused[i] += call(*args) != B.OK
            if k % 64 == 63:
                jobs[i][4].synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert refused == [0, 0], f"calls refused: {refused} of {CALLS} each"
    for job, alone in zip(jobs, want):
        assert all(torch.equal(got, ref) for got, ref in zip(job[2], alone))


@pytest.mark.parametrize("make,a,b,xt,iot", [
    (_norm_backward, 2560, 5120, "bf16", "bf16"), (_norm_backward, 1531, 2047, "bf16", "bf16"),
    (_norm_backward, 2560, 5120, "fp32", "fp32"), (_norm_forward, 2560, 5120, "fp32", "bf16"),
    (_norm_forward, 2056, 4096, "fp32", "fp32"), (_norm_forward, 6001, 8191, "fp16", "fp16")])
def test_block_norm_of_two_widths(make, a, b, xt, iot):
    _two_threads(make, a, b, xt, iot)


@pytest.mark.parametrize("tokens,a,b", [(1, 30080, 80640), (4, 8192, 20096)])
def test_4_bit_product_of_few_tokens_of_two_inner_extents(tokens, a, b):
    _two_threads(_linear, a, b, tokens, None)
