"""Norms fused with gate and residual scale, forward and gradients, against the 64-bit form and its automatic gradient.

Bounds.  u = 2^-24.  A sum over a row has at most 8 + 5 + 10 fp32 additions in sequence, so a mean is off by at most 24 u of
the row's mean magnitude, a squared deviation's mean by 28 u, r = 1 / sqrt by half of that and 2 ulp: with T = 2 max|v| r
a normalised value is off by at most 64 u T (it is at most T itself).  Each bound below carries that through the formula by
magnitudes and adds half a step of the result's type."""
import pytest
import torch

from block_ops_util import U, block_norm64, floor_step, half_step, norm64, rows_of
from paper_2607_28144_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6
T = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
GUARD = 64


def _guarded(n, c, dtype, stride=None):
    """An [n, c] tensor inside a NaN-filled buffer, `stride` elements between rows, and a check that nothing else of the
    buffer was written."""
    stride = stride or c
    buf = torch.full((n * stride + 2 * GUARD,), float("nan"), dtype=dtype, device=DEV)
    t = torch.as_strided(buf, (n, c), (stride, 1), GUARD)

    def check():
        rest = torch.ones_like(buf, dtype=torch.bool)
        torch.as_strided(rest, (n, c), (stride, 1), GUARD).fill_(False)
        assert torch.isnan(buf[rest]).all(), "wrote outside the result"
        assert torch.isfinite(t).all(), "left part of the result unwritten"

    return t, check


def _rows(t, stride):
    out = torch.empty((t.shape[0], stride), dtype=t.dtype, device=DEV)[:, : t.shape[1]]
    out.copy_(t)
    return out


def _inputs(n, c, per, seed, xt, iot, residual, gate, post, affine, mod, extra=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    x = _rows((r(n, c) * (1 + 3 * torch.rand(c, generator=g, device=DEV)) + 0.5).to(xt), c + extra)
    y = _rows(r(n, c).to(iot), c + extra) if residual else None
    mods = -(-n // per)
    six = 0.3 * r(mods, 6, c)
    p = {}
    if gate and residual:
        p["gate"] = six[:, 2]
    if mod:
        p["scale"], p["shift"] = six[:, 1], six[:, 0]
    if affine:
        p["weight"], p["bias"] = 1 + 0.2 * r(c), 0.2 * r(c)
    if post and residual:
        p["post_weight"] = 1 + 0.2 * r(c)
    return x, y, p, r


def _double(p):
    return {k: v.double() for k, v in p.items()}


def _scale_of(v, kind, eps=EPS):
    """r of a row, and T = 2 max|v| r."""
    d = v - v.mean(1, keepdim=True) if kind == 1 else v
    r = torch.rsqrt((d * d).mean(1, keepdim=True) + eps)
    return r, 2 * v.abs().amax(1, keepdim=True) * r


def _check(got, ref, bound, what):
    assert torch.isfinite(got).all(), what
    err = (got.double() - ref).abs()
    worst = (err / bound.clamp_min(1e-300)).max().item()
    assert (err <= bound).all(), f"{what}: {worst:.3g} times its bound"


def _forward_check(x, y, p, norm, post, alpha, per, x_out, h):
    pd = _double(p)
    xd, yd = x.double(), None if y is None else y.double()
    n = x.shape[0]
    rx, rh = block_norm64(xd, yd, pd, norm, post, alpha, per, EPS)
    mag = xd.abs()
    if y is not None:
        z = _scale_of(yd, post)[1].expand_as(yd) if post else yd.abs()
        for k in ("post_weight", "gate"):
            if k in pd:
                z = z * (rows_of(pd[k], per, n) if k == "gate" else pd[k]).abs()
        mag = abs(alpha) * mag + z
        _check(x_out, rx, half_step(x_out.dtype) * rx.abs() + 70 * U * mag + floor_step(x_out.dtype), "x_out")
    if not norm:
        assert h is None
        return
    r, _ = _scale_of(rx, norm)
    t = 2 * mag.amax(1, keepdim=True) * r
    w = pd.get("weight", torch.ones((), device=DEV, dtype=torch.float64)).abs()
    b = pd["bias"].abs() if "bias" in pd else 0.0
    s = 1 + rows_of(pd["scale"], per, n).abs() if "scale" in pd else 1.0
    sh = rows_of(pd["shift"], per, n).abs() if "shift" in pd else 0.0
    _check(h, rh, half_step(h.dtype) * rh.abs() + (70 + 64 + 6) * U * t * w * s + 6 * U * (b * s + sh) + floor_step(h.dtype), "h")


TYPES = [("bf16", "bf16"), ("fp16", "fp16"), ("fp32", "fp32"), ("fp32", "bf16"), ("fp32", "fp16")]
# n, c, tokens per modulation row: single elements, widths off every vector size, the widest row, modulation rows that
# begin and end inside, at, and across the ranges of thread blocks (2000 rows: four per block)
SHAPES = [(1, 1, 1), (1, 1536, 1), (3, 7, 2), (5, 100, 5), (129, 1000, 43), (33, 1531, 7), (2000, 64, 2000), (2000, 64, 613),
          (2001, 64, 4), (2003, 40, 3), (700, 64, 1), (301, 2056, 100), (200, 5120, 200), (37, 8192, 10), (20, 8191, 20)]


@pytest.mark.parametrize("n,c,per", SHAPES)
@pytest.mark.parametrize("xt,iot", TYPES)
def test_forward(n, c, per, xt, iot):
    for i, (norm, post, alpha, affine, mod, gate) in enumerate([(1, 0, 1.0, False, True, True), (2, 2, 0.5, True, True, True),
                                                                (1, 1, 1.0, True, False, False)]):
        x, y, p, _ = _inputs(n, c, per, 10 * n + c + i, T[xt], T[iot], True, gate, post, affine, mod)
        xo, check_x = _guarded(n, c, T[xt])
        h, check_h = _guarded(n, c, T[iot])
        B.regenvc_block_norm_forward(x, y, **p, norm=norm, post_norm=post, residual_scale=alpha, eps=EPS, post_eps=EPS,
                                     tokens_per_mod=per, x_out=xo, h=h)
        check_x()
        check_h()
        _forward_check(x, y, p, norm, post, alpha, per, xo, h)


@pytest.mark.parametrize("n,c,extra", [(9, 64, 8), (9, 64, 5), (300, 1536, 8), (300, 1536, 3), (50, 100, 4)])
def test_forward_of_strided_rows_in_place_and_without_parts(n, c, extra):
    x, y, p, _ = _inputs(n, c, 4, n + c, torch.bfloat16, torch.bfloat16, True, True, 2, True, True, extra)
    kw = dict(norm=1, post_norm=2, eps=EPS, post_eps=EPS, tokens_per_mod=4)
    xo, check_x = _guarded(n, c, torch.bfloat16, c + 2 * extra)
    h, check_h = _guarded(n, c, torch.bfloat16, c + extra)
    B.regenvc_block_norm_forward(x, y, **p, **kw, x_out=xo, h=h)
    check_x()
    check_h()
    _forward_check(x, y, p, 1, 2, 1.0, 4, xo, h)
    # in place on x; rows between the views keep what they hold
    x2 = _rows(x, c + extra)
    a, b = B.regenvc_block_norm_forward(x2, y, **p, **kw, x_out=x2)
    assert a is x2 and torch.equal(x2, xo) and torch.equal(b, h)
    # only the residual step; only the norm
    only_x, none = B.regenvc_block_norm_forward(x, y, gate=p["gate"], post_weight=p["post_weight"], norm=B.NORM_NONE, post_norm=2,
                                                post_eps=EPS, tokens_per_mod=4)
    assert none is None and torch.equal(only_x, xo)
    none, only_h = B.regenvc_block_norm_forward(x, norm=2, weight=p["weight"], eps=EPS)
    assert none is None
    _forward_check(x, None, {"weight": p["weight"]}, 2, 0, 1.0, n, None, only_h)
    # h without x_out: through the C entry (the binding always returns x_out)
    import ctypes
    d = B.BlockNormDesc(n, c, 4, 0, 0, 1, 2, EPS, EPS, 1.0, p["gate"].stride(0), x.stride(0), y.stride(0), 0, 0)
    h2 = torch.empty((n, c), dtype=torch.bfloat16, device=DEV)
    B._check(B.lib().regenvc_block_norm_forward(ctypes.byref(d), x.data_ptr(), y.data_ptr(), p["gate"].data_ptr(),
                                                p["post_weight"].data_ptr(), p["weight"].data_ptr(), p["bias"].data_ptr(),
                                                p["scale"].data_ptr(), p["shift"].data_ptr(), None, h2.data_ptr(),
                                                torch.cuda.current_stream().cuda_stream))
    assert torch.equal(h2, h)


def test_rows_of_one_value_large_means_zeros_and_nan():
    n, c = 8, 1536
    x = torch.zeros((n, c), dtype=torch.float32, device=DEV)
    x[1] = 3.0                                       # constant: layer norm gives exactly 0
    x[2] = 1000.0 + torch.randn(c, device=DEV, generator=torch.Generator(device=DEV).manual_seed(3))
    x[4, 7] = float("nan")
    x[5, 9] = float("inf")
    x[6] = 1e18
    _, h = B.regenvc_block_norm_forward(x, norm=1, eps=EPS)
    assert torch.equal(h[0], torch.zeros_like(h[0])) and torch.equal(h[1], torch.zeros_like(h[1]))
    assert torch.equal(h[3], torch.zeros_like(h[3])) and torch.equal(h[7], torch.zeros_like(h[7]))
    ref = norm64(x[2:3].double(), 1, EPS)
    t = _scale_of(x[2:3].double(), 1)[1]
    _check(h[2:3], ref, 64 * U * t + U * ref.abs(), "a mean of 1000 deviations")
    assert torch.isnan(h[4]).all() and torch.isnan(h[5]).any()   # and no other row saw them
    assert torch.isfinite(h[[0, 1, 2, 3, 7]]).all()


def _backward_check(x, y, dh, dxo, p, norm, post, alpha, per, got):
    n, c = x.shape
    pd = {k: v.double().requires_grad_() for k, v in p.items()}
    xd = x.double().requires_grad_()
    yd = None if y is None else y.double().requires_grad_()
    bare = {k: v for k, v in pd.items() if k not in ("gate", "post_weight")}
    dxp = torch.zeros_like(xd) if dxo is None else dxo.double()
    if norm:
        _, h = block_norm64(xd, None, bare, norm, 0, 1.0, per, EPS)
        (h * dh.double()).sum().backward()
        dxp = dxp + xd.grad
    if y is not None:
        t, _ = block_norm64(torch.zeros_like(xd), yd, {k: v for k, v in pd.items() if k in ("gate", "post_weight")}, 0, post, 0.0,
                            per, EPS)
        (t * dxp).sum().backward()
    a = {k: v.detach().abs() for k, v in pd.items()}
    one = torch.ones((), dtype=torch.float64, device=DEV)
    s1 = (1 + rows_of(pd["scale"].detach(), per, n)).abs() if "scale" in a else one
    # dx'
    err = torch.zeros_like(dxp)
    if norm:
        r, t = _scale_of(x.double(), norm)
        dha = dh.double().abs()
        d = (dha * s1 * a.get("weight", one)).amax(1, keepdim=True)
        err = 64 * U * d * r * (2 + t) ** 2 + 2 * U * dxp.abs()
    if dxo is not None:
        err = err + 2 * U * dxo.double().abs()
    err = err.expand_as(dxp)
    al = alpha if y is not None else 1.0
    _check(got["dx"], al * dxp.detach(),
           half_step(x.dtype) * (al * dxp).abs() + abs(al) * (err + 2 * U * dxp.abs()) + floor_step(x.dtype), "dx")
    sums = lambda v: torch.zeros((-(-n // per), c), dtype=torch.float64, device=DEV).index_add_(  # noqa: E731
        0, torch.arange(n, device=DEV) // per, v)
    k = (n + 256) * U
    if norm:
        w, b = a.get("weight", one), a.get("bias", 0.0 * one)
        if "scale" in p:
            _check(got["dscale"], pd["scale"].grad, k * sums(dha * (t * w + b)), "dscale")
            _check(got["dshift"], pd["shift"].grad, k * sums(dha) + 1e-300, "dshift")
        if "weight" in p:
            _check(got["dweight"], pd["weight"].grad, k * (dha * s1 * t).sum(0), "dweight")
            _check(got["dbias"], pd["bias"].grad, k * (dha * s1).sum(0), "dbias")
    if y is None:
        assert got["dy"] is None
        return
    gate = rows_of(a["gate"], per, n) if "gate" in a else one
    pw = a.get("post_weight", one)
    ry, ty = _scale_of(y.double(), post) if post else (one, y.double().abs())
    if "gate" in p:
        _check(got["dgate"], pd["gate"].grad, sums(pw * ty * (err + k * dxp.abs())), "dgate")
    if post:
        _check(got["dpost_weight"], pd["post_weight"].grad, (gate * ty * (err + k * dxp.abs())).sum(0), "dpost_weight")
    ez = gate * pw * (err + 4 * U * dxp.abs())
    if post:
        dz = (gate * pw * dxp.abs()).amax(1, keepdim=True)
        ez = ry * (2 + ty) * ez.amax(1, keepdim=True) + 64 * U * dz * ry * (2 + ty) ** 2
    ref = yd.grad
    _check(got["dy"], ref, half_step(y.dtype) * ref.abs() + ez + floor_step(y.dtype), "dy")


def _grads(x, y, dh, dxo, p, norm, post, alpha, per, **kw):
    return B.regenvc_block_norm_backward(dh, x, dx_out=dxo, y=y, **p, norm=norm, post_norm=post, residual_scale=alpha, eps=EPS,
                                         post_eps=EPS, tokens_per_mod=per, **kw)


@pytest.mark.parametrize("n,c,per", SHAPES)
@pytest.mark.parametrize("xt,iot", TYPES)
def test_backward(n, c, per, xt, iot):
    for i, (norm, post, alpha, affine, mod, gate, res) in enumerate([
            (1, 0, 1.0, False, True, True, True), (2, 2, 0.5, True, True, True, True), (1, 1, 1.0, True, False, False, True),
            (1, 0, 1.0, True, True, False, False)]):
        x, y, p, r = _inputs(n, c, per, 20 * n + c + i, T[xt], T[iot], res, gate, post, affine, mod)
        dh = r(n, c).to(T[iot])
        dxo = r(n, c).to(T[xt]) if res else None
        got = _grads(x, y, dh, dxo, p, norm, post, alpha, per)
        _backward_check(x, y, dh, dxo, p, norm, post, alpha, per, got)
        again = _grads(x, y, dh, dxo, p, norm, post, alpha, per)
        for k in got:
            assert got[k] is None or torch.equal(got[k], again[k]), f"{k}: two calls differ"


def test_backward_of_strided_rows_in_place_and_without_parts():
    n, c, per = 300, 200, 50
    x, y, p, r = _inputs(n, c, per, 5, torch.float32, torch.bfloat16, True, True, 2, True, True, 12)
    dh, dxo = _rows(r(n, c).bfloat16(), c + 7), _rows(r(n, c), c + 5)
    got = _grads(x, y, dh, dxo, p, 1, 2, 1.0, per)
    _backward_check(x, y, dh, dxo, p, 1, 2, 1.0, per, got)
    buf = _rows(dxo, c + 5)
    again = _grads(x, y, dh, buf, p, 1, 2, 1.0, per, dx=buf)
    assert again["dx"] is buf
    for k in got:
        assert torch.equal(got[k], again[k]), k
    # the residual step alone (no norm behind it), and no gradient from the residual stream
    some = {k: p[k] for k in ("gate", "post_weight")}
    got = B.regenvc_block_norm_backward(None, None, dx_out=dxo, y=y, **some, norm=0, post_norm=2, post_eps=EPS, tokens_per_mod=per)
    _backward_check(x, y, None, dxo, some, 0, 2, 1.0, per, got)
    got = _grads(x, y, dh, None, p, 2, 2, 1.0, per)
    _backward_check(x, y, dh, None, p, 2, 2, 1.0, per, got)


def test_gradients_against_differences():
    """<gradient, direction> from the kernel against the difference quotient of the 64-bit form (step 1e-5: truncation and
    rounding below 1e-8 of the terms).  The kernel's inner product is off by at most sum bound * |direction|; all
    operands fp32, so that is 1e-4 of sum |gradient| |direction| for these well-scaled rows (T < 10: 64 u (2 + T)^2 =
    5.5e-4 of a gradient's largest value in the worst case, taken here as the relative bound)."""
    n, c, per = 64, 96, 16
    x, y, p, r = _inputs(n, c, per, 9, torch.float32, torch.float32, True, True, 2, True, True)
    dh, dxo = r(n, c), r(n, c)
    # the function whose gradient is asked for, at the x' the forward pass saves
    x_out, _ = B.regenvc_block_norm_forward(x, y, **p, norm=1, post_norm=2, residual_scale=0.5, eps=EPS, post_eps=EPS, tokens_per_mod=per)
    got = _grads(x_out, y, dh, dxo, p, 1, 2, 0.5, per)
    leaves = {"x": x.double(), "y": y.double(), **_double(p)}
    # x_out is x' rounded to fp32: the plain function is shifted to go through exactly that point
    t0, _ = block_norm64(leaves["x"], leaves["y"], leaves, 0, 2, 0.5, per, EPS)
    shift = x_out.double() - t0

    def value(v):
        t, _ = block_norm64(v["x"], v["y"], v, 0, 2, 0.5, per, EPS)
        t = t + shift
        _, h = block_norm64(t, None, {k: v[k] for k in ("weight", "bias", "scale", "shift")}, 1, 0, 1.0, per, EPS)
        return (t * dxo.double()).sum() + (h * dh.double()).sum()

    for k in leaves:
        d = torch.randn(leaves[k].shape, dtype=torch.float64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(4))
        up, down = dict(leaves), dict(leaves)
        up[k], down[k] = leaves[k] + 1e-5 * d, leaves[k] - 1e-5 * d
        quotient = float(value(up) - value(down)) / 2e-5
        g = got["d" + k].double()
        assert abs(float((g * d).sum()) - quotient) <= 5.5e-4 * float(g.abs().max()) * float(d.abs().sum()) ** 0.5 * 4 + 1e-6 * abs(quotient), k


def test_other_streams_captured_graphs_and_eager_gradients_beside_them():
    n, c, per = 500, 256, 100
    x, y, p, r = _inputs(n, c, per, 31, torch.bfloat16, torch.bfloat16, True, True, 0, True, True)
    dh, dxo = r(n, c).bfloat16(), r(n, c).bfloat16()
    fwd = lambda **k: B.regenvc_block_norm_forward(x, y, **p, eps=EPS, tokens_per_mod=per, **k)  # noqa: E731
    want_x, want_h = fwd()
    want = _grads(x, y, dh, dxo, p, 1, 0, 1.0, per)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got_x, got_h = fwd(stream=side)
    got = _grads(x, y, dh, dxo, p, 1, 0, 1.0, per, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got_x, want_x) and torch.equal(got_h, want_h)
    assert all(got[k] is None or torch.equal(got[k], want[k]) for k in want)
    # two graphs of the backward pass, replayed at a time on two streams; an eager graph of the same leaves is alive
    leaf = x.float().requires_grad_()
    alive = (leaf * 2).sum()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            res = (fwd(), _grads(x, y, dh, dxo, p, 1, 0, 1.0, per))
        graphs.append((g, res))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for (g, _), s in zip(graphs, streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for _, ((gx, gh), gb) in graphs:
        assert torch.equal(gx, want_x) and torch.equal(gh, want_h)
        assert all(gb[k] is None or torch.equal(gb[k], want[k]) for k in want)
    alive.backward()
    assert torch.equal(leaf.grad, torch.full_like(leaf, 2.0))


def test_launch_counts_and_refusals_of_the_binding():
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    before = B.regenvc_kernel_launch_count()
    B.regenvc_block_norm_forward(x)
    assert B.regenvc_kernel_launch_count() == before + 1
    B.regenvc_block_norm_backward(x, x, scale=torch.zeros((1, 64), device=DEV))
    assert B.regenvc_kernel_launch_count() in (before + 2, before + 3)
    wide = torch.zeros((1, 64), dtype=torch.bfloat16, device=DEV).expand(4, 64)
    with pytest.raises(ValueError):
        B.regenvc_block_norm_forward(wide)
    with pytest.raises(ValueError):
        B.regenvc_block_norm_forward(x, scale=torch.zeros((1, 64), device=DEV).expand(4, 64), tokens_per_mod=1)
    with pytest.raises(TypeError):
        B.regenvc_block_norm_forward(x, scale=torch.zeros((2, 64), device=DEV))     # one row for all tokens is wanted
    with pytest.raises(TypeError):
        B.regenvc_block_norm_forward(x.t())
    with pytest.raises(B.RegenvcError) as e:
        B.regenvc_block_norm_forward(x, x.float())                                 # y of a type that x does not go with
    assert e.value.code == B.ERR_UNSUPPORTED
    with pytest.raises(B.RegenvcError) as e:
        B.regenvc_block_norm_forward(x, x.clone(), x_out=x, h=x)
    assert e.value.code == B.ERR_ALIASING
    with pytest.raises(B.RegenvcError) as e:
        B.regenvc_block_norm_forward(torch.zeros((2, 8200), device=DEV))
    assert e.value.code == B.ERR_BAD_SHAPE
