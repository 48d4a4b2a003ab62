"""Rows at the ends of what fp32 statistics hold: sums of squares past its range, and rows of one value whose sums are not
exact.  Bounds as in the norm's own tests."""
import pytest
import torch

from block_ops_util import U, half_step, rows_of
from paper_2607_28144_b200 import binding as B
from test_gpu_block_norm import DEV, EPS, T, _backward_check, _check, _forward_check, _grads, _inputs

pytestmark = pytest.mark.gpu


def _parts(c, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    return r, {"weight": 1 + 0.2 * r(c), "bias": 0.2 * r(c), "scale": 0.3 * r(1, c), "shift": 0.3 * r(1, c)}


@pytest.mark.parametrize("c", [200, 1531, 1536, 8192])
@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("norm", [1, 2])
def test_rows_whose_squares_pass_the_range_of_fp32(c, dt, norm):
    """Their deviation is infinite in fp32: they normalise to 0 (not to NaN), let no gradient through the norm, and leave the
    other rows and the sums over rows alone."""
    r, p = _parts(c, c + norm)
    big, rest = [0, 2, 5], [1, 3, 4]
    x = r(6, c)
    x[0] *= 1e20
    x[2] *= 1e30
    x[4] *= 1e15
    x[5] = 1e25 * torch.sign(x[5])
    x = x.to(T[dt])
    _, h = B.regenvc_block_norm_forward(x, **p, norm=norm, eps=EPS)
    pd = {k: v.double() for k, v in p.items()}
    want = (pd["bias"] * (1 + pd["scale"]) + pd["shift"]).expand(3, c)
    bound = half_step(T[dt]) * want.abs() + 6 * U * (pd["bias"].abs() * (1 + pd["scale"].abs()) + pd["shift"].abs())
    _check(h[big], want, bound, "rows of infinite deviation")
    _forward_check(x[rest], None, p, norm, 0, 1.0, 3, None, h[rest])
    # behind a branch: the residual stream goes on as it was
    z = r(6, c).to(T[dt])
    x_out, _ = B.regenvc_block_norm_forward(z, x, norm=0, post_norm=norm, post_eps=EPS)
    assert torch.equal(x_out[big], z[big])
    # gradients
    dh, more = r(6, c).to(T[dt]), r(6, c).to(T[dt])
    got = B.regenvc_block_norm_backward(dh, x, dx_out=more, **p, norm=norm, eps=EPS)
    assert torch.equal(got["dx"][big], more[big])
    plain, dh0 = x.clone(), dh.clone()
    plain[big], dh0[big] = 1, 0                    # rows that have no part in the sum over tokens
    plain[big, ::2] = -1
    alone = B.regenvc_block_norm_backward(dh0, plain, dx_out=more, **p, norm=norm, eps=EPS)
    assert torch.equal(got["dweight"], alone["dweight"]) and torch.equal(got["dx"][rest], alone["dx"][rest])
    assert all(torch.isfinite(v).all() for v in got.values() if v is not None)
    got = B.regenvc_block_norm_backward(None, None, dx_out=more, y=x, norm=0, post_norm=norm, post_eps=EPS)
    assert (got["dy"][big] == 0).all() and torch.isfinite(got["dy"]).all() and torch.equal(got["dx"], more)


def test_an_infinity_beside_finite_values():
    """RMS norm: the infinity itself has no value (inf / inf), the finite values of its row are 0."""
    for c in (96, 1531, 5120):
        x = torch.randn(3, c, device=DEV, generator=torch.Generator(device=DEV).manual_seed(c))
        x[1, 7] = float("inf")
        _, h = B.regenvc_block_norm_forward(x, norm=2, eps=EPS)
        others = torch.arange(c, device=DEV) != 7
        assert torch.isnan(h[1, 7]) and (h[1, others] == 0).all()
        _forward_check(x[[0, 2]], None, {}, 2, 0, 1.0, 2, None, h[[0, 2]])


VALUES = [12345.678, 1000.1, 1e18, 3e-3, -77777.77, 0.1, 1e-20, 3.0]


def _constant(c, dtype):
    return torch.tensor(VALUES, device=DEV).to(dtype)[:, None].expand(-1, c).contiguous()


@pytest.mark.parametrize("c", [7, 96, 200, 1000, 1531, 1536, 2056, 5120, 8191])
@pytest.mark.parametrize("xt,iot", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("fp16", "fp16")])
def test_rows_of_one_value_normalise_to_zero(c, xt, iot):
    """Layer norm of a row whose fp32 sum is not exact: the mean's error is known after the centred values' sum and goes
    out again, so the result is 0 and not that error times 1 / sqrt(eps)."""
    n = len(VALUES)
    x = _constant(c, T[xt])
    x[~torch.isfinite(x)] = 3.0                                    # (fp16's range)
    _, h = B.regenvc_block_norm_forward(x, norm=1, eps=EPS)
    assert (h == 0).all()
    # x' of one value: a product and a sum with all of fp32's bits, whatever the types
    y, gate = torch.full((n, c), 0.3, device=DEV).to(T[iot]), torch.full((1, c), 1.7, device=DEV)
    _, h = B.regenvc_block_norm_forward(x, y, gate=gate, norm=1, eps=EPS)
    assert (h == 0).all()
    # as the branch's own norm
    yc = _constant(c, T[iot])
    yc[~torch.isfinite(yc)] = 3.0
    z = torch.randn(n, c, device=DEV, generator=torch.Generator(device=DEV).manual_seed(c)).to(T[xt])
    x_out, _ = B.regenvc_block_norm_forward(z, yc, norm=0, post_norm=1, post_eps=EPS)
    assert torch.equal(x_out, z)


@pytest.mark.parametrize("c", [7, 200, 1531, 1536, 5120, 8191])
@pytest.mark.parametrize("xt,iot", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")])
def test_gradients_of_rows_of_one_value(c, xt, iot):
    """xhat = 0: no gradient of the weights, and d - mean(d) times 1 / sqrt(eps) for the row itself."""
    r, p = _parts(c, c)
    n, x, yc = len(VALUES), _constant(c, T[xt]), _constant(c, T[iot])
    dh, more = r(n, c).to(T[iot]), r(n, c).to(T[xt])
    p = {"weight": p["weight"], "scale": p["scale"], "shift": p["shift"]}
    got = B.regenvc_block_norm_backward(dh, x, **p, norm=1, eps=EPS)
    assert (got["dweight"] == 0).all() and (got["dscale"] == 0).all()
    d = dh.double() * p["weight"].double() * (1 + p["scale"].double())
    ref, top = (d - d.mean(1, keepdim=True)) / EPS ** 0.5, d.abs().amax(1, keepdim=True) / EPS ** 0.5
    _check(got["dx"], ref, half_step(T[xt]) * ref.abs() + 64 * U * top * 4, "dx")
    pw, gate = 1 + 0.2 * r(c), r(1, c)
    got = B.regenvc_block_norm_backward(None, None, dx_out=more, y=yc, gate=gate, post_weight=pw, norm=0, post_norm=1, post_eps=EPS)
    assert (got["dgate"] == 0).all() and (got["dpost_weight"] == 0).all()
    d = more.double() * gate.double() * pw.double()
    ref, top = (d - d.mean(1, keepdim=True)) / EPS ** 0.5, d.abs().amax(1, keepdim=True) / EPS ** 0.5
    _check(got["dy"], ref, half_step(T[iot]) * ref.abs() + 64 * U * top * 4, "dy")


@pytest.mark.parametrize("c", [200, 1531, 1536, 5120])
def test_rows_that_differ_by_single_bits(c):
    """Values of 12345.678 and up to two units in the last place around.  Centred values are exact; the mean's first error is
    at most 24 u of the mean, 18 ulp, against a deviation of 1.4 ulp, so r loses 14 u (1 + 18^2 / 2), and the rest is the
    ordinary 64 u T with T = 2 max|v - mean| r."""
    g = torch.Generator(device=DEV).manual_seed(c)
    x = torch.full((5, c), 12345.678, device=DEV) + 2.0 ** -10 * torch.randint(-2, 3, (5, c), generator=g, device=DEV)
    _, h = B.regenvc_block_norm_forward(x, norm=1, eps=0.0)
    d = x.double() - x.double().mean(1, keepdim=True)
    ref = d * torch.rsqrt((d * d).mean(1, keepdim=True))
    t = 2 * ref.abs().amax(1, keepdim=True)
    _check(h, ref, (64 + 14 * 163) * U * t, "h")
    # gradient: dx = r (dh - mean(dh) - xhat mean(dh xhat)), the same loss in r and xhat
    dh = torch.randn(5, c, generator=g, device=DEV)
    got = B.regenvc_block_norm_backward(dh, x, norm=1, eps=0.0)["dx"]
    r, dd = torch.rsqrt((d * d).mean(1, keepdim=True)), dh.double()
    want = r * (dd - dd.mean(1, keepdim=True) - ref * (dd * ref).mean(1, keepdim=True))
    _check(got, want, (64 + 14 * 163) * U * dd.abs().amax(1, keepdim=True) * r * (2 + t) ** 2, "dx")


@pytest.mark.parametrize("n,c,per", [(50, 256, 20), (33, 1531, 33), (300, 1536, 1)])
@pytest.mark.parametrize("xt,iot", [("bf16", "bf16"), ("fp32", "fp16")])
def test_a_weight_of_the_branch_without_a_norm_of_it(n, c, per, xt, iot):
    """z = y post_weight, a scale per channel, and its gradients."""
    x, y, p, r = _inputs(n, c, per, n + c, T[xt], T[iot], True, True, 0, True, True)
    p["post_weight"] = 1 + 0.2 * r(c)
    x_out, h = B.regenvc_block_norm_forward(x, y, **p, norm=1, eps=EPS, residual_scale=0.5, tokens_per_mod=per)
    _forward_check(x, y, p, 1, 0, 0.5, per, x_out, h)
    dh, more = r(n, c).to(T[iot]), r(n, c).to(T[xt])
    got = _grads(x_out, y, dh, more, p, 1, 0, 0.5, per)
    _backward_check(x_out, y, dh, more, p, 1, 0, 0.5, per, got)
    # dpost_weight (not among those checks without a norm): the sum of gate dx' y.  dx' is dx / 0.5 and carries its rounding;
    # 256 + n additions and two products
    dx, g = got["dx"].double() / 0.5, rows_of(p["gate"].double(), per, n)
    terms = (g * dx * y.double()).abs().sum(0)
    _check(got["dpost_weight"], (g * dx * y.double()).sum(0), (half_step(T[xt]) + (n + 256 + 4) * U) * terms, "dpost_weight")
