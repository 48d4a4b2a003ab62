"""Rows at the ends of what fp32 statistics hold: sums of squares past its range, and rows of one value whose sums are not
exact.  Bounds as in the norm's own tests."""
import pytest
import torch

from block_ops_util import U, half_step
from paper_2607_28144_b200 import binding as B
from test_gpu_block_norm import DEV, EPS, T, _check, _forward_check

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
