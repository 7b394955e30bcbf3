"""The gated activation and its gradient where exp(g) lies below what a normal fp32 number holds, and the factors beside it are
large enough that the results do not."""
import pytest
import torch

import operator_reference as R

pytestmark = pytest.mark.gpu

BF16, F32 = R.BF16, R.F32
# A result below 2^-126 is off by half of the smallest bf16, 2^-134, and each of its products in fp32 by 2^-150 at most, with
# factors of no more than 1.1 behind them.
LEAST = 2.0 ** -134 + 2.0 ** -147


def close(got, want, relative, what):
    R.assert_close(got, want, BF16 * want.abs() + (1 + BF16) * F32 * relative + LEAST, what)


def gates():
    """Every bf16 from -262 to -60, and some around 0: [n, 1]."""
    g = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    g = g[(g >= -262) & (g <= -60)]
    near = torch.tensor([-50.0, -20.0, -3.0, -1.28125, -1e-3, -0.0, 0.0, 1e-30, 0.5, 4.0, 30.0, 90.0, 200.0]).bfloat16()
    return torch.cat([g, near])[:, None].cuda()


def rows(g, *others):
    """The gates beside every pair of the other values: [n, len], one tensor for each."""
    return [t.contiguous() for t in torch.broadcast_tensors(g, *(torch.tensor(o).bfloat16().cuda()[None] for o in others))]


# With e = exp(-|g|) and s = 1 / (1 + e) or e / (1 + e): the exponent's argument is a product with a constant, off by 2 F32 of it; a power
# of 2 by a step (2 F32), three of them multiplied (8 F32), the sum and the reciprocal by 3 F32 and e's own part: s by
# (3 |g| + 16) F32 of it. Five products more.
@pytest.mark.parametrize("scale", [1.5, 1e-3, 3e10, -7e20, 1.3e38])
def test_faint_gates(tw, scale):
    g, u = rows(gates(), [scale * f for f in (1.0, 0.37, -0.011, 2.3, 1e-4, -0.9, 1.7, 0.5)])
    x = torch.cat([g, u], 1)
    out = tw.gated_silu(x)
    gd, ud = g.double(), u.double()
    want = gd * torch.sigmoid(gd) * ud
    fits = want.abs() < 2.0 ** 127
    assert int((fits & (gd < -87.5) & (want.abs() > 2.0 ** -126)).sum()) > 0 or abs(scale) < 1
    close(torch.where(fits, out, 0.0), torch.where(fits, want, 0.0), torch.where(fits, (3 * gd.abs() + 24) * want.abs(), 0.0), "gate")


# Of dout u s (1 + g (1 - s)), 1 - s is off like s; dout u, which overflows by itself, by F32.
@pytest.mark.parametrize("d_scale,u_scale", [(1.0, 1.5), (1e-3, 3e10), (1e19, 6e18), (1.2e38, 0.9), (2e-3, 1.2e38), (-3e30, -7e6)])
def test_gradients_of_faint_gates(tw, d_scale, u_scale):
    g, u, d = rows(gates(), [u_scale * f for f in (1.0, 0.37, -0.011, 0.9, 1e-4, -0.8, 1.1, 0.5)], [d_scale * f for f in (0.6, -1.0, 0.3, 1e-5, 1.1, 0.2, 0.7, -0.04)])
    dx = tw.gated_silu_backward(d, torch.cat([g, u], 1))
    gd, ud, dd = g.double(), u.double(), d.double()
    s = torch.sigmoid(gd)
    dg, du, slope = dd * ud * (s + gd * s * (1 - s)), dd * gd * s, s * (1 + gd.abs() * (1 - s))
    assert bool(((dd * ud).abs() < 2.0 ** 127).all())
    fits = du.abs() < 2.0 ** 127
    close(dx[:, :8], dg, (6 * gd.abs() + 56) * (dd * ud).abs() * slope, "gradient of the gates")
    close(torch.where(fits, dx[:, 8:], 0.0), torch.where(fits, du, 0.0), torch.where(fits, (3 * gd.abs() + 24) * du.abs(), 0.0), "gradient of the values")
    assert int(((gd < -87.5) & (dg.abs() > 2.0 ** -126)).sum()) > 0 or abs(d_scale * u_scale) < 10
