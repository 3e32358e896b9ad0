"""The activation functions of the 8-bit activations at large arguments and in relative error, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import act8_reference as ref
import paper_2002_11082_b200 as ogq
from act8_gpu import ACTS, DTYPES, assert_near, half_step, kept, smallest

pytestmark = pytest.mark.gpu


def forward_and_backward(z, dtype, act, cols, up=None, dy=None):
    """y, dx (and dup) of the values z, one in each group (all else 0), whose kept form is z itself; vector kernels for cols = 64, the others for 33."""
    d, dt = DTYPES[dtype]
    a, _ = ACTS[act]
    n = len(z)
    put = lambda v: torch.zeros(n, cols, dtype=dt, device="cuda").index_put_((torch.arange(n, device="cuda"), torch.full((n,), 7, device="cuda")), v.cuda().to(dt))  # noqa: E731
    x, dys = put(z), put(torch.ones(n) if dy is None else dy)
    ups = None if up is None else put(up)
    codes, scales = kept(n, cols)
    up_codes, up_scales = kept(n, cols)
    g = (ups, cols, up_codes.t, up_scales.t) if up is not None else (None, 0, None, None)
    y, dx, dup = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    ogq.ogq_act8_forward(x, cols, g[0], g[1], n, cols, d, a, 0, 0, 0, y, cols, codes.t, scales.t, g[2], g[3])
    ogq.ogq_act8_backward(dys, cols, codes.t, scales.t, g[2], g[3], n, cols, d, a, dx, cols, dup if up is not None else None, cols)
    unit = (scales.t.int() << 23).view(torch.float32)
    assert torch.equal(codes.t[:, 7].float() * unit[:, 0], x[:, 7].float()), "these values have a kept form of their own"
    return y[:, 7], dx[:, 7], dup[:, 7]


LARGE = [32.0, 1000.0, 2.0 ** 16 - 512, 2.0 ** 24, 2.0 ** 25, 127 * 2.0 ** 30, 2.0 ** 100, 2.0 ** 126]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("cols", [64, 33])
def test_slope_of_silu_at_large_arguments(dtype, gated, cols):
    """From z = 32 on the slope is 1 + z exp(-z) < 1 + 2^-40, f(z) = z (1 - 2^-46): to the last bit dx = dy [up] and dup = dy z.  Below -200 both are 0."""
    z = torch.tensor(LARGE + [-1000.0, -2.0 ** 25, -2.0 ** 126])
    dy, up = torch.full((len(z),), 0.75), torch.full((len(z),), -1.5) if gated else None
    _, dx, dup = forward_and_backward(z, dtype, "silu", cols, up, dy)
    n = len(LARGE)
    assert dx[:n].float().tolist() == [0.75 * (-1.5 if gated else 1.0)] * n
    assert not dx[n:].any()
    if gated:
        want = 0.75 * torch.tensor(LARGE).to(DTYPES[dtype][1])
        assert torch.equal(dup[:n].cpu(), want) and not dup[n:].any()


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("P,C,G", [(6, 32, 1), (6, 30, 1), (70000, 32, 4)])
def test_slope_of_silu_behind_a_large_gamma(dtype, P, C, G):
    """z = gamma xh beyond 2^24 in magnitude, whose slope is 0 or 1: dbeta counts the positive ones."""
    d, dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = (torch.randint(0, 2, (P, C), device="cuda", generator=gen) * 2 - 1).to(dt) * 4
    x[0], x[1] = 4, -4
    gamma = torch.full((C,), 2.0 ** 30, device="cuda")
    ws = torch.empty(ogq.ogq_group_norm_workspace_bytes(1, P, C, G), dtype=torch.uint8, device="cuda")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd, dg, db = (torch.empty(n, device="cuda") for n in (G, G, C, C))
    ogq.ogq_group_norm_forward(x, 1, P, C, G, d, gamma, None, 1e-5, ogq.OGQ_ACT_NONE, 0, 0, 0, y, mean, rstd, None, None, ws, ws.numel())
    assert bool((mean.abs() < 3.9).all())
    ogq.ogq_group_norm_backward(torch.ones_like(x), x, None, None, 1, P, C, G, d, gamma, None, ogq.OGQ_ACT_SILU, mean, rstd, dx, dg, db, ws, ws.numel())
    assert torch.equal(db, (x > 0).sum(0).float())


def kept_grid(least, most, per):
    """Values of both signs whose kept form is themselves (at most seven bits), `per` (8 to 64, a power of two) in each power of two."""
    m = torch.arange(64, 128, 64 // per, dtype=torch.float64)
    z = torch.cat([m * 2.0 ** e for e in range(-12, 3)])
    z = z[(z >= least) & (z <= most)]
    return torch.cat([z, -z])


SUBNORMAL = 2.0 ** -149


@pytest.mark.parametrize("cols", [64, 33])
@pytest.mark.parametrize("gated", [False, True])
def test_silu_in_fp32_relative_to_its_value(cols, gated):
    """In half steps of fp32 (2^-24): ex2 is off by 4 at most (2^-22), the correction of its argument, 1 + exp, the product with z and a gate's by one each, rcp by 2
    (one step of 2^-23): 10 of f(z), whatever z.  The slope s + f (1 - s): f by 9 (without the gate), 1 - s = exp s by 5 + 8 + 1, the sum's two roundings are of s + f (1 - s)
    and s is off by 8, the product with dy and a gate's by one each: 27 of |s| + |f (1 - s)|."""
    z = kept_grid(2.0 ** -6, 86.0, 64)
    up = torch.full((len(z),), 1.25) if gated else None
    y, dx, dup = forward_and_backward(z, "f32", "silu", cols, up)
    zn = z.double().numpy()
    f, s = ref.value(ref.SILU, zn), 1 / (1 + np.exp(-zn))
    g = 1.25 if gated else 1.0
    h = 2.0 ** -24
    assert_near(y.double().cpu().numpy(), g * f, 10 * h * g * np.abs(f) + SUBNORMAL, "y")
    assert_near(dx.double().cpu().numpy(), g * ref.slope(ref.SILU, zn), 27 * h * g * (s + np.abs(f) / (1 + np.exp(zn))) + SUBNORMAL, "dx")
    if gated:
        assert_near(dup.double().cpu().numpy(), f, 10 * h * np.abs(f) + SUBNORMAL, "dup")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("cols", [64, 33])
def test_gelu_relative_to_its_value(dtype, cols):
    """Phi(-|z|) is the fit of a function of t = 1 / (1 + p |z|), 1.7e-6 off at most in 16 bits and 1.2e-7 in fp32, times an exponential.  In half steps of fp32: t is
    off by 5 (its factor of |z|, the sum, rcp), which the fitted function takes at most 2.5 times; the polynomial's additions, ex2 and the last products make 15 more;
    the exponential's argument, z^2/2 and in fp32 up to 1.3 more, has been rounded 7 times at most.  So the tail is off by 32 + 7 (z^2/2 + 1.3) half steps and the fit.
    exp(-z^2/2) is taken as 0 where it is below 2^-126 (z beyond 13.2), which the range leaves out.  The slope Phi + z phi: the same of both terms."""
    _, dt = DTYPES[dtype]
    z = kept_grid(2.0 ** -6, 12.5, 64)
    y, dx, _ = forward_and_backward(z, dtype, "gelu", cols)
    zn = z.double().numpy()
    rel = (1.2e-7 if dtype == "f32" else 1.7e-6) + (32 + 7 * (zn ** 2 / 2 + 1.3)) * 2.0 ** -24
    f, phi = ref.value(ref.GELU, zn), np.abs(zn) * np.exp(-zn ** 2 / 2) / np.sqrt(2 * np.pi)
    last, low = half_step(dt) * 1.01, smallest(dt) + SUBNORMAL
    assert_near(y.double().cpu().numpy(), f, (last + rel) * np.abs(f) + low, "y")
    s = ref.slope(ref.GELU, zn)
    assert_near(dx.double().cpu().numpy(), s, last * np.abs(s) + rel * (np.abs(f / zn) + phi) + low, "dx")


@pytest.mark.parametrize("cols", [64, 33])
@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_gate_and_gradient_whose_product_alone_overflows(act, cols):
    """dx = dy f'(x^) up^: where the slope is 0 or tiny, dy up^ alone must not become infinite."""
    z = torch.tensor([-1.0 if act == "relu" else -100.0, -1.0 if act == "relu" else -200.0])
    big = torch.full((2,), 2.0 ** 70)
    _, dx, dup = forward_and_backward(z, "f32", act, cols, big, big)
    assert bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dup).all())
    if act == "relu":
        assert not dx.any()
