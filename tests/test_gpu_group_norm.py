"""Group norm with an activation, channels last, against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import act8_reference as ref
import paper_2002_11082_b200 as ogq
from act8_gpu import ACTS, DTYPES, U24, Guarded, assert_near, half_step, kept, smallest

pytestmark = pytest.mark.gpu
EPS = 1e-5

#        N, P, C, G
SHAPES = [(1, 1, 8, 1), (2, 49, 64, 32), (1, 196, 256, 32), (3, 7, 30, 5), (2, 33, 40, 8), (2, 64, 96, 3), (1, 300, 33, 1), (4, 16, 2048, 32),
          (2, 5, 2056, 8), (1, 2, 4096, 1), (5, 100, 24, 24), (1, 1500, 32, 4), (1, 3000, 128, 8), (2, 257, 320, 32)]


def inputs(N, P, C, dt, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((N, P, C)) * np.exp(0.5 * rng.standard_normal(C)) + rng.standard_normal(C) * 2
    dy = rng.standard_normal((N, P, C)) * 0.3
    gamma, beta = 1 + 0.3 * rng.standard_normal(C), 0.3 * rng.standard_normal(C)
    t = lambda v, d: torch.from_numpy(v).to(d)  # noqa: E731
    return t(x, dt), t(dy, dt), t(gamma, torch.float32), t(beta, torch.float32)


class Call:
    def __init__(self, N, P, C, G, dtype, shift=0):
        self.N, self.P, self.C, self.G, self.shift = N, P, C, G, shift
        self.d, self.dt = DTYPES[dtype]
        self.ws = torch.full((ogq.ogq_group_norm_workspace_bytes(N, P, C, G),), 0xA5, dtype=torch.uint8, device="cuda")
        self.codes, self.scales = kept(N * P, C)

    def guarded(self, data=None):
        return Guarded(self.N * self.P, self.C, self.C, self.dt, self.shift, None if data is None else data.cuda().view(self.N * self.P, self.C))

    def forward(self, x, gamma, beta, act, keep=True, rounding=0, seed=0, stream_id=0, out=None):
        gx = x if isinstance(x, Guarded) else self.guarded(x)
        y = out or self.guarded()
        self.mean, self.rstd = Guarded(self.N, self.G, self.G, torch.float32), Guarded(self.N, self.G, self.G, torch.float32)
        ogq.ogq_group_norm_forward(gx.t, self.N, self.P, self.C, self.G, self.d, gamma, beta, EPS, act, rounding, seed, stream_id, y.t, self.mean.t,
                                   self.rstd.t, self.codes.t if keep else None, self.scales.t if keep else None, self.ws, self.ws.numel())
        for b in (y, self.mean, self.rstd, self.codes, self.scales):
            b.check()
        return y

    def backward(self, dy, x, gamma, beta, act, out=None, want=(True, True)):
        gdy = dy if isinstance(dy, Guarded) else self.guarded(dy)
        gx = None if x is None else self.guarded(x)
        dx = out or self.guarded()
        dg, db = Guarded(1, self.C, self.C, torch.float32), Guarded(1, self.C, self.C, torch.float32)
        ogq.ogq_group_norm_backward(gdy.t, gx.t if gx else None, None if gx else self.codes.t, None if gx else self.scales.t, self.N, self.P, self.C,
                                    self.G, self.d, gamma, beta, act, self.mean.t, self.rstd.t, dx.t, dg.t if want[0] else None, db.t if want[1] else None,
                                    self.ws, self.ws.numel())
        for b in (dx, dg, db):
            b.check()
        return dx, dg, db


def check_forward(c, x, y, gamma, beta, r):
    """A thread sums at most 64 values, rows of threads are at most 256, then 64 bits: the mean is off by less than 400 steps of 2^-24 of
    the largest magnitude (one for each addition of such a chain, and the rounding of the result), the variance by that many of itself
    and twice the mean's error times the deviation; the function's slope is below 1.13."""
    N, P, C, G = c.N, c.P, c.C, c.G
    xn = x.double().numpy()
    mean, rstd = ref.group_stats(xn, G, EPS)
    top = np.abs(xn).reshape(N, P, G, C // G).max(axis=(1, 3))
    d_mean = 400 * U24 * top
    d_rstd = (400 * U24 + d_mean * rstd) * rstd
    assert_near(c.mean.numpy(), mean, d_mean, "mean")
    assert_near(c.rstd.numpy(), rstd, d_rstd, "rstd")
    xh = (xn - ref.wide(mean, C)) * ref.wide(rstd, C)
    z = gamma * xh + beta
    d_z = np.abs(gamma) * (ref.wide(d_mean * rstd, C) + np.abs(xh) * ref.wide(d_rstd / rstd, C)) + 8 * U24 * (np.abs(gamma * xh) + np.abs(beta))
    want = ref.value(r, z)
    tol = half_step(c.dt) * np.abs(want) * 1.01 + 1.13 * d_z + np.maximum(np.abs(z), 0.05) * 3e-6 + smallest(c.dt)
    assert_near(y.numpy().reshape(N, P, C), want, tol, "y")


def check_backward(c, dy, x, mean, rstd, gamma, beta, r, dx, dg, db):
    """mean and rstd are given in fp32, so that xh is off by 4 steps, dz by the slope's error (below 3e-6 times 1 + |z|, see the tests of
    the activation functions; its own slope is below 1) and 4 steps; the sums over n values by 300 steps of the sum of magnitudes."""
    N, P, C, G = c.N, c.P, c.C, c.G
    dn = dy.double().numpy()
    want_dx, want_dg, want_db, xh, dz = ref.group_norm_backward(dn, x, mean, rstd, gamma, beta, G, r)
    z = gamma * xh + beta
    centre = np.abs(ref.wide(mean * rstd, C)) + np.abs(x) * ref.wide(rstd, C)
    d_xh = 4 * U24 * (np.abs(xh) + centre)
    d_z = np.abs(gamma) * d_xh + 4 * U24 * (np.abs(gamma * xh) + np.abs(beta))
    d_dz = np.abs(dn) * (3e-6 * (1 + np.abs(z)) + d_z) + 4 * U24 * np.abs(dz)
    n = 300 * U24
    t_db = (d_dz + n * np.abs(dz)).sum(axis=(0, 1))
    t_dg = (d_dz * np.abs(xh) + np.abs(dz) * d_xh + n * np.abs(dz * xh)).sum(axis=(0, 1))
    per = C // G
    mean_g = lambda v: v.reshape(N, P, G, per).mean(axis=(1, 3))  # noqa: E731
    d_m1 = mean_g(np.abs(gamma) * (d_dz + n * np.abs(dz)))
    d_m2 = mean_g(np.abs(gamma) * (d_dz * np.abs(xh) + np.abs(dz) * d_xh + n * np.abs(dz * xh)))
    m2 = mean_g(gamma * dz * xh)
    m1 = mean_g(gamma * dz)
    t_dx = ref.wide(rstd, C) * (np.abs(gamma) * d_dz + ref.wide(d_m1, C) + np.abs(xh) * ref.wide(d_m2, C) + d_xh * np.abs(ref.wide(m2, C)) +
                                8 * U24 * (np.abs(gamma * dz) + np.abs(ref.wide(m1, C)) + np.abs(xh * ref.wide(m2, C))))
    if dg is not None:
        assert_near(dg.numpy()[0], want_dg, t_dg + U24 * np.abs(want_dg), "dgamma")
    if db is not None:
        assert_near(db.numpy()[0], want_db, t_db + U24 * np.abs(want_db), "dbeta")
    assert_near(dx.numpy().reshape(N, P, C), want_dx, half_step(c.dt) * np.abs(want_dx) * 1.01 + t_dx * 1.01 + smallest(c.dt), "dx")


def relu_is_clear(x, mean, rstd, gamma, beta):
    """Whether no normalised value is so near 0 that rounding decides the side."""
    C = x.shape[2]
    return np.abs(gamma * (x - ref.wide(mean, C)) * ref.wide(rstd, C) + beta).min() > 1e-5


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "relu"])
@pytest.mark.parametrize("N,P,C,G", SHAPES)
def test_forward_and_backward(dtype, act, N, P, C, G):
    a, r = ACTS[act]
    c = Call(N, P, C, G, dtype)
    x, dy, gamma, beta = inputs(N, P, C, c.dt, N + P + C)
    gd, bd = gamma.cuda(), beta.cuda()
    y = c.forward(x, gd, bd, a)
    g64, b64 = gamma.double().numpy(), beta.double().numpy()
    check_forward(c, x, y, g64, b64, r)
    wc, wsc = ref.encode(x.float().numpy().reshape(N * P, C)) if N * P * C < 60000 else (None, None)
    if wc is not None:
        assert np.array_equal(c.codes.t.cpu().numpy(), wc) and np.array_equal(c.scales.t.cpu().numpy(), wsc)
    kx = ref.decode(c.codes.t.cpu().numpy(), c.scales.t.cpu().numpy()).reshape(N, P, C)
    mean, rstd = c.mean.numpy(), c.rstd.numpy()
    for source, x64 in ((None, kx), (x, x.double().numpy())):
        if act == "relu" and not relu_is_clear(x64, mean, rstd, g64, b64):
            continue
        dx, dg, db = c.backward(dy, source, gd, bd, a)
        check_backward(c, dy, x64, mean, rstd, g64, b64, r, dx, dg, db)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,P,C,G", [(2, 31, 64, 8), (1, 65, 30, 3), (3, 9, 128, 4)])
def test_unaligned_addresses_and_no_parameters(dtype, N, P, C, G):
    c = Call(N, P, C, G, dtype, shift=1)
    x, dy, _, _ = inputs(N, P, C, c.dt, 5)
    y = c.forward(x, None, None, ogq.OGQ_ACT_SILU, keep=False)
    one, zero = np.ones(C), np.zeros(C)
    check_forward(c, x, y, one, zero, ref.SILU)
    dx, dg, db = c.backward(dy, x, None, None, ogq.OGQ_ACT_SILU)
    check_backward(c, dy, x.double().numpy(), c.mean.numpy(), c.rstd.numpy(), one, zero, ref.SILU, dx, dg, db)
    dx2, dg2, _ = c.backward(dy, x, None, None, ogq.OGQ_ACT_SILU, want=(False, True))
    assert torch.equal(dx.t, dx2.t) and float(dg2.t.max()) == -77.0


@pytest.mark.parametrize("C", [64, 40])
def test_in_place_and_random_rounding(C):
    N, P, G = 2, 21, 8
    c = Call(N, P, C, G, "bf16")
    x, dy, gamma, beta = inputs(N, P, C, c.dt, 6)
    gamma, beta = gamma.cuda(), beta.cuda()
    y = c.forward(x, gamma, beta, ogq.OGQ_ACT_GELU, rounding=ogq.OGQ_ROUND_RANDOM, seed=99, stream_id=3)
    wc, wsc = ref.encode(x.float().numpy().reshape(N * P, C), (99, 3, 0))
    assert np.array_equal(c.codes.t.cpu().numpy(), wc) and np.array_equal(c.scales.t.cpu().numpy(), wsc)
    z = c.guarded(x)
    c.forward(z, gamma, beta, ogq.OGQ_ACT_GELU, rounding=ogq.OGQ_ROUND_RANDOM, seed=99, stream_id=3, out=z)
    assert torch.equal(y.t, z.t) and np.array_equal(c.codes.t.cpu().numpy(), wc)
    dx, _, _ = c.backward(dy, None, gamma, beta, ogq.OGQ_ACT_GELU)
    dz = c.guarded(dy)
    c.backward(dz, None, gamma, beta, ogq.OGQ_ACT_GELU, out=dz)
    assert torch.equal(dx.t, dz.t)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset", [1000.0, -3e4])
@pytest.mark.parametrize("P,C,G", [(500, 64, 8), (500, 30, 3)])
def test_a_mean_far_above_the_deviation(dtype, offset, P, C, G):
    """Moments about a value of the data: a large offset costs the offset's own rounding and nothing more.  First pixel an outlier."""
    c = Call(1, P, C, G, dtype)
    rng = np.random.default_rng(8)
    step = 8.0 if dtype == "f32" else 256.0  # values that the type holds
    x = torch.from_numpy(np.round(rng.standard_normal((1, P, C)) * 3) * step + offset).to(c.dt)
    x[0, 0] *= 3
    ones, zeros = np.ones(C), np.zeros(C)
    y = c.forward(x, None, None, ogq.OGQ_ACT_NONE, keep=False)
    check_forward(c, x, y, ones, zeros, ref.NONE)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("N,P,C,G", [(1, 49, 64, 8), (1, 49, 30, 3), (400, 49, 64, 8)])
def test_gradient_of_gamma_with_a_mean_far_above_the_deviation(dtype, N, P, C, G):
    """dgamma = sum dy (x - mean) rstd without a function: the difference is rounded once, the product, the sum's result and its factor once each,
    and a sum of P values rounds none of them more than P - 1 times, whatever the order; samples are joined in 64 bits.  So P + 8 steps of the
    sum of magnitudes, and nothing in proportion to |mean| rstd, 1200 (fp16) and 300 (bf16) here."""
    c = Call(N, P, C, G, dtype)
    rng = np.random.default_rng(21)
    step, offset = (1.0, 1040.0) if dtype == "f16" else (1.0, 250.0)
    x = torch.from_numpy(rng.integers(-1, 2, (N, P, C)) * step + offset).to(c.dt)
    dy = torch.from_numpy(0.5 + rng.random((N, P, C))).to(c.dt)
    c.forward(x, None, None, ogq.OGQ_ACT_NONE, keep=False)
    _, dg, db = c.backward(dy, x, None, None, ogq.OGQ_ACT_NONE)
    xn, dn = x.double().numpy(), dy.double().numpy()
    xh = (xn - ref.wide(c.mean.numpy(), C)) * ref.wide(c.rstd.numpy(), C)
    assert np.abs(ref.wide(c.mean.numpy() * c.rstd.numpy(), C)).min() > 250
    for got, terms in ((dg, dn * xh), (db, dn)):
        assert_near(got.numpy()[0], terms.sum(axis=(0, 1)), (P + 8) * U24 * np.abs(terms).sum(axis=(0, 1)), "dgamma, dbeta")


def test_constant_groups_and_non_finite_values():
    """Variance 0: rstd is 1 / sqrt(eps) and the outputs are beta.  A NaN or an infinity stays in its group of its sample."""
    N, P, C, G = 2, 40, 64, 8
    c = Call(N, P, C, G, "f32")
    x = torch.full((N, P, C), 3.25)
    beta = torch.linspace(-1, 1, C)
    y = c.forward(x, None, beta.cuda(), ogq.OGQ_ACT_NONE)
    assert torch.equal(c.mean.t.cpu(), torch.full((N, G), 3.25))
    assert_near(c.rstd.numpy(), np.full((N, G), EPS ** -0.5), 1e-3 * EPS ** -0.5 * 1e-3, "rstd")
    assert torch.equal(y.t.cpu().view(N, P, C), beta.expand(N, P, C))
    x = torch.randn(N, P, C)
    x[0, 5, 9] = float("nan")
    x[1, 7, 63] = float("inf")
    y = c.forward(x, None, None, ogq.OGQ_ACT_SILU).t.cpu().view(N, P, G, C // G)
    bad = ~torch.isfinite(y).all(3).all(1)
    want = torch.zeros(N, G, dtype=torch.bool)
    want[0, 1] = want[1, 7] = True
    assert torch.equal(bad, want)


def test_nothing_to_do():
    for N, P, C, G in ((0, 9, 64, 8), (2, 0, 64, 8), (2, 9, 0, 1)):
        d = ogq.OGQ_F32
        ws = torch.empty(ogq.ogq_group_norm_workspace_bytes(N, P, C, G) + 256, dtype=torch.uint8, device="cuda")
        mean, rstd = torch.full((N, G), -1.0, device="cuda"), torch.full((N, G), -1.0, device="cuda")
        ogq.ogq_group_norm_forward(None, N, P, C, G, d, None, None, EPS, 0, 0, 0, 0, None, mean, rstd, None, None, ws, ws.numel())
        if N and C:
            assert float(mean.abs().max()) == 0.0 and abs(float(rstd[0, 0]) * EPS ** 0.5 - 1) < 1e-6
        dg, db = torch.full((C,), 5.0, device="cuda"), torch.full((C,), 5.0, device="cuda")
        ogq.ogq_group_norm_backward(None, None, None, None, N, P, C, G, d, None, None, 0, mean, rstd, None, dg, db, ws, ws.numel())
        assert not dg.any() and not db.any()


@pytest.mark.parametrize("P,C,G", [(3136, 64, 8), (4100, 64, 64), (20000, 32, 4)])
def test_same_bits_again_and_large_maps(P, C, G):
    N = 3
    c = Call(N, P, C, G, "bf16")
    x, dy, gamma, beta = inputs(N, P, C, c.dt, 9)
    gd, bd = gamma.cuda(), beta.cuda()
    y = c.forward(x, gd, bd, ogq.OGQ_ACT_SILU)
    check_forward(c, x, y, gamma.double().numpy(), beta.double().numpy(), ref.SILU)
    kx = ref.decode(c.codes.t.cpu().numpy(), c.scales.t.cpu().numpy()).reshape(N, P, C)
    mean, rstd = c.mean.numpy(), c.rstd.numpy()
    dx, dg, db = c.backward(dy, None, gd, bd, ogq.OGQ_ACT_SILU)
    check_backward(c, dy, kx, mean, rstd, gamma.double().numpy(), beta.double().numpy(), ref.SILU, dx, dg, db)
    for _ in range(3):
        y2 = c.forward(x, gd, bd, ogq.OGQ_ACT_SILU)
        dx2, dg2, db2 = c.backward(dy, None, gd, bd, ogq.OGQ_ACT_SILU)
        assert torch.equal(y.t, y2.t) and torch.equal(dx.t, dx2.t) and torch.equal(dg.t, dg2.t) and torch.equal(db.t, db2.t)
