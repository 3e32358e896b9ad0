"""Group norm where it can lose what matters: constant groups, means far above the deviation, values at the mean, and both families of kernels
(a slab of channels in registers over a cluster, and streaming over many chunks of pixels) by name."""
import numpy as np
import pytest
import torch

import act8_reference as ref
import paper_2002_11082_b200 as ogq
from act8_gpu import ACTS, DTYPES, U24, assert_near, half_step, smallest
from test_gpu_group_norm import EPS, Call, check_backward, check_forward, inputs

pytestmark = pytest.mark.gpu

RESIDENT = [(2, 49, 64, 8), (1, 196, 256, 32), (1, 1300, 32, 1), (1, 700, 40, 8)]
STREAMED = [(3, 20000, 32, 4), (2, 9000, 64, 8)]
SINGLE = [(2, 49, 30, 3), (1, 1500, 33, 11)]  # channels one by one
ALL = RESIDENT + STREAMED + SINGLE


def kernels(f):
    """What f returns, and the names of the kernels that it launched."""
    ogq.ogq_profile_enable(True)
    try:
        got = f()
        torch.cuda.synchronize()
        return got, [name for name, _ in ogq.ogq_profile_collect()]
    finally:
        ogq.ogq_profile_enable(False)


def assert_family(shape, forward, backward):
    if shape in RESIDENT:
        assert forward == ["k_gn_forward"] and backward[0] == "k_gn_backward"
    else:
        assert "k_gn_apply" in forward and backward[0] == "k_gn_grad_sums" and backward[-1] == "k_gn_grad"


CONSTANTS = {"f32": [3.25, 1000.1, -29999.7, 1e6 + 0.3], "f16": [100.0, 1000.5, -60000.0], "bf16": [100.0, 2000.0, -29952.0]}


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,P,C,G", ALL)
def test_constant_groups_of_every_type(dtype, N, P, C, G):
    """Variance 0, whatever the value: the mean is that value and every output beta, to the last bit; dx = rstd (dz - m1), xh = 0.  rstd = 1 / sqrt(eps): where the
    kernel takes squares about a mean that is off by k steps before it corrects it, what is left of them is some steps of (k 2^-24 c)^2, 1e-4 of eps at most."""
    c = Call(N, P, C, G, dtype)
    beta = torch.linspace(-1, 1, C).cuda()
    gamma = torch.linspace(0.5, 2, C).cuda()
    for v in CONSTANTS[dtype]:
        x = torch.full((N, P, C), v).to(c.dt)
        for keep in (False, True):
            y = c.forward(x, gamma, beta, ogq.OGQ_ACT_NONE, keep=keep)
            assert torch.equal(c.mean.t, x[0, 0, 0].float().cuda().expand(N, G))
            assert_near(c.rstd.numpy(), np.full((N, G), EPS ** -0.5), 1e-4 * EPS ** -0.5, "rstd")
            assert torch.equal(y.t, beta.to(c.dt).expand(N * P, C)), v
        dy = torch.from_numpy(np.random.default_rng(3).standard_normal((N, P, C))).to(c.dt)
        dx, dg, db = c.backward(dy, x, gamma, beta, ogq.OGQ_ACT_NONE)
        assert not dg.t.any()
        check_backward(c, dy, x.double().numpy(), c.mean.numpy(), c.rstd.numpy(), gamma.double().cpu().numpy(), beta.double().cpu().numpy(), ref.NONE, dx, dg, db)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,P,C,G", ALL)
def test_the_mean_is_off_by_its_own_rounding(dtype, N, P, C, G):
    """Sums are taken about a value near the mean: at most 64 additions in a thread, 256 rows of threads, the rest in 64 bits or within a warp, each off by half a step
    of what deviates; of the mean itself only the roundings of up to four means on the way count."""
    c = Call(N, P, C, G, dtype)
    rng = np.random.default_rng(5)
    offset, step = {"f32": (1e5, 2.0 ** -7), "f16": (1500.0, 1.0), "bf16": (200.0, 1.0)}[dtype]
    x = torch.from_numpy(rng.integers(-3, 4, (N, P, C)) * step + offset).to(c.dt)
    y = c.forward(x, None, None, ogq.OGQ_ACT_NONE, keep=False)
    xn = x.double().numpy()
    mean, rstd = ref.group_stats(xn, G, EPS)
    d_mean = U24 * (4 * np.abs(mean) + 400 * 6 * step)
    assert_near(c.mean.numpy(), mean, d_mean, "mean")
    # the mean that the function subtracts is the one it reports
    z = (xn - ref.wide(c.mean.numpy(), C)) * ref.wide(c.rstd.numpy(), C)
    assert_near(y.numpy().reshape(N, P, C), z, half_step(c.dt) * np.abs(z) * 1.01 + 4 * U24 * np.abs(z) + smallest(c.dt), "y")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("N,P,C,G", ALL)
def test_values_at_the_mean_are_on_one_side(dtype, keep, N, P, C, G):
    """As many values one step above the mean as below it, and some at it: z = gamma (x - mean) rstd has the sign of gamma (x - mean), and the forward pass and every
    kernel of the backward pass take the same side of ReLU."""
    c = Call(N, P, C, G, dtype)
    rng = np.random.default_rng(6)
    per = C // G
    offset = 96.0  # 95, 96, 97 are kept in 8 bits as they are
    d = np.zeros(P * per)
    d[:P * per // 3] = 1
    d[P * per // 3:2 * (P * per // 3)] = -1
    x = np.stack([np.concatenate([rng.permutation(d).reshape(P, per) for _ in range(G)], axis=1) for _ in range(N)])
    gamma = torch.from_numpy(rng.standard_normal(C)).float()
    xt = torch.from_numpy(x + offset).to(c.dt)
    y = c.forward(xt, gamma.cuda(), None, ogq.OGQ_ACT_RELU, keep=keep)
    above = torch.from_numpy((x + offset - ref.wide(c.mean.numpy(), C)) * gamma.numpy() > 0)
    assert torch.equal(y.t.cpu().view(N, P, C) > 0, above)
    dy = torch.ones(N, P, C, dtype=c.dt)
    dx, _, db = c.backward(dy, None if keep else xt, gamma.cuda(), None, ogq.OGQ_ACT_RELU)
    assert torch.equal(db.t[0].cpu(), above.float().sum((0, 1)))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("act", ["none", "silu", "gelu", "relu"])
@pytest.mark.parametrize("N,P,C,G", [(2, 49, 64, 8), (1, 1300, 32, 1), (1, 700, 40, 8), (3, 20000, 32, 4), (2, 9000, 64, 8)])
def test_both_families_of_kernels(dtype, act, N, P, C, G):
    """Slabs in registers, in one CTA or a cluster, and streaming over several chunks of pixels.  Where rounding decides the side of ReLU, dy is 0."""
    a, r = ACTS[act]
    c = Call(N, P, C, G, dtype)
    x, dy, gamma, beta = inputs(N, P, C, c.dt, N + P + C + 1)
    gd, bd = gamma.cuda(), beta.cuda()
    g64, b64 = gamma.double().numpy(), beta.double().numpy()
    keep = C % 32 == 0
    y, fw = kernels(lambda: c.forward(x, gd, bd, a, keep=keep))
    check_forward(c, x, y, g64, b64, r)
    if not keep:  # the encoder's own pass, and the streaming kernels
        check_forward(c, x, c.forward(x, gd, bd, a), g64, b64, r)
    kx = ref.decode(c.codes.t.cpu().numpy(), c.scales.t.cpu().numpy()).reshape(N, P, C)
    mean, rstd = c.mean.numpy(), c.rstd.numpy()
    for source, x64 in ((None, kx), (x, x.double().numpy())):
        d = dy.clone()
        if act == "relu":
            near = np.abs(g64 * (x64 - ref.wide(mean, C)) * ref.wide(rstd, C) + b64) < 1e-5
            assert near.mean() < 1e-3
            d[torch.from_numpy(near)] = 0
        (dx, dg, db), bw = kernels(lambda: c.backward(d, source, gd, bd, a))
        assert_family((N, P, C, G), fw, bw)
        check_backward(c, d, x64, mean, rstd, g64, b64, r, dx, dg, db)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("N,P,C,G", STREAMED)
def test_gradient_of_gamma_over_many_chunks(dtype, N, P, C, G):
    """dgamma = sum dy (x - mean) rstd: a thread rounds a term's difference, its product and up to 64 sums, the factor and a chunk's sum once each;
    the rest is in 64 bits.  80 half steps of the sum of magnitudes, nothing in proportion to |mean| rstd (250 and more here)."""
    c = Call(N, P, C, G, dtype)
    rng = np.random.default_rng(22)
    x = torch.from_numpy(rng.integers(-1, 2, (N, P, C)) + (1040.0 if dtype == "f16" else 250.0)).to(c.dt)
    dy = torch.from_numpy(0.5 + rng.random((N, P, C))).to(c.dt)
    c.forward(x, None, None, ogq.OGQ_ACT_NONE, keep=False)
    (_, dg, db), names = kernels(lambda: c.backward(dy, x, None, None, ogq.OGQ_ACT_NONE))
    assert names == ["k_gn_grad_sums", "k_gn_grad_join", "k_gn_grad"]
    xn, dn = x.double().numpy(), dy.double().numpy()
    xh = (xn - ref.wide(c.mean.numpy(), C)) * ref.wide(c.rstd.numpy(), C)
    for got, terms in ((dg, dn * xh), (db, dn)):
        assert_near(got.numpy()[0], terms.sum(axis=(0, 1)), 80 * U24 * np.abs(terms).sum(axis=(0, 1)), "dgamma, dbeta")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,P,C,G", [(1, 900, 96, 3), (1, 2000, 64, 64), (2, 60, 480, 2), (1, 100, 200, 5), (4, 333, 72, 3), (1, 700, 40, 8)])
def test_slabs_of_uneven_widths_over_clusters(dtype, N, P, C, G):
    """Clusters of one to eight CTAs whose warps hold different numbers of groups, channels or rows when they come to the cluster's barriers."""
    c = Call(N, P, C, G, dtype)
    x, dy, gamma, beta = inputs(N, P, C, c.dt, N + P + C + 2)
    gd, bd, g64, b64 = gamma.cuda(), beta.cuda(), gamma.double().numpy(), beta.double().numpy()
    first = None
    for _ in range(3):
        y, fw = kernels(lambda: c.forward(x, gd, bd, ogq.OGQ_ACT_SILU, keep=C % 32 == 0))
        check_forward(c, x, y, g64, b64, ref.SILU)
        (dx, dg, db), bw = kernels(lambda: c.backward(dy, x, gd, bd, ogq.OGQ_ACT_SILU))
        assert fw == ["k_gn_forward"] and bw[0] == "k_gn_backward"
        check_backward(c, dy, x.double().numpy(), c.mean.numpy(), c.rstd.numpy(), g64, b64, ref.SILU, dx, dg, db)
        got = [t.t.clone() for t in (y, dx, dg, db)]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))


@pytest.mark.parametrize("N,P,C,G", STREAMED + RESIDENT[2:3])
def test_in_place_and_replayed(N, P, C, G):
    """y over x and dx over dy, captured: every replay on fresh inputs gives the bits of the calls on buffers of their own."""
    c = Call(N, P, C, G, "bf16")
    x, dy, gamma, beta = inputs(N, P, C, c.dt, 31)
    gd, bd = gamma.cuda(), beta.cuda()
    y = c.forward(x, gd, bd, ogq.OGQ_ACT_SILU).t.clone()
    codes, scales = c.codes.t.clone(), c.scales.t.clone()
    want = [t.t.clone() for t in c.backward(dy, None, gd, bd, ogq.OGQ_ACT_SILU)]
    a, b = x.cuda().view(N * P, C).clone(), dy.cuda().view(N * P, C).clone()
    dg, db = torch.zeros(C, device="cuda"), torch.zeros(C, device="cuda")
    size = (N, P, C, G, c.d)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ogq.ogq_group_norm_forward(a, *size, gd, bd, EPS, ogq.OGQ_ACT_SILU, 0, 0, 0, a, c.mean.t, c.rstd.t, c.codes.t, c.scales.t, c.ws, c.ws.numel())
        ogq.ogq_group_norm_backward(b, None, c.codes.t, c.scales.t, *size, gd, bd, ogq.OGQ_ACT_SILU, c.mean.t, c.rstd.t, b, dg, db, c.ws, c.ws.numel())
    for _ in range(3):
        a.copy_(x.view(N * P, C))
        b.copy_(dy.view(N * P, C))
        c.codes.t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, y) and torch.equal(c.codes.t, codes) and torch.equal(c.scales.t, scales)
        assert torch.equal(b, want[0]) and torch.equal(dg, want[1][0]) and torch.equal(db, want[2][0])
    del graph


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("N,P,C,G", ALL)
def test_mean_of_a_group_with_infinities(dtype, N, P, C, G):
    """Infinities of one sign, at a thread's first pixel or a later one: the mean is that infinity, of both signs or with a NaN it is NaN; rstd is NaN and so are the
    group's outputs.  The other groups are as without it, to the last bit."""
    c = Call(N, P, C, G, dtype)
    x, _, _, _ = inputs(N, P, C, c.dt, 33)
    clean = [t.t.clone() for t in (c.forward(x, None, None, ogq.OGQ_ACT_NONE, keep=False), c.mean, c.rstd)]
    inf = float("inf")
    for at, value in ((((0, 0),), (inf,)), (((0, P - 1),), (-inf,)), (((0, 0), (0, P // 2), (0, P - 1)), (inf,) * 3), (((0, 1), (0, P - 1)), (inf, -inf)),
                      (((0, P // 3),), (float("nan"),))):
        z = x.clone()
        for (n, p), v in zip(at, value):
            z[n, p, C - 1] = v
        y = c.forward(z, None, None, ogq.OGQ_ACT_NONE, keep=False)
        want = sum(value)
        got = float(c.mean.t[0, G - 1])
        assert got == want or (got != got and want != want), (at, value, got)
        assert bool(torch.isnan(c.rstd.t[0, G - 1])) and bool(torch.isnan(y.t.view(N, P, G, C // G)[0, :, G - 1]).all())
        rest = torch.ones(N, G, dtype=torch.bool, device="cuda")
        rest[0, G - 1] = False
        assert torch.equal(c.mean.t[rest], clean[1][rest]) and torch.equal(c.rstd.t[rest], clean[2][rest])
        pick = rest[:, None, :, None].expand(N, P, G, C // G)
        assert torch.equal(y.t.view(N, P, G, C // G)[pick], clean[0].view(N, P, G, C // G)[pick])
