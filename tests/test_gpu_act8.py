"""Activations in 8 bits on the GPU: codes bit for bit, decoded values, the activation functions and their backward passes, against
the definitions in 64 bits.  Sizes: one element to some thousand, ends inside a group, strides, unaligned addresses."""
import numpy as np
import pytest
import torch

import act8_reference as ref
import paper_2002_11082_b200 as ogq
from act8_gpu import ACTS, DTYPES, U24, Guarded, activations, assert_near, half_step, kept, smallest

pytestmark = pytest.mark.gpu

#        rows, cols, extra stride, shift of the address in elements
SHAPES = [(1, 1, 0, 0), (3, 7, 0, 0), (2, 32, 0, 0), (5, 33, 0, 0), (4, 40, 0, 0), (7, 64, 64, 0), (3, 1000, 0, 0), (3, 1001, 0, 0), (2, 96, 8, 3),
          (9, 256, 0, 8), (33, 128, 3, 0), (2, 4104, 0, 0), (17, 24, 8, 8), (70, 8, 0, 0)]


def encode(x, ld, dtype, rounding=ogq.OGQ_ROUND_NEAREST, seed=0, stream_id=0, shift=0, code_shift=0):
    rows, cols = x.shape
    g = Guarded(rows, cols, ld, x.dtype, shift, x.cuda())
    codes, scales = kept(rows, cols, code_shift)
    ogq.ogq_act8_encode(g.t, ld, rows, cols, dtype, rounding, seed, stream_id, codes.t, scales.t)
    codes.check()
    scales.check()
    return codes, scales


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols,extra,shift", SHAPES)
def test_codes_and_values(dtype, rows, cols, extra, shift):
    d, dt = DTYPES[dtype]
    x = activations(np.random.default_rng(rows * 1000 + cols), rows, cols, dt)
    codes, scales = encode(x, cols + extra, d, shift=shift, code_shift=shift)
    w_codes, w_scales = ref.encode(x.float().numpy())
    assert np.array_equal(scales.t.cpu().numpy(), w_scales)
    assert np.array_equal(codes.t.cpu().numpy(), w_codes)
    out = Guarded(rows, cols, cols + extra, dt, shift)
    ogq.ogq_act8_decode(codes.t, scales.t, rows, cols, d, out.t, cols + extra)
    out.check()
    want = torch.from_numpy(ref.decode(w_codes, w_scales)).to(dt)  # one rounding, which only fp16 needs
    assert torch.equal(out.t.cpu(), want)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols,extra,shift", [(3, 40, 0, 0), (2, 64, 8, 0), (5, 33, 0, 1), (1, 1, 0, 0), (2, 128, 0, 8)])
def test_random_rounding_is_that_of_the_definition(dtype, rows, cols, extra, shift):
    d, dt = DTYPES[dtype]
    x = activations(np.random.default_rng(cols), rows, cols, dt)
    seed, stream = 0x1234567890ABCDEF, 77
    codes, scales = encode(x, cols + extra, d, ogq.OGQ_ROUND_RANDOM, seed, stream, shift=shift)
    w_codes, w_scales = ref.encode(x.float().numpy(), (seed, stream, 0))
    assert np.array_equal(scales.t.cpu().numpy(), w_scales)
    assert np.array_equal(codes.t.cpu().numpy(), w_codes)


def special_groups(dt):
    big, tiny = float(torch.finfo(dt).max), float(torch.finfo(dt).smallest_normal) * torch.finfo(dt).eps
    rows = [[big, -big, 1.0, 0.0], [tiny, -tiny, 0.0, 3 * tiny], [float("nan"), 1.0, 2.0, -3.0], [float("inf"), 1.0, -2.0, 0.0],
            [-float("inf"), float("nan"), 0.0, 0.0], [127.0, -127.0, 63.5, 0.5], [127.5, -128.0, 0.25, 254.0], [0.0, -0.0, 0.0, 0.0],
            [2.0 ** -14, 2.0 ** -20, -2.0 ** -13, 1e-4]]
    x = torch.zeros(len(rows), 64, dtype=dt)
    for i, r in enumerate(rows):
        x[i, 3:7] = torch.tensor(r, dtype=dt)
        x[i, 32:36] = 1.5  # the neighbouring group stays as it is
    return x


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shift", [0, 1])
def test_special_values(dtype, shift):
    """The type's largest and smallest numbers, NaN and infinities (their group alone reads as NaN), zeros."""
    d, dt = DTYPES[dtype]
    x = special_groups(dt)
    codes, scales = encode(x, 64, d, shift=shift)
    w_codes, w_scales = ref.encode(x.float().numpy())
    assert np.array_equal(scales.t.cpu().numpy(), w_scales)
    assert np.array_equal(codes.t.cpu().numpy(), w_codes)
    out = Guarded(len(x), 64, 64, torch.float32, shift)
    ogq.ogq_act8_decode(codes.t, scales.t, len(x), 64, ogq.OGQ_F32, out.t, 64)
    out.check()
    assert np.array_equal(out.numpy(), ref.decode(w_codes, w_scales), equal_nan=True)
    assert torch.isnan(out.t[2, :32]).all() and not torch.isnan(out.t[2, 32:]).any()


def tolerances(dt, z, f32):
    """Error of f(z) and of its slope before the last rounding.  fp32: CUDA's expf and erfcf, a few steps each, and about ten operations:
    16 steps of 2^-24.  The 16-bit types: exp.approx is off by (2 + 1.18 |z|) steps of 2^-23 (or z^2/2 in place of |z| in the density, where
    exp(-z^2/2) z^2 < 1), Phi by 7.5e-8 and ten operations; |z| <= 30 here, where values past 17 are 0 or z."""
    a = 16 * U24 if f32 else (2 + 1.18 * np.minimum(np.abs(z), 17)) * 2 ** -23 + 7.5e-8 + 10 * U24
    return a * np.maximum(np.abs(z), 0.05), a * (1 + np.abs(z))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows,cols,extra,shift", [(3, 40, 0, 0), (5, 33, 0, 0), (6, 256, 256, 0), (2, 1001, 0, 1), (1, 1, 0, 0), (9, 64, 8, 8)])
def test_pointwise_forward_and_backward(dtype, act, gated, rows, cols, extra, shift):
    d, dt = DTYPES[dtype]
    a, r = ACTS[act]
    rng = np.random.default_rng(rows * cols)
    ld = cols + extra
    x = Guarded(rows, cols, ld, dt, shift, activations(rng, rows, cols, dt).cuda())
    up = Guarded(rows, cols, ld, dt, shift, activations(rng, rows, cols, dt).cuda())
    y = Guarded(rows, cols, cols + 5, dt)
    codes, scales = kept(rows, cols)
    up_codes, up_scales = kept(rows, cols)
    g = (up.t, ld, up_codes.t, up_scales.t) if gated else (None, 0, None, None)
    ogq.ogq_act8_forward(x.t, ld, g[0], g[1], rows, cols, d, a, ogq.OGQ_ROUND_NEAREST, 0, 0, y.t, cols + 5, codes.t, scales.t, g[2], g[3])
    for b in (x, up, y, codes, scales, up_codes, up_scales):
        if b in (x, up):
            continue
        b.check()
    xn, un = x.numpy(), up.numpy()
    want = ref.value(r, xn)
    fy, _ = tolerances(dt, xn, dtype == "f32")
    if gated:
        want, fy = want * un, fy * np.abs(un) + U24 * np.abs(want * un)
    assert_near(y.numpy(), want, half_step(dt) * np.abs(want) * 1.01 + fy * 1.01 + smallest(dt), "y")
    wc, ws = ref.encode(x.t.float().cpu().numpy())
    assert np.array_equal(codes.t.cpu().numpy(), wc) and np.array_equal(scales.t.cpu().numpy(), ws)
    kx = ref.decode(wc, ws)
    ku = np.ones_like(kx)
    if gated:
        uc, us = ref.encode(up.t.float().cpu().numpy())
        assert np.array_equal(up_codes.t.cpu().numpy(), uc) and np.array_equal(up_scales.t.cpu().numpy(), us)
        ku = ref.decode(uc, us)

    dy = Guarded(rows, cols, ld, dt, shift, activations(rng, rows, cols, dt).cuda())
    dx, dup = Guarded(rows, cols, ld, dt, shift), Guarded(rows, cols, ld, dt, shift)
    ogq.ogq_act8_backward(dy.t, ld, codes.t, scales.t, g[2], g[3], rows, cols, d, a, dx.t, ld, dup.t if gated else None, ld if gated else 0)
    dx.check()
    dup.check() if gated else None
    dn = dy.numpy()
    fy, fs = tolerances(dt, kx, dtype == "f32")
    want = dn * ku * ref.slope(r, kx)
    assert_near(dx.numpy(), want, half_step(dt) * np.abs(want) * 1.01 + np.abs(dn * ku) * (fs + 4 * U24) * 1.01 + smallest(dt), "dx")
    if gated:
        want = dn * ref.value(r, kx)
        assert_near(dup.numpy(), want, half_step(dt) * np.abs(want) * 1.01 + np.abs(dn) * (fy + 4 * U24 * np.abs(kx)) * 1.01 + smallest(dt), "dup")


@pytest.mark.parametrize("cols", [64, 33])
def test_in_place(cols):
    """y over x and dx over dy."""
    d, dt = DTYPES["bf16"]
    rows = 50
    x = activations(np.random.default_rng(1), rows, cols, dt).cuda()
    codes, scales = kept(rows, cols)
    y, z = torch.empty_like(x), x.clone()
    ogq.ogq_act8_forward(x, cols, None, 0, rows, cols, d, ogq.OGQ_ACT_SILU, 0, 0, 0, y, cols, codes.t, scales.t, None, None)
    first = codes.t.clone()
    ogq.ogq_act8_forward(z, cols, None, 0, rows, cols, d, ogq.OGQ_ACT_SILU, 0, 0, 0, z, cols, codes.t, scales.t, None, None)
    assert torch.equal(y, z) and torch.equal(first, codes.t)
    dy = torch.randn_like(x)
    dx, dz = torch.empty_like(x), dy.clone()
    ogq.ogq_act8_backward(dy, cols, codes.t, scales.t, None, None, rows, cols, d, ogq.OGQ_ACT_GELU, dx, cols, None, 0)
    ogq.ogq_act8_backward(dz, cols, codes.t, scales.t, None, None, rows, cols, d, ogq.OGQ_ACT_GELU, dz, cols, None, 0)
    assert torch.equal(dx, dz)


def test_far_arguments():
    """Values far outside the functions' middle: 0 or z, no NaN from an overflowing exponential."""
    z = torch.tensor([-1e4, -200.0, -90.0, -30.0, 30.0, 90.0, 200.0, 1e4], device="cuda")
    x = torch.zeros(8, 32, device="cuda")
    x[:, 0] = z
    for dtype in ("f32", "bf16"):
        d, dt = DTYPES[dtype]
        xx = x.to(dt)
        for act in ("silu", "gelu"):
            a, r = ACTS[act]
            codes, scales = kept(8, 32)
            y, dx = torch.empty_like(xx), torch.empty_like(xx)
            ogq.ogq_act8_forward(xx, 32, None, 0, 8, 32, d, a, 0, 0, 0, y, 32, codes.t, scales.t, None, None)
            ogq.ogq_act8_backward(torch.ones_like(xx), 32, codes.t, scales.t, None, None, 8, 32, d, a, dx, 32, None, 0)
            y, dx, zz = y[:, 0].double().cpu().numpy(), dx[:, 0].double().cpu().numpy(), xx[:, 0].double().cpu().numpy()
            assert np.all(np.isfinite(y)) and np.all(np.isfinite(dx))
            assert_near(y, np.where(zz > 0, zz, 0.0), 1e-11 + np.abs(zz) * 2.0 ** -8 * (zz > 0), act)
            assert_near(dx, (zz > 0).astype(float), 1e-11 + 2.0 ** -8 * (zz > 0), act)


def test_empty():
    for rows, cols in ((0, 64), (4, 0)):
        ogq.ogq_act8_encode(None, cols, rows, cols, ogq.OGQ_F32, 0, 0, 0, None, None)
        ogq.ogq_act8_decode(None, None, rows, cols, ogq.OGQ_F32, None, cols)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_matrix_equals_its_rows(dtype):
    """2^26 and more elements, many trips of the kernels' loops: every row equals the row encoded alone."""
    d, dt = DTYPES[dtype]
    rows, cols = 20011, 4096
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(rows, cols, device="cuda", generator=gen).to(dt)
    codes, scales = kept(rows, cols)
    ogq.ogq_act8_encode(x, cols, rows, cols, d, 0, 0, 0, codes.t, scales.t)
    out = torch.empty_like(x)
    ogq.ogq_act8_decode(codes.t, scales.t, rows, cols, d, out, cols)
    unit = ((scales.t.int() << 23).view(torch.float32)).repeat_interleave(32, 1)
    assert torch.equal(out.float(), (codes.t.float() * unit).to(dt).float())
    assert bool((((out.float() - x.float()).abs() / unit) <= 0.5).all())
    top = codes.t.view(rows, -1, 32).abs().amax(2)
    assert int(top.min()) >= 64 and int(top.max()) <= 127
    for r in (0, 7, rows - 1):
        c1, s1 = kept(1, cols)
        ogq.ogq_act8_encode(x[r:r + 1], cols, 1, cols, d, 0, 0, 0, c1.t, s1.t)
        assert torch.equal(c1.t[0], codes.t[r]) and torch.equal(s1.t[0], scales.t[r])
