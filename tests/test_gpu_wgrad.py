"""Weight and bias gradient from the 8-bit input, against the sums in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2002_11082_b200 as ogq
from act8_gpu import DTYPES, Guarded, assert_near

pytestmark = pytest.mark.gpu

#        rows, cols, out_cols
SHAPES = [(1, 1, 1), (1, 64, 128), (7, 33, 5), (31, 40, 72), (64, 64, 128), (65, 256, 128), (100, 100, 100), (130, 300, 257), (1000, 64, 256),
          (33, 1000, 1000), (200, 17, 1024), (200, 1032, 24), (3000, 128, 136), (5, 4104, 64)]


# the same with more rows or weights than one launch takes without the tensor cores
LARGER = [(2049, 130, 70), (4100, 1, 1), (2500, 17, 24), (700, 333, 999), (64, 1000, 1100), (1, 1032, 1040), (130, 1100, 1300), (513, 96, 130), (2177, 260, 513),
          (33, 1100, 1001), (6000, 64, 250)]


def kept_matrix(gen, rows, cols):
    codes = torch.randint(-127, 128, (rows, cols), device="cuda", generator=gen, dtype=torch.int8)
    scales = torch.randint(115, 124, (rows, -(-cols // 32)), device="cuda", generator=gen).to(torch.uint8)
    return codes, scales


def decoded(codes, scales):
    unit = torch.ldexp(torch.ones_like(scales, dtype=torch.float64), scales.int() - 127)
    return codes.double() * unit.repeat_interleave(32, 1)[:, :codes.shape[1]]


def run(dy, ld, codes, scales, rows, cols, out, dtype, accumulate=0, dw=None, db=None, bias=True):
    ws = torch.full((ogq.ogq_act8_wgrad_workspace_bytes(rows, cols, out, dtype),), 0xA5, dtype=torch.uint8, device="cuda")
    dw = dw or Guarded(out, cols, cols, torch.float32)
    db = db or Guarded(1, out, out, torch.float32)
    ogq.ogq_act8_wgrad(dy, ld, codes, scales, rows, cols, out, dtype, accumulate, dw.t, db.t if bias else None, ws, ws.numel())
    dw.check()
    db.check()
    return dw, db


def check(dy, x, dw, db, before_w=0.0, before_b=0.0):
    """Products are exact; each addition of 16 products may drop two bits below the 24 of the running sum, or a chain of single additions
    rounds each time: at most rows + 64 steps of 2^-24 of the sum of magnitudes, or a quarter of those as steps of 2^-22."""
    rows = dy.shape[0]
    d = dy.double()
    steps = (rows + 64) * 2.0 ** -24
    want, size = d.t() @ x, d.abs().t() @ x.abs()
    assert_near(dw.numpy(), (want + before_w).cpu().numpy(), (size * steps + (want + before_w).abs() * 2.0 ** -23).cpu().numpy(), "dw")
    if db is not None:
        want, size = d.sum(0), d.abs().sum(0)
        assert_near(db.numpy()[0], (want + before_b).cpu().numpy(), (size * steps + (want + before_b).abs() * 2.0 ** -23).cpu().numpy(), "db")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols,out", SHAPES + LARGER)
@pytest.mark.parametrize("extra,shift", [(0, 0), (8, 0), (3, 1)])
def test_against_the_sums(dtype, rows, cols, out, extra, shift):
    d, dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(rows + cols + out)
    codes, scales = kept_matrix(gen, rows, cols)
    dy = Guarded(rows, out, out + extra, dt, shift, torch.randn(rows, out, device="cuda", generator=gen).to(dt))
    dw, db = run(dy.t, out + extra, codes, scales, rows, cols, out, d)
    x = decoded(codes, scales)
    check(dy.t, x, dw, db)
    # no bias, added to what is there, at unaligned addresses
    start = torch.randn(out, cols, device="cuda", generator=gen)
    dw2 = Guarded(out, cols, cols, torch.float32, 1, start)
    db2 = Guarded(1, out, out, torch.float32)
    run(dy.t, out + extra, codes, scales, rows, cols, out, d, 1, dw2, db2, bias=False)
    check(dy.t, x, dw2, None, start.double())
    assert bool((db2.t == -77.0).all())


@pytest.mark.parametrize("rows", [0, 1, 70])
@pytest.mark.parametrize("cols", [0, 64, 65])
def test_rows_of_none_and_accumulation(rows, cols):
    gen = torch.Generator(device="cuda").manual_seed(3)
    out = 48
    codes, scales = kept_matrix(gen, rows, cols)
    x = decoded(codes, scales)
    dy = torch.randn(rows, out, device="cuda", generator=gen).bfloat16()
    dw, db = run(dy, out, codes, scales, rows, cols, out, ogq.OGQ_BF16)
    check(dy, x, dw, db)
    w0, b0 = dw.t.clone(), db.t.clone()
    run(dy, out, codes, scales, rows, cols, out, ogq.OGQ_BF16, 1, dw, db)
    check(dy, x, dw, db, w0.double(), b0[0].double())


def test_a_column_that_was_not_finite_and_units_of_all_sizes():
    """Units from 2^-120 to 2^121 in their own columns; a group that reads as NaN makes its columns NaN and no others; an infinity in dy its row."""
    rows, cols, out = 96, 128, 64
    gen = torch.Generator(device="cuda").manual_seed(5)
    codes, _ = kept_matrix(gen, rows, cols)
    scales = torch.tensor([7, 127, 240, 120], dtype=torch.uint8, device="cuda").repeat(rows, 1)
    dy = (torch.randn(rows, out, device="cuda", generator=gen) * 0.01).bfloat16()
    dw, db = run(dy, out, codes, scales, rows, cols, out, ogq.OGQ_BF16)
    check(dy, decoded(codes, scales), dw, db)
    scales[17, 3] = 255
    codes[17, 96:] = 0
    dw, db = run(dy, out, codes, scales, rows, cols, out, ogq.OGQ_BF16)
    assert bool(torch.isnan(dw.t[:, 96:]).all()) and bool(torch.isfinite(dw.t[:, :96]).all()) and bool(torch.isfinite(db.t).all())
    scales[17, 3] = 120
    dy[3, 9] = float("inf")
    dw, db = run(dy, out, codes, scales, rows, cols, out, ogq.OGQ_BF16)
    bad = ~torch.isfinite(dw.t)
    assert bool(bad[9][codes[3] != 0].all()) and not bool(bad[torch.arange(out) != 9].any())


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_types_lose_nothing(dtype):
    """One row: every weight is a single product, exact up to its rounding to fp32 (fp32 gradients: products of 24 and 7 bits, in three terms)."""
    d, dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(6)
    codes, scales = kept_matrix(gen, 1, 96)
    dy = torch.randn(1, 200, device="cuda", generator=gen).to(dt)
    dw, db = run(dy, 200, codes, scales, 1, 96, 200, d)
    want = (dy.double().t() @ decoded(codes, scales)).cpu().numpy()
    assert_near(dw.numpy(), want, np.abs(want) * 2.0 ** -22, "dw")
    assert np.array_equal(db.numpy()[0], dy[0].double().cpu().numpy()) or dtype == "f32"


@pytest.mark.parametrize("rows,cols,out,dtype", [(20000, 64, 256, "bf16"), (4096, 1024, 1000, "bf16"), (9000, 320, 640, "f16"), (5000, 512, 200, "f32"),
                                                 (70000, 40, 24, "bf16")])
def test_long_sums_and_the_same_bits_again(rows, cols, out, dtype):
    d, dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(7)
    codes, scales = kept_matrix(gen, rows, cols)
    dy = torch.randn(rows, out, device="cuda", generator=gen).to(dt)
    dw, db = run(dy, out, codes, scales, rows, cols, out, d)
    x = decoded(codes, scales)
    check(dy, x, dw, db)
    want = dy.double().t() @ x  # and in the norm, where a missing tile shows that the bound above would let pass
    assert float((dw.t.double() - want).norm() / want.norm()) < 1e-5
    for _ in range(3):
        dw2, db2 = run(dy, out, codes, scales, rows, cols, out, d)
        assert torch.equal(dw.t, dw2.t) and torch.equal(db.t, db2.t)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols,out", [(32, 2048, 300), (128, 130, 70), (129, 2049, 258), (700, 2304, 513), (2000, 4096, 1000), (1, 2048, 1)])
def test_bias_beside_the_product(dtype, rows, cols, out):
    """Eight tiles of a column and more, or one step of 128 rows: the product's kernel adds up dy itself; added to what is there too."""
    d, dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    codes, scales = kept_matrix(gen, rows, cols)
    ld = (out + 7) // 8 * 8
    dy = Guarded(rows, out, ld, dt, 0, torch.randn(rows, out, device="cuda", generator=gen).to(dt))
    x = decoded(codes, scales)
    dw, db = run(dy.t, ld, codes, scales, rows, cols, out, d)
    check(dy.t, x, dw, db)
    w0, b0 = dw.t.clone(), db.t.clone()
    run(dy.t, ld, codes, scales, rows, cols, out, d, 1, dw, db)
    check(dy.t, x, dw, db, w0.double(), b0[0].double())


@pytest.mark.parametrize("rows,cols,out", [(700, 512, 700), (3000, 100, 300), (40, 96, 64), (2300, 48, 40)])
@pytest.mark.parametrize("code_shift,scale_shift", [(1, 0), (0, 1), (16, 4), (3, 2)])
def test_codes_and_scales_at_any_address(rows, cols, out, code_shift, scale_shift):
    gen = torch.Generator(device="cuda").manual_seed(11)
    codes, scales = kept_matrix(gen, rows, cols)
    c = Guarded(rows, cols, cols, torch.int8, code_shift, codes)
    s = Guarded(rows, scales.shape[1], scales.shape[1], torch.uint8, scale_shift, scales)
    dy = torch.randn(rows, out, device="cuda", generator=gen).bfloat16()
    dw, db = run(dy, out, c.t, s.t, rows, cols, out, ogq.OGQ_BF16)
    check(dy, decoded(codes, scales), dw, db)
