"""8-bit activations and the operators on them past 2^31 elements, with many samples, on other streams, and captured into a graph by the first
calls that a process makes."""
import subprocess
import sys

import pytest
import torch

import paper_2002_11082_b200 as ogq
from act8_gpu import DTYPES

pytestmark = pytest.mark.gpu
BF = ogq.OGQ_BF16


def kept(rows, cols):
    return torch.empty(rows, cols, dtype=torch.int8, device="cuda"), torch.empty(rows, -(-cols // 32), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("cols", [32768, 32765])
def test_a_matrix_past_2_to_the_31_elements(cols):
    """The last rows equal those rows alone: vector and single-element kernels, forward and backward."""
    rows, last = 66000, 3
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    codes, scales = kept(rows, cols)
    y = torch.empty_like(x)
    ogq.ogq_act8_forward(x, cols, None, 0, rows, cols, BF, ogq.OGQ_ACT_SILU, 0, 0, 0, y, cols, codes, scales, None, None)
    c1, s1 = kept(last, cols)
    tail = x[-last:].clone()
    y1 = torch.empty_like(tail)
    ogq.ogq_act8_forward(tail, cols, None, 0, last, cols, BF, ogq.OGQ_ACT_SILU, 0, 0, 0, y1, cols, c1, s1, None, None)
    assert torch.equal(codes[-last:], c1) and torch.equal(scales[-last:], s1) and torch.equal(y[-last:], y1)
    ogq.ogq_act8_backward(x, cols, codes, scales, None, None, rows, cols, BF, ogq.OGQ_ACT_GELU, y, cols, None, 0)
    ogq.ogq_act8_backward(tail, cols, c1, s1, None, None, last, cols, BF, ogq.OGQ_ACT_GELU, y1, cols, None, 0)
    assert torch.equal(y[-last:], y1)


def test_random_rounding_counts_past_2_to_the_32():
    """The counter of element 2^32 and more differs from that of element 0 (its high word is used)."""
    rows, cols = 131073, 32768
    x = torch.full((1, cols), 0.3, dtype=torch.bfloat16, device="cuda")
    x[0, 0::32] = 100.0
    wide = x.expand(rows, cols).contiguous()
    codes, scales = kept(rows, cols)
    ogq.ogq_act8_encode(wide, cols, rows, cols, BF, ogq.OGQ_ROUND_RANDOM, 7, 0, codes, scales)
    assert not torch.equal(codes[0], codes[131072])
    one, s1 = kept(1, cols)
    ogq.ogq_act8_encode(x, cols, 1, cols, BF, ogq.OGQ_ROUND_RANDOM, 7, 0, one, s1)
    assert torch.equal(codes[0], one[0])


@pytest.mark.parametrize("N,P,C,G", [(3, 12000000, 64, 8), (70000, 3, 64, 4), (100001, 1, 8, 1), (4097, 40, 33, 3), (300, 7, 2048, 64)])
def test_group_norm_of_many_elements_or_samples(N, P, C, G):
    """The last sample equals that sample alone, up to the order of the additions (the launches differ): a few steps of bf16."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty(N, P, C, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    dy = x if N * P * C > 1 << 31 else torch.empty_like(x).normal_(generator=gen)
    gamma, beta = torch.ones(C, device="cuda"), torch.zeros(C, device="cuda")

    def run(x, dy):
        n = x.shape[0]
        ws = torch.empty(ogq.ogq_group_norm_workspace_bytes(n, P, C, G), dtype=torch.uint8, device="cuda")
        y, mean, rstd = torch.empty_like(x), torch.empty(n, G, device="cuda"), torch.empty(n, G, device="cuda")
        ogq.ogq_group_norm_forward(x, n, P, C, G, BF, gamma, beta, 1e-3, ogq.OGQ_ACT_SILU, 0, 0, 0, y, mean, rstd, None, None, ws, ws.numel())
        last = y[-1].clone()
        dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        ogq.ogq_group_norm_backward(dy, x, None, None, n, P, C, G, BF, gamma, beta, ogq.OGQ_ACT_SILU, mean, rstd, y, dg, db, ws, ws.numel())
        return last, mean[-1], rstd[-1], y[-1].clone(), dg, db

    a, b = run(x, dy), run(x[-1:].clone(), dy[-1:].clone())
    for i, tol in ((0, 2.0 ** -7), (1, 1e-4), (2, 1e-4), (3, 2.0 ** -6)):
        d = (a[i].float() - b[i].float()).abs()
        assert float(d.max()) <= tol * (float(b[i].float().abs().max()) + 1), i
    assert bool(torch.isfinite(a[4]).all()) and bool(torch.isfinite(a[5]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_weight_gradient_past_2_to_the_31_elements(dtype):
    d, dt = DTYPES[dtype]
    rows, cols, out = 530000, 48, 4096
    gen = torch.Generator(device="cuda").manual_seed(3)
    dy = torch.empty(rows, out, dtype=dt, device="cuda").normal_(generator=gen)
    codes = torch.randint(-127, 128, (rows, cols), device="cuda", generator=gen, dtype=torch.int8)
    scales = torch.randint(118, 124, (rows, 2), device="cuda", generator=gen).to(torch.uint8)
    ws = torch.empty(ogq.ogq_act8_wgrad_workspace_bytes(rows, cols, out, d), dtype=torch.uint8, device="cuda")
    dw, db = torch.empty(out, cols, device="cuda"), torch.empty(out, device="cuda")
    ogq.ogq_act8_wgrad(dy, out, codes, scales, rows, cols, out, d, 0, dw, db, ws, ws.numel())
    unit = torch.ldexp(torch.ones_like(scales, dtype=torch.float64), scales.int() - 127).repeat_interleave(32, 1)[:, :cols]
    x = codes.double() * unit
    want, size, bias = 0, 0, 0
    for t in range(0, rows, 53000):
        part = dy[t:t + 53000].double()
        want, size, bias = want + part.t() @ x[t:t + 53000], size + part.abs().t() @ x[t:t + 53000].abs(), bias + part.sum(0)
    # running sums of 512 rows, then additions in fp32: 1,100 parts, each addition half a step of the sum of magnitudes at most
    assert bool(((dw.double() - want).abs() <= size * 1200 * 2.0 ** -24).all())
    assert float((dw.double() - want).norm() / want.norm()) < 1e-5
    assert float((db.double() - bias).norm() / bias.norm()) < 1e-5


def test_on_another_stream_than_the_default():
    """Work goes to the stream that is given, in its order."""
    rows, cols = 4096, 1024
    x = torch.randn(rows, cols, device="cuda")
    codes, scales = kept(rows, cols)
    out = torch.zeros_like(x)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x.mul_(2.0)
    ogq.ogq_act8_encode(x, cols, rows, cols, ogq.OGQ_F32, 0, 0, 0, codes, scales, stream=side)
    ogq.ogq_act8_decode(codes, scales, rows, cols, ogq.OGQ_F32, out, cols, stream=side.cuda_stream)
    side.synchronize()
    top = x.view(rows, -1, 32).abs().amax(2, keepdim=True)
    assert bool(((out - x).view(rows, -1, 32).abs() <= top / 127).all())


FIRST = """
import torch
import paper_2002_11082_b200 as ogq
BF, N, P, C, G = ogq.OGQ_BF16, 2, 64, 128, 8
T = N * P
z = lambda *s, d=torch.bfloat16: torch.zeros(s, device="cuda", dtype=d)
x = torch.randn(T, C, device="cuda").bfloat16()
y, dx, mean, rstd = z(T, C), z(T, C), z(N, G, d=torch.float32), z(N, G, d=torch.float32)
codes, scales = z(T, C, d=torch.int8), z(T, C // 32, d=torch.uint8)
dw, db, dg, dbe = z(C, C, d=torch.float32), z(C, d=torch.float32), z(C, d=torch.float32), z(C, d=torch.float32)
ws = z(1 << 27, d=torch.uint8)
def step():
    ogq.ogq_group_norm_forward(x, N, P, C, G, BF, None, None, 1e-5, 2, 0, 0, 0, y, mean, rstd, codes, scales, ws, ws.numel())
    ogq.ogq_act8_wgrad(y, C, codes, scales, T, C, C, BF, 0, dw, db, ws, ws.numel())
    ogq.ogq_group_norm_backward(y, None, codes, scales, N, P, C, G, BF, None, None, 2, mean, rstd, dx, dg, dbe, ws, ws.numel())
    ogq.ogq_act8_forward(dx, C, None, 0, T, C, BF, 3, 0, 0, 0, y, C, codes, scales, None, None)
    ogq.ogq_act8_backward(dx, C, codes, scales, None, None, T, C, BF, 3, y, C, None, 0)
    ogq.ogq_act8_encode(y, C, T, C, BF, 0, 0, 0, codes, scales)
    ogq.ogq_act8_decode(codes, scales, T, C, BF, y, C)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (y, dx, dw, db, dg, dbe)]
step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dw, db, dg, dbe))) and float(dw.abs().max()) > 0
del graph
print("same")
"""


def test_captured_by_the_first_calls_of_a_process():
    r = subprocess.run([sys.executable, "-c", FIRST], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("cols", [64, 33])
def test_random_rounding_of_a_gate_has_numbers_of_its_own(dtype, cols):
    """d_up is rounded with counters whose third word is 1; the activation's input as the encoder alone does it."""
    import act8_reference as ref

    d, dt = DTYPES[dtype]
    rows = 6
    gen = torch.Generator(device="cuda").manual_seed(8)
    x, up = (torch.randn(rows, cols, device="cuda", generator=gen).to(dt) for _ in range(2))
    y = torch.empty_like(x)
    k = [kept(rows, cols) for _ in range(2)]
    ogq.ogq_act8_forward(x, cols, up, cols, rows, cols, d, ogq.OGQ_ACT_RELU, ogq.OGQ_ROUND_RANDOM, 12345, 6, y, cols, *k[0], *k[1])
    for t, (codes, scales), which in ((x, k[0], 0), (up, k[1], 1)):
        wc, ws = ref.encode(t.float().cpu().numpy(), (12345, 6, which))
        assert (codes.cpu().numpy() == wc).all() and (scales.cpu().numpy() == ws).all()


@pytest.mark.parametrize("N,P,C,G", [(2, 9000, 32, 4), (40, 3000, 64, 8), (1, 30, 64, 8), (3, 50, 40, 8)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_group_norm_keeps_what_the_encoder_keeps(dtype, N, P, C, G):
    """Streamed, resident and by the encoder itself: the same codes, rounded to nearest and at random."""
    d, dt = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn(N * P, C, device="cuda", generator=gen).to(dt)
    x[5, 3] = float("nan")
    ws = torch.empty(ogq.ogq_group_norm_workspace_bytes(N, P, C, G), dtype=torch.uint8, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
    for rounding in (ogq.OGQ_ROUND_NEAREST, ogq.OGQ_ROUND_RANDOM):
        a, b = kept(N * P, C), kept(N * P, C)
        ogq.ogq_group_norm_forward(x, N, P, C, G, d, None, None, 1e-5, ogq.OGQ_ACT_GELU, rounding, 77, 1, y, mean, rstd, *a, ws, ws.numel())
        ogq.ogq_act8_encode(x, C, N * P, C, d, rounding, 77, 1, *b)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("N,P,C,G", [(2, 9000, 32, 4), (1, 30, 64, 8), (3, 50, 40, 8)])
def test_group_norm_with_codes_at_an_odd_address(N, P, C, G):
    """The same results as with aligned codes: forward bit for bit, backward up to the order of the additions."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    x, dy = (torch.randn(N * P, C, device="cuda", generator=gen).bfloat16() for _ in range(2))
    ws = torch.empty(ogq.ogq_group_norm_workspace_bytes(N, P, C, G), dtype=torch.uint8, device="cuda")
    got = []
    for shift in (0, 1):
        flat, bytes_ = torch.zeros(N * P * C + 16, dtype=torch.int8, device="cuda"), torch.zeros(N * P * 2 + 16, dtype=torch.uint8, device="cuda")
        codes, scales = flat[shift:shift + N * P * C], bytes_[shift:shift + N * P * (-(-C // 32))]
        y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
        dg, db = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        ogq.ogq_group_norm_forward(x, N, P, C, G, BF, None, None, 1e-5, ogq.OGQ_ACT_SILU, 0, 0, 0, y, mean, rstd, codes, scales, ws, ws.numel())
        ogq.ogq_group_norm_backward(dy, None, codes, scales, N, P, C, G, BF, None, None, ogq.OGQ_ACT_SILU, mean, rstd, dx, dg, db, ws, ws.numel())
        got.append((codes.clone(), scales.clone(), y, dx, dg, db))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    for i, tol in ((2, 2.0 ** -7), (3, 2.0 ** -6), (4, 1e-4), (5, 1e-4)):
        a, b = got[0][i].float(), got[1][i].float()
        assert float((a - b).abs().max()) <= tol * (float(a.abs().max()) + 1), i
