"""The 8-bit activations as a training step uses them, together with the gradient codec: group norm that keeps its input, a gated unit
that keeps both of its, a linear layer whose input is kept, all gradients written into one bucket, the bucket encoded and decoded.
Also replayed as a graph on a stream of its own, and two steps at once on two streams."""
import numpy as np
import pytest
import torch

import act8_reference as ref
import oracle
import paper_2002_11082_b200 as ogq
from act8_gpu import assert_near

pytestmark = pytest.mark.gpu
BF = ogq.OGQ_BF16


class Step:
    """x [N, P, C] -> group norm, SiLU -> h = y V^T (2F wide) -> silu(gate) up -> u -> o = u W^T; gradients of W, bias, gamma, beta."""

    def __init__(self, N=2, P=50, C=64, G=8, F=96, O=40, seed=0):
        self.N, self.P, self.C, self.G, self.F, self.O = N, P, C, G, F, O
        T = N * P
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(s, device="cuda", generator=gen)  # noqa: E731
        new = lambda *s, dtype=torch.bfloat16: torch.zeros(s, device="cuda", dtype=dtype)  # noqa: E731
        self.x, self.do = rand(T, C).bfloat16(), rand(T, O).bfloat16()
        self.V, self.W = (rand(2 * F, C) / C ** 0.5).bfloat16(), (rand(O, F) / F ** 0.5).bfloat16()
        self.gamma, self.beta = 1 + 0.1 * rand(C), 0.1 * rand(C)
        self.y, self.h, self.u, self.o = new(T, C), new(T, 2 * F), new(T, F), new(T, O)
        self.du, self.dh, self.dyy, self.dx = new(T, F), new(T, 2 * F), new(T, C), new(T, C)
        kept = lambda c: (new(T, c, dtype=torch.int8), new(T, ref.groups(c), dtype=torch.uint8))  # noqa: E731
        self.kx, self.ky, self.kg, self.kup, self.ku = kept(C), kept(C), kept(F), kept(F), kept(F)
        f32 = torch.float32
        self.mean, self.rstd = new(N, G, dtype=f32), new(N, G, dtype=f32)
        sizes = [2 * F * C, 2 * F, O * F, O, C, C]
        self.n = sum(sizes)
        self.bucket = new(self.n, dtype=f32)
        self.dV, self.dVb, self.dW, self.db, self.dgamma, self.dbeta = self.bucket.split(sizes)
        self.ws = torch.empty(max(ogq.ogq_act8_wgrad_workspace_bytes(T, C, 2 * F, BF), ogq.ogq_act8_wgrad_workspace_bytes(T, F, O, BF),
                                  ogq.ogq_group_norm_workspace_bytes(N, P, C, G)), dtype=torch.uint8, device="cuda")
        self.d = 128
        nb = -(-self.n // self.d)
        self.levels, self.status = new(nb, 9, dtype=f32), new(nb, dtype=torch.int32)
        self.packed = new(ogq.ogq_bucket_packed_words(self.n, self.d, 4), dtype=torch.int32)
        self.avg = new(self.n, dtype=f32)
        self.pk, self.pl = ogq.device_pointer_array([self.packed]), ogq.device_pointer_array([self.levels])

    def run(self):
        T, F, C = self.N * self.P, self.F, self.C
        wsb = self.ws.numel()
        silu = ogq.OGQ_ACT_SILU
        ogq.ogq_group_norm_forward(self.x, self.N, self.P, C, self.G, BF, self.gamma, self.beta, 1e-5, silu, 0, 0, 0, self.y, self.mean, self.rstd,
                                   *self.kx, self.ws, wsb)
        ogq.ogq_act8_encode(self.y, C, T, C, BF, 0, 0, 0, *self.ky)
        torch.matmul(self.y, self.V.t(), out=self.h)
        ogq.ogq_act8_forward(self.h, 2 * F, self.h[:, F:], 2 * F, T, F, BF, silu, 0, 0, 0, self.u, F, *self.kg, *self.kup)
        ogq.ogq_act8_encode(self.u, F, T, F, BF, 0, 0, 0, *self.ku)
        torch.matmul(self.u, self.W.t(), out=self.o)
        # backward
        ogq.ogq_act8_wgrad(self.do, self.O, *self.ku, T, F, self.O, BF, 0, self.dW, self.db, self.ws, wsb)
        torch.matmul(self.do, self.W, out=self.du)
        ogq.ogq_act8_backward(self.du, F, *self.kg, *self.kup, T, F, BF, silu, self.dh, 2 * F, self.dh[:, F:], 2 * F)
        ogq.ogq_act8_wgrad(self.dh, 2 * F, *self.ky, T, C, 2 * F, BF, 0, self.dV, self.dVb, self.ws, wsb)
        torch.matmul(self.dh, self.V, out=self.dyy)
        ogq.ogq_group_norm_backward(self.dyy, None, *self.kx, self.N, self.P, C, self.G, BF, self.gamma, self.beta, silu, self.mean, self.rstd, self.dx,
                                    self.dgamma, self.dbeta, self.ws, wsb)
        # the gradient bucket, onto the wire and back
        ogq.ogq_bucket_encode(self.bucket, self.n, self.d, ogq.OGQ_ORQ, 9, 0, 0.0, 5, 0, self.levels, None, self.status, self.packed)
        ogq.ogq_bucket_decode_sum(self.pk, self.pl, 1, self.n, self.d, 9, 1.0, self.avg)

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in (self.y, self.u, self.dh, self.dx, self.bucket, self.packed, self.avg)]


def check(s: Step):
    """Every link against its definition in 64 bits on what the link before it wrote.  bf16 results: half a step of 2^-8 and the functions'
    own errors, together below 0.6 of a step; sums of T fp32 products: T + 64 steps of 2^-24 of the sum of magnitudes."""
    N, P, C, G, F = s.N, s.P, s.C, s.G, s.F
    T = N * P
    torch.cuda.synchronize()
    f64 = lambda t: t.double().cpu().numpy()  # noqa: E731
    back = lambda k: ref.decode(k[0].cpu().numpy(), k[1].cpu().numpy())  # noqa: E731
    for kept, full in ((s.kx, s.x), (s.ky, s.y), (s.kg, s.h[:, :F]), (s.kup, s.h[:, F:]), (s.ku, s.u)):
        wc, wsc = ref.encode(full.float().cpu().numpy())
        assert np.array_equal(kept[0].cpu().numpy(), wc) and np.array_equal(kept[1].cpu().numpy(), wsc)
    x = f64(s.x).reshape(N, P, C)
    mean, rstd = ref.group_stats(x, G, 1e-5)
    gamma, beta = f64(s.gamma), f64(s.beta)
    y = ref.value(ref.SILU, (x - ref.wide(mean, C)) * ref.wide(rstd, C) * gamma + beta).reshape(T, C)
    near = lambda want: np.abs(want) * 0.6 * 2.0 ** -7 + 3e-5  # noqa: E731
    assert_near(f64(s.y), y, near(y), "y")
    h = f64(s.h)
    u = ref.value(ref.SILU, h[:, :F]) * h[:, F:]
    assert_near(f64(s.u), u, near(u), "u")
    du, kg, kup = f64(s.du), back(s.kg), back(s.kup)
    dh = np.concatenate([du * kup * ref.slope(ref.SILU, kg), du * ref.value(ref.SILU, kg)], 1)
    assert_near(f64(s.dh), dh, near(dh), "dh")
    steps = (T + 64) * 2.0 ** -24
    for dy, kept, dw, db in ((s.do, s.ku, s.dW, s.db), (s.dh, s.ky, s.dV, s.dVb)):
        d, k = f64(dy), back(kept)
        assert_near(f64(dw).reshape(d.shape[1], -1), d.T @ k, np.abs(d).T @ np.abs(k) * steps, "dw")
        assert_near(f64(db), d.sum(0), np.abs(d).sum(0) * steps, "db")
    dx, dgamma, dbeta, xh, dz = ref.group_norm_backward(f64(s.dyy).reshape(N, P, C), back(s.kx).reshape(N, P, C), f64(s.mean), f64(s.rstd), gamma, beta,
                                                        G, ref.SILU)
    assert_near(f64(s.dx), dx.reshape(T, C), near(dx.reshape(T, C)), "dx")
    wide = np.abs(f64(s.dyy)).sum(0) * 2e-5  # the slope's error and the sums' (tests of the group norm)
    assert_near(f64(s.dgamma), dgamma, wide * np.abs(xh).max() * 1.2, "dgamma")
    assert_near(f64(s.dbeta), dbeta, wide, "dbeta")
    b = s.bucket.cpu().numpy()
    off = np.minimum(np.arange(-(-s.n // s.d) + 1, dtype=np.int64) * s.d, s.n)
    w_lv, _ = oracle.bucket_levels_orq(b, off, 9)
    w_pk, _ = oracle.bucket_quantize_pack(b, off, oracle.ORQ, 9, w_lv, None, 5, 0)
    assert np.array_equal(s.levels.cpu().numpy(), w_lv) and np.array_equal(s.packed.cpu().numpy().view(np.uint32), w_pk)
    assert np.array_equal(s.avg.cpu().numpy(), oracle.bucket_unpack_sum([w_pk], [w_lv], off, 9, 1.0))


@pytest.mark.parametrize("sizes", [{}, {"N": 1, "P": 1}, {"N": 3, "P": 37, "C": 40, "G": 5, "F": 33, "O": 7}, {"N": 4, "P": 300, "C": 128, "F": 256, "O": 136}])
def test_a_step(sizes):
    s = Step(**sizes)
    s.run()
    check(s)


def test_replayed_as_a_graph_and_on_other_streams():
    s = Step(seed=1)
    s.run()
    want = s.results()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            s.run()
    for t in (s.y, s.u, s.dh, s.dx, s.bucket, s.packed, s.avg):
        t.zero_()
    s.ws.fill_(0xA5)
    graph.replay()
    for a, b in zip(want, s.results()):
        assert torch.equal(a, b)
    # another input of the same sizes through the same graph
    other = Step(seed=2)
    other.run()
    for name in ("x", "do", "V", "W", "gamma", "beta"):
        getattr(s, name).copy_(getattr(other, name))
    graph.replay()
    for a, b in zip(other.results(), s.results()):
        assert torch.equal(a, b)
    del graph


def test_two_steps_at_once():
    steps = [Step(seed=k, P=400) for k in (3, 4)]
    want = []
    for s in steps:
        s.run()
        want.append(s.results())
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, st in zip(steps, streams):
            with torch.cuda.stream(st):
                s.run()
    for s, w in zip(steps, want):
        for a, b in zip(w, s.results()):
            assert torch.equal(a, b)
