"""Activations in 8 bits, group norm and weight gradient: the reference against brute force and differences, sizes, and every
refusal that a call makes before it touches the device (no GPU needed)."""
import math

import numpy as np
import pytest

import act8_reference as ref
import paper_2002_11082_b200 as ogq

P = 4096  # an address that is never dereferenced: the checks come first
INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3


def code(f, *args):
    with pytest.raises(ogq.OgqError) as e:
        f(*args, stream=0)
    return e.value.code


def test_groups():
    assert [ogq.ogq_act8_groups(c) for c in (-1, 0, 1, 31, 32, 33, 64, 1001)] == [-1, 0, 1, 1, 1, 2, 2, 32]


def test_the_unit_is_the_smallest_that_holds_the_group():
    for amax in (0.0, 1e-45, 1e-38, 0.5, 1.0, 127.0, np.nextafter(np.float32(127), np.float32(200)), 254.0, 3e38, float(np.finfo(np.float32).max)):
        b = ref.byte_of(float(amax))
        e = b - 127
        assert -120 <= e <= 121
        if e < 121:
            assert amax <= 127 * 2.0 ** e
        if e > -120:
            assert amax > 127 * 2.0 ** (e - 1)
    assert ref.byte_of(math.inf) == 255 and ref.byte_of(math.nan) == 255


def test_kept_values_are_bf16_numbers():
    for b in (7, 127, 248):
        v = (np.arange(-127, 128) * ref.unit(b)).astype(np.float32)
        assert np.all(v.astype(np.float64) == np.arange(-127, 128) * ref.unit(b))
        assert np.all((v.view(np.uint32) & 0xFFFF) == 0)


@pytest.mark.parametrize("act", [ref.NONE, ref.SILU, ref.GELU])
def test_reference_slopes_against_differences(act):
    z, h = np.linspace(-6, 6, 97), 1e-5
    d = (ref.value(act, z + h) - ref.value(act, z - h)) / (2 * h)
    assert np.max(np.abs(d - ref.slope(act, z))) < 1e-9


def test_reference_group_norm_gradient_against_differences():
    rng = np.random.default_rng(3)
    N, Px, C, G, eps = 2, 5, 6, 2, 1e-3
    x, dy = rng.normal(size=(N, Px, C)), rng.normal(size=(N, Px, C))
    gamma, beta = rng.normal(size=C), rng.normal(size=C)

    def loss(x, gamma, beta):
        mean, rstd = ref.group_stats(x, G, eps)
        return float((dy * ref.value(ref.SILU, (x - ref.wide(mean, C)) * ref.wide(rstd, C) * gamma + beta)).sum())

    mean, rstd = ref.group_stats(x, G, eps)
    dx, dgamma, dbeta, _, _ = ref.group_norm_backward(dy, x, mean, rstd, gamma, beta, G, ref.SILU)
    h = 1e-6
    for at in [(0, 0, 0), (1, 4, 5), (0, 2, 3)]:
        e = np.zeros_like(x)
        e[at] = h
        assert abs((loss(x + e, gamma, beta) - loss(x - e, gamma, beta)) / (2 * h) - dx[at]) < 1e-7
    for c in range(C):
        e = np.zeros(C)
        e[c] = h
        assert abs((loss(x, gamma + e, beta) - loss(x, gamma - e, beta)) / (2 * h) - dgamma[c]) < 1e-7
        assert abs((loss(x, gamma, beta + e) - loss(x, gamma, beta - e)) / (2 * h) - dbeta[c]) < 1e-7


def test_random_rounding_of_the_reference_is_unbiased():
    x = np.array([[0.3, -0.7, 1.9, -2.2, 100.0, 0.01, -99.7, 5.5]], np.float32)
    n = 2000
    mean = np.mean([ref.decode(*ref.encode(x, (s, 9, 0))) for s in range(n)], axis=0)
    unit = ref.unit(ref.byte_of(100.0))
    assert np.max(np.abs(mean - x)) < 5 * 0.5 * unit / math.sqrt(n)  # five standard deviations of a sum of n roundings, each at most unit / 2


def test_encode_refuses():
    f, bf, near = ogq.ogq_act8_encode, ogq.OGQ_BF16, ogq.OGQ_ROUND_NEAREST
    good = [P, 64, 4, 64, bf, near, 0, 0, P, P]

    def bad(**kw):
        a = list(good)
        for k, v in kw.items():
            a[int(k[1:])] = v
        return code(f, *a)

    assert bad(_0=None) == INVALID and bad(_8=None) == INVALID and bad(_9=None) == INVALID
    assert bad(_0=P + 1) == INVALID          # bf16 at an odd address
    assert bad(_1=63) == INVALID             # rows overlap
    assert bad(_2=-1) == INVALID and bad(_3=-1) == INVALID
    assert bad(_4=3) == INVALID and bad(_4=-1) == INVALID and bad(_5=2) == INVALID
    assert bad(_2=1 << 31) == UNSUPPORTED and bad(_2=1 << 30, _3=96, _1=96) == UNSUPPORTED
    assert bad(_4=ogq.OGQ_F32, _0=P + 2) == INVALID
    f(None, 0, 0, 64, bf, near, 0, 0, None, None, stream=0)  # nothing to do
    f(None, 0, 4, 0, bf, near, 0, 0, None, None, stream=0)


def test_decode_refuses():
    f = ogq.ogq_act8_decode
    assert code(f, None, P, 4, 64, ogq.OGQ_F16, P, 64) == INVALID
    assert code(f, P, None, 4, 64, ogq.OGQ_F16, P, 64) == INVALID
    assert code(f, P, P, 4, 64, ogq.OGQ_F16, None, 64) == INVALID
    assert code(f, P, P, 4, 64, 7, P, 64) == INVALID
    assert code(f, P, P, 4, 64, ogq.OGQ_F32, P, 32) == INVALID
    assert code(f, P, P, 1 << 31, 1, ogq.OGQ_F32, P, 1) == UNSUPPORTED
    f(None, None, 0, 64, ogq.OGQ_F32, None, 0, stream=0)


def test_pointwise_refuses():
    f, bf, silu = ogq.ogq_act8_forward, ogq.OGQ_BF16, ogq.OGQ_ACT_SILU
    good = [P, 64, P, 64, 4, 64, bf, silu, 0, 0, 0, P, 64, P, P, P, P]
    for i, v, want in ((0, None, INVALID), (11, None, INVALID), (13, None, INVALID), (14, None, INVALID), (15, None, INVALID), (16, None, INVALID),
                       (1, 8, INVALID), (3, 8, INVALID), (12, 8, INVALID), (6, 9, INVALID), (7, 4, INVALID), (7, -1, INVALID), (8, 2, INVALID),
                       (2, None, INVALID),  # codes of a gate without a gate
                       (11, P + 1, INVALID), (2, P + 1, INVALID), (1, 1 << 40, INVALID)):
        a = list(good)
        a[i] = v
        assert code(f, *a) == want, (i, v)
    b = ogq.ogq_act8_backward
    good = [P, 64, P, P, P, P, 4, 64, bf, silu, P, 64, P, 64]
    for i, v, want in ((0, None, INVALID), (2, None, INVALID), (3, None, INVALID), (4, None, INVALID), (5, None, INVALID), (10, None, INVALID),
                       (12, None, INVALID), (1, 63, INVALID), (11, 63, INVALID), (13, 63, INVALID), (8, 5, INVALID), (9, 9, INVALID),
                       (6, -4, INVALID), (6, 1 << 32, UNSUPPORTED)):
        a = list(good)
        a[i] = v
        assert code(b, *a) == want, (i, v)


def test_wgrad_refuses():
    f = ogq.ogq_act8_wgrad
    good = [P, 64, P, P, 16, 32, 64, ogq.OGQ_BF16, 0, P, P, P, 1 << 40]
    for i, v, want in ((0, None, INVALID), (1, 63, INVALID), (2, None, INVALID), (3, None, INVALID), (4, -1, INVALID), (5, -1, INVALID),
                       (6, -1, INVALID), (7, 3, INVALID), (8, 2, INVALID), (9, None, INVALID), (9, P + 2, INVALID), (10, P + 2, INVALID),
                       (4, 1 << 31, UNSUPPORTED), (6, 1 << 31, UNSUPPORTED)):
        a = list(good)
        a[i] = v
        assert code(f, *a) == want, (i, v)
    assert ogq.ogq_act8_wgrad_workspace_bytes(16, 32, 64, 5) == 0
    assert ogq.ogq_act8_wgrad_workspace_bytes(-1, 32, 64, 0) == 0
    assert ogq.ogq_act8_wgrad_workspace_bytes(100352, 64, 256, ogq.OGQ_BF16) > 0
    for rows, cols, out in ((0, 32, 64), (16, 0, 64), (16, 32, 0), (0, 0, 0), (1, 1, 1)):
        for d in (ogq.OGQ_F32, ogq.OGQ_F16, ogq.OGQ_BF16):
            assert ogq.ogq_act8_wgrad_workspace_bytes(rows, cols, out, d) >= 256


def test_group_norm_refuses():
    f, bf = ogq.ogq_group_norm_forward, ogq.OGQ_BF16
    good = [P, 2, 9, 64, 8, bf, P, P, 1e-5, 0, 0, 0, 0, P, P, P, P, P, P, 1 << 40]
    for i, v, want in ((0, None, INVALID), (1, -1, INVALID), (2, -1, INVALID), (3, -1, INVALID), (4, 0, INVALID), (4, 7, INVALID), (5, 4, INVALID),
                       (6, P + 2, INVALID), (8, 0.0, INVALID), (8, -1.0, INVALID), (8, math.nan, INVALID), (8, math.inf, INVALID), (9, 4, INVALID),
                       (10, 3, INVALID), (13, None, INVALID), (14, None, INVALID), (15, None, INVALID), (16, None, INVALID), (17, None, INVALID),
                       (18, None, WORKSPACE), (18, P + 128, WORKSPACE), (19, 16, WORKSPACE), (2, 1 << 31, UNSUPPORTED), (1, 1 << 31, UNSUPPORTED),
                       (2, 1 << 28, UNSUPPORTED), (1, 1 << 30, UNSUPPORTED)):
        a = list(good)
        a[i] = v
        assert code(f, *a) == want, (i, v)
    f(None, 0, 9, 64, 8, bf, None, None, 1e-5, 0, 0, 0, 0, None, None, None, None, None, None, 0, stream=0)
    b = ogq.ogq_group_norm_backward
    good = [P, None, P, P, 2, 9, 64, 8, bf, P, P, 0, P, P, P, P, P, P, 1 << 40]
    for i, v, want in ((0, None, INVALID), (1, P, INVALID), (2, None, INVALID), (3, None, INVALID), (7, 5, INVALID), (8, 3, INVALID), (11, 7, INVALID),
                       (12, None, INVALID), (13, None, INVALID), (14, None, INVALID), (15, P + 1, INVALID), (17, P + 1, WORKSPACE), (18, 8, WORKSPACE)):
        a = list(good)
        a[i] = v
        assert code(b, *a) == want, (i, v)
    a = list(good)
    a[2] = a[3] = None  # neither x nor codes
    assert code(b, *a) == INVALID
    assert ogq.ogq_group_norm_workspace_bytes(2, 9, 64, 7) == 0 and ogq.ogq_group_norm_workspace_bytes(2, 9, 64, 8) > 0


def test_c_types_of_the_new_calls_match_the_binding():
    """The header's parameter lists against the C module's signatures, name by name."""
    import os
    import re

    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "ogq.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    for name in ("ogq_act8_encode", "ogq_act8_decode", "ogq_act8_forward", "ogq_act8_backward", "ogq_act8_wgrad", "ogq_group_norm_forward",
                 "ogq_group_norm_backward"):
        params = re.search(name + r"\s*\(([^)]*)\)", text).group(1)
        names = [re.search(r"(\w+)\s*$", p.strip()).group(1) for p in params.split(",")]
        assert names == re.match(r"\((.*)\)", getattr(ogq, name).__text_signature__).group(1).replace("=None", "").split(", "), name
