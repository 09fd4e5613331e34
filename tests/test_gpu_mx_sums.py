"""Products of microscaled operands where the order and the width of the sums show."""
import numpy as np
import pytest

from oracle import mx as ref
from test_gpu_mx import DT, FMT, KIND, f64, operand, resid_of, run_linear, weights

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def cancelling(rng, M, N, K, wide):
    """Rows whose large products cancel in pairs of neighbouring columns, and one small element that is left: in every
    block of 32 a pair of +-448 (e4m3's largest code and its scale 1), in one block of a row a code of 2^-9 .. 15 2^-9 in
    the pair's group of eight.  W's columns are equal where x's cancel."""
    x, w = np.zeros((M, K)), rng.choice([0.5, -1.0, 1.5, 2.0, -3.0, 4.0, -6.0], (wide, K))
    w[:, 1::8], w[:, 3::8] = w[:, 0::8], w[:, 2::8]
    sign = rng.choice([-1.0, 1.0], (M, K // 32))
    x[:, 0::32], x[:, 1::32] = 448 * sign, -448 * sign
    x[:, 10::32], x[:, 11::32] = -448 * sign, 448 * sign
    at = rng.integers(0, K // 32, M)
    rows = np.arange(M)
    x[rows, at * 32 + 6] = rng.integers(1, 16, M) * 2.0 ** -9
    return x, w


def silu_product(z, N):
    return z[:, :N] / (1 + np.exp(-z[:, :N])) * z[:, N:]


# rows, outputs: each kernel of few rows (W of up to 8192 rows or more), and tiles
FEW = [(1, 40), (4, 8300), (32, 512), (33, 512), (48, 8300), (64, 96)]
MANY = [(65, 40), (100, 8300), (128, 96), (200, 512), (330, 1300)]


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("M,N", FEW + MANY)
def test_products_that_cancel_leave_the_small_ones(kind, M, N):
    K = 544
    rng = np.random.default_rng(M + N)
    wide = 2 * N if kind == "swiglu" else N
    x, w = cancelling(rng, M, N, K, wide)
    a, av = operand(x, "e4m3")
    assert np.array_equal(av, x)
    wt, wv = weights(w, kind, N)
    assert np.array_equal(wv, w)
    z = av @ wv.T                                             # one product of 4 by 2 bits: exact in every type
    assert np.array_equal(z, (av * (np.abs(av) < 1)) @ wv.T) and (z != 0).all()
    for dtype in DT:
        r = resid_of(rng, kind, dtype, M, N)
        if r is not None:
            r.zero_()
        out = f64(run_linear(a, wt, r, kind, dtype, "e4m3", M, N, K))
        f32_out = dtype == "f32" or kind == "resid"
        half = 2.0 ** -24 if f32_out else 2.0 ** -8
        if f32_out or M <= 64:
            cut = 0.0
        else:
            # per group of eight: 2^-13 of the largest of eight terms each; no other error than that
            cut = 8 * 2.0 ** -13 * 448 * 6 * 2 * (K // 32) * np.ones_like(z)
        if kind == "swiglu":
            want, g, u = silu_product(z, N), np.abs(z[:, :N]), np.abs(z[:, N:])
            cg = cut if np.isscalar(cut) else cut[:, :N]
            # silu's slope is at most 1.1; its own steps as an fp32 function: |g| + 8 of them at most
            tol = (1.1 * cg + np.abs(g) * (g + cg + 8) * 2.0 ** -23) * (u + cg) + 1.1 * (g + cg) * cg
        elif kind == "gelu":
            from scipy.special import ndtr
            want, tol = z * ndtr(z), 1.13 * cut + np.abs(z) * 4 * 2.0 ** -23
        else:
            want, tol = z, cut
        tol = tol + half * (np.abs(want) + tol) + 2.0 ** -133
        if kind in ("swiglu", "gelu") or not np.isscalar(cut):
            assert (np.abs(out - want) <= tol).all(), (dtype, float((np.abs(out - want) / tol).max()))
        else:
            assert np.array_equal(out, want), (dtype, float(np.abs(out - want).max()))


@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
@pytest.mark.parametrize("M,N", [(4, 40), (100, 96), (330, 200)])
def test_swiglu_of_far_negative_gates(fmt, M, N):
    """Gates down to -88.6, whose silu fp32 still holds as a normal number."""
    K = 64
    x, w = np.zeros((M, K)), np.zeros((2 * N, K))
    x[:, 0] = np.resize([56.0, 48.0, 40.0, 32.0] if fmt == "e4m3" else [48.0, 32.0, 24.0, 16.0], M)
    x[:, 1] = np.resize([4.5, 4.0, 3.5] if fmt == "e4m3" else [16.0], M)
    x[:, 32] = 1024.0
    w[:N, 0], w[:N, 1], w[N:, 32] = -np.resize([1.5, 1.0, 0.5], N), -1.0, np.resize([6.0, -2.0, 1.0], N)
    a, av = operand(x, fmt)
    assert np.array_equal(av, x)
    wt, wv = weights(w, "swiglu", N)
    z = av @ wv.T
    assert (z[:, :N] > -88.7).all() and (z[:, :N] < -87.4).any()
    want = silu_product(z, N)
    for dtype in DT:
        out = f64(run_linear(a, wt, None, "swiglu", dtype, fmt, M, N, K))
        half = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
        # the exponential of an fp32 argument, |z| steps of 2^-23, and eight more: the reciprocal's (a subnormal number of 21
        # bits: four), the products' and the exponential's own
        tol = np.abs(want) * ((np.abs(z[:, :N]) + 8) * 2.0 ** -23 + half)
        assert (np.abs(out - want) <= tol).all(), (dtype, float((np.abs(out - want) / tol).max()))
