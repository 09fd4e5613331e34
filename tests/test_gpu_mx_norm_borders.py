"""The norm into a microscaled operand at its codes' borders: the codes and scales
are those of the formula in 64 bits on the sum of x and delta as it is."""
import numpy as np
import pytest

from oracle import mx as ref
from test_gpu_mx import DT, FMT, f64, rows_of, run_norm

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# What a code may hang on.  The kernel and this file's formula hold squares, root and products in 64 bits: a sum of at
# most 24576 squares in any order that adds 12 x 8 of them in a row at most and ten partial ones is off by 106 x 2^-53
# of it, its root by half, and the root, the quotient and two products round by 2^-53 each: below 2^-46 on either side.
NEAR = 2.0 ** -45


def borders(fmt):
    """Halfway between neighbouring codes, in units of the scale."""
    g = ref.grid(fmt)[:8 if fmt == "e2m1" else 127]
    return (g[1:] + g[:-1]) / 2


def border_gains(fmt, cols):
    """Gains that put |h| r = 1 on borders of codes: per block one element that holds the scale (in every fourth block the
    largest code itself, the scale's border), then the borders in turn, of either sign.  Few bits each: bf16 holds them."""
    g = np.resize(borders(fmt), cols) * np.where(np.arange(cols) % 3 == 0, -1.0, 1.0)
    top = ref.TOP[fmt]
    first = np.arange(0, cols, 32)
    g[first] = np.where(first // 32 % 4 == 3, top, top * 0.75)
    return g[None]


def check_exact(y, codes, scales, fmt, cols):
    """Every code and scale of y in 64 bits, and none of them nearer than NEAR to a border."""
    want_c, want_s = ref.quantize(y, fmt)
    for f in (1 - NEAR, 1 + NEAR):
        c, s = ref.quantize(y * f, fmt)
        assert np.array_equal(c, want_c) and np.array_equal(s, want_s)
    nb = want_s.shape[1]
    wrong = ref.grid(fmt)[codes[:, :nb]] != ref.grid(fmt)[want_c]
    assert np.array_equal(scales[:, :nb], want_s), np.argwhere(scales[:, :nb] != want_s)[:4]
    assert not wrong.any(), (int(wrong.sum()), np.argwhere(wrong)[:4])


def formula(h, gain, eps):
    return h / np.sqrt(np.mean(h * h, -1, keepdims=True) + float(np.float32(eps))) * gain


@pytest.mark.parametrize("sdt,dt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
@pytest.mark.parametrize("rows,cols", [(3, 264), (33, 4096), (2, 24576)])
def test_the_part_of_the_sum_that_fp32_drops_counts(sdt, dt, fmt, rows, cols):
    """x + delta = 2^q (1 +- 2^-30): 2^q in fp32, and on either side of a code's border in 64 bits."""
    sign = np.where(np.arange(cols) % 2 == 0, 1.0, -1.0)
    scale = np.exp2(np.arange(rows) % 5 - 2.0)[:, None]
    x, d = scale * np.ones(cols), scale * sign * 2.0 ** -30
    gain = border_gains(fmt, cols)
    h, (codes, scales) = run_norm(rows_of(x, sdt), rows_of(d, dt), rows_of(gain, dt), sdt, dt, fmt, rows, cols, 2.0 ** -70)
    assert np.array_equal(f64(h), x)
    check_exact(formula(x + d, gain, 2.0 ** -70), codes, scales, fmt, cols)


@pytest.mark.parametrize("sdt,dt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
@pytest.mark.parametrize("bits", [26, 30, 34])
@pytest.mark.parametrize("side", [-1, 1])
def test_rows_just_beside_every_border(sdt, dt, fmt, bits, side):
    """|h| = 1 but for one element of 1/2, whose 3/4 / cols the mean lacks: eps makes up for them but for 2^-bits."""
    rows, cols = 5, 4096
    x = np.where(np.arange(cols) % 5 == 0, -1.0, 1.0) * np.ones((rows, 1))
    x[:, 32] = 0.5
    eps = 0.75 / cols - side * 2.0 ** -bits
    assert float(np.float32(eps)) == eps
    gain = border_gains(fmt, cols)
    for d in (None, x / 2):
        xs = x if d is None else x - d
        _, (codes, scales) = run_norm(rows_of(xs, sdt), None if d is None else rows_of(d, dt), rows_of(gain, dt), sdt, dt, fmt,
                                      rows, cols, eps)
        check_exact(formula(x, gain, eps), codes, scales, fmt, cols)


@pytest.mark.parametrize("sdt,dt", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
def test_random_rows_have_the_codes_of_64_bits(sdt, dt, fmt):
    """Four million elements, of which a few lie within fp32's roundings of a border."""
    rows, cols = 512, 8192
    g = torch.Generator(device="cuda").manual_seed(11)
    x = torch.randn((rows, cols), device="cuda", generator=g).mul_(4).to(DT[sdt][1])
    d = torch.randn((rows, cols), device="cuda", generator=g).to(DT[dt][1])
    gain = (1 + 0.1 * torch.randn((1, cols), device="cuda", generator=g)).to(DT[dt][1])
    _, (codes, scales) = run_norm(x, d, gain, sdt, dt, fmt, rows, cols, 1e-6)
    y = formula(f64(x) + f64(d), f64(gain), 1e-6)
    want_c, want_s = ref.quantize(y, fmt)
    (lo_c, lo_s), (hi_c, hi_s) = (ref.quantize(y * f, fmt) for f in (1 - NEAR, 1 + NEAR))
    sure = lo_s == hi_s
    assert np.array_equal(scales[sure], want_s[sure])
    sure = sure[..., None] & (lo_c == hi_c)
    assert sure.mean() > 1 - 1e-6
    assert np.array_equal(ref.grid(fmt)[codes][sure], ref.grid(fmt)[want_c][sure])


@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
def test_small_elements_under_large_gains(fmt):
    """Elements far below fp32's normal numbers once divided by the row's root, and gains that bring them back."""
    rows, cols = 7, 520
    rng = np.random.default_rng(2)
    x = rng.standard_normal((rows, cols))
    small = np.arange(cols) // 32 % 2 == 1
    x = np.where(small, x * 2.0 ** -40, x * 2.0 ** 100).astype(np.float32).astype(np.float64)
    gain = np.where(small, 2.0 ** 110, 1.0) * rng.uniform(1.0, 2.0, (1, cols))
    gain = gain.astype(np.float32).astype(np.float64)
    _, (codes, scales) = run_norm(rows_of(x, "f32"), None, rows_of(gain, "f32"), "f32", "f32", fmt, rows, cols, 1e-6)
    check_exact(formula(x, gain, 1e-6), codes, scales, fmt, cols)


@pytest.mark.parametrize("side", [-1, 1])
@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
def test_borders_of_the_smallest_codes(fmt, side):
    """Values at borders of codes of the least scale, 2^-127: subnormal numbers of fp32."""
    rows, cols = 3, 4096
    x = np.ones((rows, cols))
    x[:, 32] = 0.5
    eps = 0.75 / cols - side * 2.0 ** -30
    gain = border_gains(fmt, cols) * 2.0 ** -127
    gain[:, ::32] = (1.0 if fmt == "e2m1" else 64.0) * 2.0 ** -127
    _, (codes, scales) = run_norm(rows_of(x, "f32"), None, rows_of(gain, "f32"), "f32", "f32", fmt, rows, cols, eps)
    check_exact(formula(x, gain, eps), codes, scales, fmt, cols)


@pytest.mark.parametrize("fmt", ["e2m1", "e4m3"])
def test_rows_and_gains_of_the_largest_numbers(fmt):
    rows, cols = 4, 264
    rng = np.random.default_rng(3)
    x = (rng.uniform(0.5, 1.0, (rows, cols)) * 3.4e38).astype(np.float32).astype(np.float64)
    x[1] *= 2.0 ** -120
    gain = rng.uniform(0.5, 1.0, (1, cols)) * 1.5e38
    gain = gain.astype(np.float32).astype(np.float64)
    _, (codes, scales) = run_norm(rows_of(x, "f32"), None, rows_of(gain, "f32"), "f32", "f32", fmt, rows, cols, 1e-6)
    check_exact(formula(x, gain, 1e-6), codes, scales, fmt, cols)


def test_zeros_stay_zeros_of_their_sign():
    rows, cols = 3, 264
    x = np.zeros((rows, cols))
    x[1, ::2], x[2, 5:9] = -0.0, 1.0
    gain = np.ones((1, cols))
    gain[0, 7] = 0.0
    for fmt in FMT:
        h, (codes, scales) = run_norm(rows_of(x, "f32"), None, rows_of(gain, "f32"), "f32", "f32", fmt, rows, cols, 1e-6)
        assert np.array_equal(f64(h), x) and np.array_equal(np.signbit(f64(h)), np.signbit(x))
        check_exact(formula(x, gain, 1e-6), codes, scales, fmt, cols)
