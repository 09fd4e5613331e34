"""Microscaled operands on the host: sizes and layout, every refusal (found before
any launch: no GPU needed), and pins of their oracle."""
import ctypes as ct
import os
import re

import numpy as np
import pytest

from oracle import mx as ref
from paper_2308_16369_amd import sarathi as S

A, B, C, D, E = (0x10000000 * i for i in range(1, 6))   # never dereferenced: validation fails first
BIG = 1 << 27


def test_every_function_of_the_header_is_bound():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "include", "sarathi_mx.h")) as f:
        names = set(re.findall(r"\b(sarathi_mx_\w+)\s*\(", re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)))
    assert names and all(n in S.EXPORTS and getattr(S.lib(), n) and getattr(S, n) for n in names), names


@pytest.mark.parametrize("fmt,name", [(S.MX_E2M1, "e2m1"), (S.MX_E4M3, "e4m3")])
@pytest.mark.parametrize("rows,cols", [(1, 8), (32, 256), (33, 264), (70, 1000)])
def test_layout(fmt, name, rows, cols):
    L = S.sarathi_mx_get_layout(fmt, rows, cols)
    nb = -(-cols // 32)
    codes = np.arange(rows * nb * 32).reshape(rows, nb, 32) % (16 if fmt == S.MX_E2M1 else 251)
    scales = (np.arange(rows * nb).reshape(rows, nb) % 249).astype(np.uint8)
    buf = ref.pack(codes.astype(np.uint8), scales, name)
    assert len(buf) == L.total == S.sarathi_mx_bytes(fmt, rows, cols)
    bits = 4 if fmt == S.MX_E2M1 else 8
    for r in {0, rows - 1, rows // 2}:
        for c in {0, cols - 1, cols // 2, min(cols - 1, 31)}:
            bit = c * bits
            at = r // 32 * L.tile + bit // 128 * L.unit + r % 32 * L.row + bit % 128 // 8
            assert (buf[at] >> (bit % 8)) & ((1 << bits) - 1) == codes[r, c // 32, c % 32]
            b = c // 32
            at = (L.scale_offset + r // 32 * L.scale_tile + b // 8 * L.scale_cols + b % 2 * L.scale_half +
                  r % 32 * L.scale_row + b % 8 // 2)
            assert buf[at] == scales[r, b]
    got = ref.unpack(buf, name, rows, cols)
    assert np.array_equal(got[0][:, :nb], codes) and np.array_equal(got[1][:, :nb], scales)


def test_bytes_of_bad_arguments():
    for args in [(2, 4, 64), (-1, 4, 64), (0, 0, 64), (0, 4, 0), (0, -1, 64), (0, 2 ** 31 - 1, 2 ** 28)]:
        assert S.sarathi_mx_bytes(*args) == 0
    assert S.sarathi_mx_bytes(0, 1 << 20, 1 << 15) == (1 << 34) + (1 << 30)     # beyond 32 bits
    assert S.lib().sarathi_mx_get_layout(0, 4, 64, None) == S.EINVAL
    assert S.sarathi_mx_linear_scratch_bytes(0, 8) == S.sarathi_mx_linear_scratch_bytes(8, 0) == 0


QUANT = dict(dtype=S.BF16, format=S.MX_E2M1, rows=40, cols=64, x=A, ld_x=64, operand=B, operand_bytes=BIG)
BAD_QUANT = [
    (dict(dtype=2), S.EUNSUPPORTED), (dict(format=2), S.EUNSUPPORTED), (dict(format=-1), S.EUNSUPPORTED),
    (dict(rows=0), S.EINVAL), (dict(cols=0), S.EINVAL), (dict(cols=-8), S.EINVAL), (dict(cols=60), S.EUNSUPPORTED),
    (dict(rows=2 ** 31 - 1, cols=2 ** 20, ld_x=2 ** 20), S.EUNSUPPORTED), (dict(x=0), S.EINVAL), (dict(x=A + 8), S.EINVAL),
    (dict(ld_x=56), S.EINVAL), (dict(ld_x=68), S.EINVAL), (dict(ld_x=2 ** 33), S.EINVAL), (dict(operand=0), S.EINVAL),
    (dict(operand=B + 4), S.EINVAL), (dict(operand_bytes=0), S.ENOSPC),
    (dict(operand_bytes=S.sarathi_mx_bytes(S.MX_E2M1, 40, 64) - 1), S.ENOSPC), (dict(operand=A), S.EINVAL),
    (dict(operand=A + 39 * 128 + 112), S.EINVAL), (dict(dtype=S.F32, ld_x=66), S.EINVAL),
]


@pytest.mark.parametrize("kw,code", BAD_QUANT, ids=[str(i) for i in range(len(BAD_QUANT))])
def test_quantize_and_dequantize_refuse(kw, code):
    a = {**QUANT, **kw}
    assert S.sarathi_mx_quantize(**a, check=False) == code, S.sarathi_last_error()
    assert S.sarathi_mx_dequantize(a["format"], a["rows"], a["cols"], a["operand"], a["operand_bytes"], a["dtype"], a["x"],
                                   a["ld_x"], check=False) == code, S.sarathi_last_error()


NORM = dict(stream_dtype=S.F32, dtype=S.BF16, format=S.MX_E4M3, rows=40, cols=64, eps=1e-6, x=A, ld_x=64, delta=B,
            ld_delta=64, gain=C, h_out=D, ld_h=64, operand=E, operand_bytes=BIG)
BAD_NORM = [
    (dict(stream_dtype=2), S.EUNSUPPORTED), (dict(dtype=-1), S.EUNSUPPORTED),
    (dict(stream_dtype=S.BF16, dtype=S.F32), S.EUNSUPPORTED), (dict(format=3), S.EUNSUPPORTED), (dict(rows=0), S.EINVAL),
    (dict(cols=0), S.EINVAL), (dict(cols=20), S.EUNSUPPORTED), (dict(rows=2 ** 24 - 255), S.EUNSUPPORTED),
    (dict(cols=24584, ld_x=24584, ld_delta=24584, ld_h=24584), S.EUNSUPPORTED), (dict(eps=0.0), S.EINVAL),
    (dict(eps=-1.0), S.EINVAL), (dict(eps=float("nan")), S.EINVAL), (dict(eps=float("inf")), S.EINVAL),
    (dict(x=0), S.EINVAL), (dict(x=A + 4), S.EINVAL), (dict(ld_x=32), S.EINVAL), (dict(delta=B + 2), S.EINVAL),
    (dict(ld_delta=63), S.EINVAL), (dict(gain=0), S.EINVAL), (dict(gain=C + 8), S.EINVAL), (dict(h_out=D + 8), S.EINVAL),
    (dict(ld_h=65), S.EINVAL), (dict(operand=0), S.EINVAL), (dict(operand_bytes=64), S.ENOSPC),
    (dict(h_out=A, ld_h=72), S.EINVAL), (dict(h_out=A + 256), S.EINVAL), (dict(h_out=B), S.EINVAL),
    (dict(h_out=C), S.EINVAL), (dict(operand=A), S.EINVAL), (dict(operand=B), S.EINVAL), (dict(operand=C), S.EINVAL),
    (dict(operand=D), S.EINVAL),
]


@pytest.mark.parametrize("kw,code", BAD_NORM, ids=[str(i) for i in range(len(BAD_NORM))])
def test_norm_refuses(kw, code):
    assert S.sarathi_mx_norm(**{**NORM, **kw}, check=False) == code, S.sarathi_last_error()


LINEAR = dict(dtype=S.BF16, kind=S.LINEAR_RESID_F32IN, a_format=S.MX_E4M3, M=40, N=48, K=64, a=A, w=B, resid=C, out=D)
BAD_LINEAR = [
    (dict(dtype=2), S.EUNSUPPORTED), (dict(kind=-1), S.EINVAL), (dict(kind=5), S.EINVAL), (dict(a_format=2), S.EUNSUPPORTED),
    (dict(M=0), S.EINVAL), (dict(N=0), S.EINVAL), (dict(K=0), S.EINVAL), (dict(K=-8), S.EINVAL), (dict(K=36), S.EUNSUPPORTED),
    (dict(M=2 ** 31 - 1, N=2 ** 31 - 1), S.EUNSUPPORTED), (dict(M=2 ** 31 - 1, K=2 ** 20), S.EUNSUPPORTED),
    (dict(M=1, N=2 ** 28 - 31), S.EUNSUPPORTED), (dict(scratch=D, scratch_bytes=1 << 20, M=200), S.EINVAL),
    (dict(scratch=A, scratch_bytes=1 << 20, M=200), S.EINVAL), (dict(scratch=B, scratch_bytes=1 << 20, M=200), S.EINVAL),
    (dict(scratch=C, scratch_bytes=1 << 20, M=200), S.EINVAL),
    (dict(a=0), S.EINVAL), (dict(w=0), S.EINVAL), (dict(out=0), S.EINVAL), (dict(resid=0), S.EINVAL),
    (dict(kind=S.LINEAR_RESID, resid=0), S.EINVAL), (dict(a=A + 8), S.EINVAL), (dict(w=B + 4), S.EINVAL),
    (dict(out=D + 8), S.EINVAL), (dict(resid=C + 4), S.EINVAL), (dict(out=A), S.EINVAL), (dict(out=B), S.EINVAL),
    (dict(out=C), S.EINVAL), (dict(out=C + 64), S.EINVAL),
    (dict(kind=S.LINEAR_SWIGLU, out=B + S.sarathi_mx_bytes(S.MX_E2M1, 48, 64)), S.EINVAL),
]


@pytest.mark.parametrize("kw,code", BAD_LINEAR, ids=[str(i) for i in range(len(BAD_LINEAR))])
def test_linear_refuses(kw, code):
    assert S.sarathi_mx_linear(**{**LINEAR, **kw}, check=False) == code, S.sarathi_last_error()


def test_linear_plan():
    assert S.sarathi_mx_linear_scratch_bytes(64, 1 << 20) == 0
    full = S.sarathi_mx_linear_scratch_bytes(200, 5120)
    assert 0 < full <= 8 * 200 * 5120 * 4 and S.sarathi_mx_linear_scratch_bytes(4096, 28000) <= 64 << 20
    args = (S.BF16, S.LINEAR_PLAIN, S.MX_E2M1, 200, 5120, 13824)
    bm, bn, n = S.sarathi_mx_linear_plan(*args, full)
    assert n > 1 and n * 200 * 5120 * 4 <= full and S.sarathi_mx_linear_plan(*args, 0)[2] == 1
    assert S.sarathi_mx_linear_plan(*args, 2 * 200 * 5120 * 4)[2] <= 2
    assert S.sarathi_mx_linear_plan(S.BF16, S.LINEAR_SWIGLU, S.MX_E2M1, 200, 512, 13824, full)[2] == 1
    assert S.sarathi_mx_linear_plan(S.BF16, S.LINEAR_PLAIN, S.MX_E4M3, 1, 64, 64, 0) == (32, 32, 1)
    one = ct.c_int()
    lib = S.lib()
    assert lib.sarathi_mx_linear_plan(*args, 0, None, ct.byref(one), ct.byref(one)) == S.EINVAL
    for kw, code in BAD_LINEAR[:11]:
        a = {**LINEAR, **kw}
        assert lib.sarathi_mx_linear_plan(a["dtype"], a["kind"], a["a_format"], a["M"], a["N"], a["K"], 0, ct.byref(one),
                                          ct.byref(one), ct.byref(one)) == (code if "resid" not in kw else S.OK)


# ------------------------------------------------------------------ pins of the oracle

def test_grids():
    assert list(ref.grid("e2m1")[:8]) == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    g = ref.grid("e4m3")
    assert g[1] == 2.0 ** -9 and g[0x38] == 1.0 and g[0x7e] == 448.0 and np.isnan(g[0x7f]) and g[0x80 + 0x38] == -1.0


def test_ties_and_borders():
    y = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0])
    assert list(np.abs(ref.grid("e2m1")[ref.nearest_codes(y, "e2m1")])) == [0, 1, 1, 2, 2, 4, 4, 0, 4]
    for fmt, top in ref.TOP.items():
        x = np.zeros((4, 32))
        x[0, 3], x[1, 3], x[2, 3] = top, np.nextafter(np.float32(top), np.float32(1e9)), top / 2
        c, s = ref.quantize(x, fmt)
        assert list(s[:, 0]) == [127, 128, 126, 0]
        assert ref.values(c, s, fmt, 32)[0, 3] == top and ref.values(c, s, fmt, 32)[2, 3] == top / 2


def test_quantized_values_quantize_to_themselves():
    rng = np.random.default_rng(0)
    for fmt in ref.TOP:
        x = rng.standard_normal((20, 100)) * np.exp2(rng.integers(-30, 30, (20, 1)))
        v = ref.values(*ref.quantize(x, fmt), fmt, 100)
        assert np.array_equal(ref.values(*ref.quantize(v, fmt), fmt, 100), v)
        assert np.abs(v - x).max() <= np.abs(x).max() * (1 / 4 if fmt == "e2m1" else 1 / 16)
