"""Microscaled products on the paths that only some sizes take: split columns in place, replayed and on two streams at
once, random numbers in every block shape, every kernel of few rows, and scratch memory that is not used."""
import numpy as np
import pytest

import test_gpu_mx as base
from paper_2308_16369_amd import sarathi as S
from test_gpu_mx import DT, FMT, KIND, PICKS, resid_of, run_linear, stream

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def held(v, fmt):
    """Rows (device, fp32) as an operand, and the values that it holds."""
    rows, cols = v.shape
    n = S.sarathi_mx_bytes(FMT[fmt], rows, cols)
    op = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    S.sarathi_mx_quantize(S.F32, FMT[fmt], rows, cols, v.data_ptr(), cols, op.data_ptr(), n, stream())
    back = torch.empty_like(v)
    S.sarathi_mx_dequantize(FMT[fmt], rows, cols, op.data_ptr(), n, S.F32, back.data_ptr(), cols, stream())
    return op, back.double()


def normal(seed, rows, cols, size=1.0):
    """N(0,1) rows, a channel in fifty twenty times stronger, columns of several magnitudes."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((rows, cols), device="cuda", generator=g)
    strong = torch.rand((cols,), device="cuda", generator=g) < 0.02
    return x * torch.where(strong, 20.0, 1.0) * torch.exp2(torch.randint(-2, 3, (cols,), device="cuda", generator=g).float()) * size


def bound(a, w, fmt, exact):
    """What the sums can be off by, of values in 64 bits on the device.  A matrix instruction takes 64 columns: eight sums of
    eight and the accumulator, cut below 24 bits of the largest: nine terms off by 2^-23 of it each; partial sums are joined
    with one rounding each, at most 32.  e4m3 rows in one product: eight terms cut 13 bits below the largest of the eight (at
    most the largest of |a| times the largest of |w| there)."""
    K = a.shape[1]
    s = a.abs() @ w.abs().T
    tol = (9 * -(-K // 64) * (2 if fmt == "e4m3" and exact else 1) + 32) * 2.0 ** -23 * s
    if fmt == "e4m3" and not exact:
        top = lambda v: torch.nn.functional.pad(v.abs(), (0, -K % 8)).view(v.shape[0], -1, 8).amax(-1)  # noqa: E731
        tol = tol + 8 * 2.0 ** -13 * (top(a) @ top(w).T)
    return tol


def expected(kind, dtype, fmt, a, ws, r, rows):
    """The product of the values in 64 bits, and what the output may be off by."""
    f32_out = dtype == "f32" or kind == "resid"
    half = 2.0 ** -24 if f32_out else 2.0 ** -8
    z = [a @ w.T for w in ws]
    t = [bound(a, w, fmt, f32_out or rows <= 64) for w in ws]
    if kind == "swiglu":
        s = z[0] * torch.sigmoid(z[0])
        ts = 1.1 * t[0] + s.abs() * (z[0].abs() + 8) * 2.0 ** -23
        want, tol = s * z[1], ts * (z[1].abs() + t[1]) + s.abs() * t[1]
    elif kind == "gelu":
        want, tol = z[0] * torch.special.ndtr(z[0]), 1.13 * t[0] + z[0].abs() * 4 * 2.0 ** -23
    else:
        want = z[0] + (r.double() if r is not None else 0.0)
        tol = t[0] + 2.0 ** -24 * (want.abs() + t[0])
    return want, tol + half * (want.abs() + tol) + 2.0 ** -133


def plan(dtype, kind, fmt, M, N, K):
    return S.sarathi_mx_linear_plan(DT[dtype][0], KIND[kind], FMT[fmt], M, N, K, S.sarathi_mx_linear_scratch_bytes(M, N))


@pytest.mark.parametrize("fmt,dtype,kind,M,N,K,bm,bn,split", PICKS, ids=["-".join(map(str, c[:6])) for c in PICKS])
def test_every_block_shape_of_random_numbers(fmt, dtype, kind, M, N, K, bm, bn, split):
    assert plan(dtype, kind, fmt, M, N, K)[:2] == (bm, bn) and (plan(dtype, kind, fmt, M, N, K)[2] > 1) == bool(split)
    a, av = held(normal(M + N, M, K), fmt)
    parts = [held(normal(M + N + 1 + i, N, K, 0.05), "e2m1") for i in range(2 if kind == "swiglu" else 1)]
    r = resid_of(np.random.default_rng(M), kind, dtype, M, N)
    out = run_linear(a, torch.cat([p[0] for p in parts]), r, kind, dtype, fmt, M, N, K)
    want, tol = expected(kind, dtype, fmt, av, [p[1] for p in parts], r, M)
    off = (out.double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


# rows, W rows: 8 or 16 waves with W of more than 256 tiles or fewer; SwiGLU's tiles count twice
STREAMS = [(5, 8300, "plain", 32), (5, 700, "plain", 32), (32, 8300, "gelu", 32), (40, 8300, "plain", 32), (64, 700, "resid", 32),
           (64, 8300, "resid_f32in", 32), (7, 4200, "swiglu", 64), (50, 4200, "swiglu", 64), (96, 8000, "plain", 32),
           (100, 8000, "resid_f32in", 32), (128, 640, "plain", 32), (70, 4000, "swiglu", 64), (100, 4000, "swiglu", 64),
           (128, 96, "swiglu", 64)]


@pytest.mark.parametrize("fmt", list(FMT))
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("M,N,kind,bn", STREAMS)
def test_every_kernel_of_few_rows(fmt, dtype, M, N, kind, bn):
    K = 2568                                                 # eleven quads of columns: an odd share for 4, 8 and 16 waves
    assert plan(dtype, kind, fmt, M, N, K) == (-(-M // 32) * 32, bn, 1)
    base.test_every_block_shape(fmt, dtype, kind, M, N, 520, -(-M // 32) * 32, bn, 0)    # sums that are exact
    a, av = held(normal(M + N, M, K), fmt)
    parts = [held(normal(M + N + 1 + i, N, K, 0.05), "e2m1") for i in range(2 if kind == "swiglu" else 1)]
    r = resid_of(np.random.default_rng(M), kind, dtype, M, N)
    out = run_linear(a, torch.cat([p[0] for p in parts]), r, kind, dtype, fmt, M, N, K)
    want, tol = expected(kind, dtype, fmt, av, [p[1] for p in parts], r, M)
    off = (out.double() - want).abs()
    assert bool((off <= tol).all()), float((off / tol).max())


# ------------------------------------------------------------------ split columns

SPLIT = [("e2m1", "resid", "f32", 200, 512, 8712), ("e4m3", "resid", "f32", 200, 512, 8712),
         ("e4m3", "resid_f32in", "f32", 130, 1003, 4104), ("e2m1", "resid_f32in", "f32", 70, 3500, 14600)]


class Onto:
    """A product onto its residual in place, columns split, with scratch of its own."""

    def __init__(self, fmt, kind, dtype, M, N, K, seed):
        self.args = (DT[dtype][0], KIND[kind], FMT[fmt], M, N, K)
        self.bytes = S.sarathi_mx_linear_scratch_bytes(M, N)
        assert S.sarathi_mx_linear_plan(*self.args, self.bytes)[2] > 1
        self.a, av = held(normal(seed, M, K), fmt)
        self.w, wv = held(normal(seed + 1, N, K, 0.05), "e2m1")
        self.r = resid_of(np.random.default_rng(seed), kind, dtype, M, N)
        self.want, self.tol = expected(kind, dtype, fmt, av, [wv], self.r, M)
        self.out = torch.empty_like(self.r)
        self.scratch = torch.full((self.bytes,), 0xff, dtype=torch.uint8, device="cuda")   # NaN

    def run(self):
        self.out.copy_(self.r)
        S.sarathi_mx_linear(*self.args, self.a.data_ptr(), self.w.data_ptr(), self.out.data_ptr(), self.out.data_ptr(),
                            self.scratch.data_ptr(), self.bytes, stream())

    def check(self):
        off = (self.out.double() - self.want).abs()
        assert bool((off <= self.tol).all()), float((off / self.tol).max())


@pytest.mark.parametrize("fmt,kind,dtype,M,N,K", SPLIT)
def test_split_columns_onto_their_residual_in_place(fmt, kind, dtype, M, N, K):
    o = Onto(fmt, kind, dtype, M, N, K, M)
    first = None
    for _ in range(3):
        o.run()
        torch.cuda.synchronize()
        o.check()
        first = o.out.clone() if first is None else first
        assert torch.equal(o.out, first)                     # the same each time
    apart = run_linear(o.a, o.w, o.r, kind, dtype, fmt, M, N, K)
    assert torch.equal(apart, first)


@pytest.mark.parametrize("fmt,kind,dtype,M,N,K", SPLIT)
def test_split_columns_captured_and_replayed(fmt, kind, dtype, M, N, K):
    o = Onto(fmt, kind, dtype, M, N, K, M)
    o.run()
    torch.cuda.synchronize()
    want = o.out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        o.run()
    for i in range(4):
        o.out.fill_(9.0)
        o.scratch.fill_(0xff)
        o.r.mul_(2.0 if i else 1.0)                          # an exact change of the residual between replays
        graph.replay()
        torch.cuda.synchronize()
        got = o.out.clone()
        o.run()                                              # eager work of its own between the replays
        torch.cuda.synchronize()
        assert torch.equal(got, o.out), i
        if i == 0:
            assert torch.equal(got, want)
            o.check()


def test_split_columns_on_two_streams_at_once():
    os_ = [Onto("e4m3", "resid", "f32", 200, 512, 8712, 1), Onto("e4m3", "resid", "f32", 200, 512, 8712, 7),
           Onto("e2m1", "resid_f32in", "f32", 70, 3500, 14600, 9)]
    want = []
    for o in os_:
        o.run()
        torch.cuda.synchronize()
        o.check()
        want.append(o.out.clone())
    streams = [torch.cuda.Stream() for _ in os_]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(6):
        for o, s in zip(os_, streams):
            with torch.cuda.stream(s):
                o.run()
    torch.cuda.synchronize()
    for o, w in zip(os_, want):
        assert torch.equal(o.out, w)


def test_scratch_that_is_not_aligned_is_not_used():
    fmt, kind, dtype, M, N, K = SPLIT[1]
    o = Onto(fmt, kind, dtype, M, N, K, 3)
    memory = torch.full((o.bytes + 64,), 0x5a, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(o.r)
    S.sarathi_mx_linear(*o.args, o.a.data_ptr(), o.w.data_ptr(), o.r.data_ptr(), out.data_ptr(), memory.data_ptr() + 8, o.bytes,
                        stream())
    torch.cuda.synchronize()
    assert (memory == 0x5a).all()
    assert torch.equal(out, run_linear(o.a, o.w, o.r, kind, dtype, fmt, M, N, K, scratch=False))
