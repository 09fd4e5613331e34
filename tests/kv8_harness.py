"""Helpers of the 8-bit KV cache's tests: a cache in guarded device memory, the
operators through their C-ABI, and the checks against the float64 oracle."""
from __future__ import annotations

import math
from dataclasses import dataclass, field
from typing import List, Sequence, Tuple

import numpy as np
import torch

from oracle import kv8 as ref
from paper_2308_16369_amd import sarathi as S

LAYOUTS = {"half": S.ROPE_HALF, "interleaved": S.ROPE_INTERLEAVED}
SCALINGS = {"plain": S.ROPE_PLAIN, "linear": S.ROPE_LINEAR, "ntk": S.ROPE_NTK, "bands": S.ROPE_BANDS}
FORMATS = {"int8": S.KV8_INT8, "e4m3": S.KV8_E4M3}
GUARD = 4096


@dataclass
class Spec:
    heads: int = 4
    kv_heads: int = 2
    dim: int = 64
    dtype: str = "bf16"
    fmt: str = "int8"
    block: int = 16
    layers: int = 1
    slots: int = 4
    seq: int = 300
    norm: bool = False
    eps: float = 1e-6
    rot: int = 0
    layout: str = "half"
    scaling: str = "plain"
    base: float = 10000.0
    factor: float = 1.0
    mscale: float = 0.0
    softmax_scale: float = 0.0

    @property
    def group(self):
        return self.heads // self.kv_heads

    @property
    def tdt(self):
        return torch.bfloat16 if self.dtype == "bf16" else torch.float32

    def cfg(self):
        return S.make_kv8_cfg(self.heads, self.kv_heads, self.dim, n_layers=self.layers,
                              dtype=S.BF16 if self.dtype == "bf16" else S.F32, format=FORMATS[self.fmt], block=self.block,
                              softmax_scale=self.softmax_scale, qk_norm=int(self.norm), qk_eps=self.eps, rope_dim=self.rot,
                              rope_layout=LAYOUTS[self.layout], rope_scaling=SCALINGS[self.scaling], rope_base=self.base,
                              rope_factor=self.factor, rope_low=1.0, rope_high=8.0, rope_orig_len=256,
                              rope_mscale=self.mscale)

    def thetas(self):
        return ref.thetas(self.rot, self.base, self.scaling, self.factor, 1.0, 8.0, 256)


@dataclass
class Batch:
    chunks: Sequence[Tuple[int, int, int]] = field(default_factory=list)   # (slot, offset, length)
    decodes: Sequence[Tuple[int, int]] = field(default_factory=list)       # (slot, context)

    def seqs(self) -> List[Tuple[int, int, int]]:
        return [tuple(c) for c in self.chunks] + [(s, c, 1) for s, c in self.decodes]

    def rows(self):
        """(slot, position) of every row."""
        return [(s, p) for s, o, n in self.seqs() for p in range(o, o + n)]

    @property
    def T(self):
        return sum(n for _, _, n in self.seqs())


class Cache:
    """An 8-bit cache whose memory starts as 0xff (NaN scales, NaN codes of e4m3) between guards."""

    def __init__(self, spec: Spec):
        self.spec, self.c = spec, spec.cfg()
        self.bytes = S.sarathi_kv8_bytes(self.c, spec.slots, spec.seq)
        assert self.bytes > 0, S.sarathi_last_error()
        self.mem = torch.full((self.bytes + 2 * GUARD,), 255, dtype=torch.uint8, device="cuda")
        self.kv = S.sarathi_kv8_alloc(self.c, spec.slots, spec.seq, self.mem.data_ptr() + GUARD, self.bytes)
        self.lay = self.kv.layout()
        self.keep = []

    def views(self):
        """Device views: codes [layer, slot, 2, head, pos, dim] (bytes) and scales [layer, slot, 2, head, block]."""
        p = self.spec
        n = p.layers * p.slots * 2 * p.kv_heads * p.seq * p.dim
        nb = -(-p.seq // p.block)
        codes = self.mem[GUARD:GUARD + n].view(p.layers, p.slots, 2, p.kv_heads, p.seq, p.dim)
        at = GUARD + self.lay.scale_offset
        scales = self.mem[at:at + 4 * p.layers * p.slots * 2 * p.kv_heads * nb].view(torch.float32)
        return codes, scales.view(p.layers, p.slots, 2, p.kv_heads, nb)

    def host(self):
        codes, scales = self.views()
        return codes.cpu().numpy(), scales.cpu().numpy()

    def values(self):
        """Float64 values of the whole cache (NaN where nothing was written)."""
        codes, scales = self.host()
        v = ref.code_values(self.spec.fmt)[codes]
        return v * np.repeat(scales.astype(np.float64), self.spec.block, -1)[..., :self.spec.seq, None]

    def fill(self, g):
        """Random codes and scales everywhere, as many appends would leave them."""
        codes, scales = self.views()
        if self.spec.fmt == "int8":
            codes.copy_(torch.randint(-127, 128, codes.shape, device="cuda", generator=g).to(torch.int8).view(torch.uint8))
            scales.uniform_(0.004, 0.03, generator=g)
        else:
            x = torch.randn(codes.shape, device="cuda", generator=g) * 100
            codes.copy_(x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
            scales.copy_(torch.exp2(torch.randint(-8, -5, scales.shape, device="cuda", generator=g).float()))

    def plan(self, batch: Batch, stream=None):
        rows, n = batch.T, len(batch.chunks)
        size = S.sarathi_kv8_plan_bytes(self.c, rows, n, self.spec.seq)
        ws = torch.full((size + GUARD,), 255, dtype=torch.uint8, device="cuda")
        b, keep = S.make_mixed_batch(list(batch.chunks), [d[0] for d in batch.decodes], [d[1] for d in batch.decodes])
        if stream is None:
            stream = torch.cuda.current_stream().cuda_stream
        else:
            torch.cuda.synchronize()           # the fill runs on the current stream, the upload on another
        p = S.sarathi_kv8_plan_create(self.kv, b, ws.data_ptr(), size, stream)
        p.ws = ws
        return p

    def guards_intact(self):
        return bool((self.mem[:GUARD] == 255).all()) and bool((self.mem[GUARD + self.bytes:] == 255).all())


def cur():
    return torch.cuda.current_stream().cuda_stream


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def make_rows(spec: Spec, T: int, g, ld_extra: int = 0):
    """qkv rows [T, ld] of N(0, 1) (a few strong key channels) and gains."""
    cols = (spec.heads + 2 * spec.kv_heads) * spec.dim
    x = torch.randn((T, cols + ld_extra), device="cuda", generator=g)
    x[:, spec.heads * spec.dim:(spec.heads + spec.kv_heads) * spec.dim:17] *= 4
    gains = 1 + 0.2 * torch.randn((2, spec.dim), device="cuda", generator=g)
    return x.to(spec.tdt), gains.to(spec.tdt)


def expected_rows(spec: Spec, qkv, gains, pos):
    """Float64 q, k, v heads [T, heads, dim] as the definition gives them."""
    T, hd, nh, nkv = qkv.shape[0], spec.dim, spec.heads, spec.kv_heads
    x = f64(qkv)[:, :(nh + 2 * nkv) * hd].reshape(T, nh + 2 * nkv, hd)
    q, k, v = x[:, :nh], x[:, nh:nh + nkv], x[:, nh + nkv:]
    if spec.norm:
        gq, gk = f64(gains)
        q, k = ref.head_norm(q, gq, spec.eps), ref.head_norm(k, gk, spec.eps)
    if spec.rot:
        th, m = spec.thetas(), spec.mscale or 1.0
        q, k = ref.rotate(q, pos, th, spec.layout, m), ref.rotate(k, pos, th, spec.layout, m)
    return q, k, v


def check_append(spec: Spec, batch: Batch, before, after, q_out, q, k, v, layer=0):
    """The cache after an append (host codes, scales before and after), and q.

    Tolerances.  The fp32 arithmetic of norm and rotation: a dozen roundings of
    2^-24 and a sine and cosine to 2^-22, on pairs of magnitude up to m =
    mscale * sqrt(2) * max|x| of the head: slack 2^-19 m.  Scales: that slack on
    the block's largest element.  A code: half a step of its format beyond it."""
    (c0, s0), (c1, s1) = before, after
    vals = ref.code_values(spec.fmt)
    half = 2.0 ** -8 if spec.dtype == "bf16" else 2.0 ** -24
    m = 2.0 ** -19 * np.abs(q).max(-1, keepdims=True) * 2
    assert np.all(np.abs(f64(q_out).reshape(q.shape) - q) <= half * np.abs(q) + m)
    touched_c, touched_s = np.zeros(c0.shape, bool), np.zeros(s0.shape, bool)
    row = 0
    for slot, off, n in batch.seqs():
        for b in range(off // spec.block, (off + n - 1) // spec.block + 1):
            lo, hi = max(off, b * spec.block), min(off + n, (b + 1) * spec.block)
            old = slice(b * spec.block, lo)
            touched_s[layer, slot, :, :, b] = True
            touched_c[layer, slot, :, :, b * spec.block:hi] = True
            for which, x in ((0, k), (1, v)):
                new = x[row + lo - off:row + hi - off].transpose(1, 0, 2)           # [head, pos, dim]
                slack = 2.0 ** -18 * np.abs(new).max((1, 2)) if which == 0 else 2.0 ** -23 * np.abs(new).max((1, 2))
                was = s0[layer, slot, which, :, b].astype(np.float64) if lo > b * spec.block else np.zeros(spec.kv_heads)
                now = s1[layer, slot, which, :, b].astype(np.float64)
                top = np.abs(new).max((1, 2))
                lo_s = np.maximum(was, ref.scale_needed(np.maximum(top - slack, 0), spec.fmt))
                hi_s = np.maximum(was, ref.scale_needed(top + slack, spec.fmt))
                assert np.all(now >= lo_s * (1 - 2.0 ** -23)) and np.all(now <= hi_s * (1 + 2.0 ** -23)), (now, lo_s, hi_s)
                got = vals[c1[layer, slot, which, :, lo:hi]]
                assert np.all(np.abs(got) <= ref.QMAX[spec.fmt])
                unit = now[:, None, None]
                want = np.divide(new, unit, out=np.zeros_like(new), where=unit > 0)
                tol = ref.half_step(want, spec.fmt) + (slack / np.where(now > 0, now, 1))[:, None, None] + 2.0 ** -22 * np.abs(want)
                assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) - tol)
                # earlier positions of the block: as they were, or rounded once to the new scale
                g0, g1 = vals[c0[layer, slot, which, :, old]], vals[c1[layer, slot, which, :, old]]
                for h in range(spec.kv_heads):
                    if now[h] == was[h]:
                        assert np.array_equal(c0[layer, slot, which, h, old], c1[layer, slot, which, h, old])
                    elif lo > b * spec.block:
                        moved = g0[h] * (was[h] / now[h])
                        t = ref.half_step(moved, spec.fmt) + 2.0 ** -22 * np.abs(moved)
                        assert np.all(np.abs(g1[h] - moved) <= t)
        row += n
    assert np.array_equal(c0[~touched_c], c1[~touched_c])
    same = (s0.view(np.uint32) == s1.view(np.uint32))
    assert np.all(same[~touched_s])


def offset_error(spec: Spec, batch: Batch, row, scales, w):
    """What the offset of the codes adds to the tolerance of a decode of bf16 rows over int8 codes, from weights w.

    The kernel sums p_j u_j (u = code + 128 <= 255) in fp32 and takes 128 sum(p)
    out again.  Of n keys a wave sums n / 4 in steps of 32: 32 products and the
    sum so far, each added with an error of at most 2^-23 (truncation) of a sum
    that 255 sum(p) bounds; the sum of the p's takes 8 more of a bound half as
    large, the merge 4: below 40 ceil(n / 128) 2^-23 255 in codes, times the
    weights and their scales."""
    if spec.dtype != "bf16" or spec.fmt != "int8" or row < batch.T - len(batch.decodes):
        return 0.0
    n = len(w)
    return 40 * -(-n // 128) * 2.0 ** -23 * 255 * float(w @ np.repeat(scales, spec.block)[:n])


def check_attention(spec: Spec, batch: Batch, values, q, out, layer=0, scales=None):
    """Outputs against float64 over the cache's own values.

    Tolerances, of the weighted sum A = sum_j w_j |v_j|.  Scores: 2 D + 8
    fp32 roundings of sum |q k| (three times the products in fp32 rows), an
    exponent and its argument (|s| 2^-23): a relative error of every weight,
    twice (numerator and row sum).  bf16 rows: the probabilities' rounding,
    2^-8, twice, and the output's own.  With scales (of the cache): the codes'
    offset as well, for inputs whose heavy keys have small values."""
    scale = spec.softmax_scale or 1 / math.sqrt(spec.dim)
    qv, ov = f64(q).reshape(-1, spec.heads, spec.dim), f64(out).reshape(-1, spec.heads, spec.dim)
    worst = 0.0
    for r, (slot, pos) in enumerate(batch.rows()):
        for h in range(spec.heads):
            kv = values[layer, slot, :, h // spec.group, :pos + 1]
            o, a, mag = ref.attend(qv[r, h], kv[0], kv[1], scale)
            terms = 3 if spec.dtype == "f32" else 1
            rel = (2 * spec.dim * terms + 16) * 2.0 ** -24 * max(mag, 1.0) + 2.0 ** -20
            tol = 2 * rel * a + (2 * 2.0 ** -8 * a + 2.0 ** -8 * np.abs(o) if spec.dtype == "bf16" else 2.0 ** -23 * np.abs(o))
            if scales is not None:
                sc = scales[layer, slot, :, h // spec.group].astype(np.float64)
                s = scale * (kv[0] @ qv[r, h])
                w = np.exp(s - s.max())
                tol = tol + offset_error(spec, batch, r, sc[1], w / w.sum())
            d = np.abs(ov[r, h] - o)
            assert np.all(d <= tol + 1e-30), (r, h, slot, pos, float(np.max(d / (tol + 1e-30))))
            worst = max(worst, float(np.max(d / (tol + 1e-30))))
    return worst
