"""Microscaled operands (4 and 8 bits) of the linear ops, as cases to time.

32 consecutive elements of a row share a scale 2^e, the smallest power of two
(at least 2^-127) for which none of them passes the largest code: 6 of e2m1 (4
bits: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), 448 of e4m3 (8 bits).
Codes are rounded to nearest, ties to even; the last block of a row may be
short; a block that holds an infinity or NaN stands for NaN.  ``op``:

  quantize  rows [rows, cols] of ``dtype`` to ``format``; the values that the
            codes and scales stand for.
  norm      h = x + delta (``stream`` is the type of x and h, ``dtype`` that of
            delta and the gains), then h / sqrt(mean h^2 + eps) * gain to
            ``format``; h and the values.
  linear    x W^T of x [rows, cols] held in ``format`` and W [n, cols] held in
            e2m1, with the epilogue ``kind``: plain; resid (r + x W^T, r of
            dtype, fp32 out); resid_f32in (r fp32, dtype out); swiglu
            (silu(x Wg^T) x Wu^T); gelu.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 32
EPS = 1e-6
TOP = {"e2m1": 6.0, "e4m3": 448.0}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
KINDS = ("plain", "resid", "resid_f32in", "swiglu", "gelu")
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, op, dtype, fmt, rows, cols, n=0, kind="plain", stream=None):
    c = {"op": op, "dtype": dtype, "format": fmt, "rows": rows, "cols": cols}
    if op == "norm":
        c["stream"] = stream or dtype
    if op == "linear":
        c.update(n=n, kind=kind)
    return {"name": name, **c} if name else c


def listed():
    return [
        # The smallest: the attention output of four decodes; all latency.
        _case("quantize_b4_e4m3", "quantize", "bf16", "e4m3", 4, 5120),
        # The activations of a long prompt before the down projection, odd rows.
        _case("quantize_1021_e2m1", "quantize", "bf16", "e2m1", 1021, 13824),
        # A layer's largest weight, once when a model is loaded.
        _case("quantize_w_up", "quantize", "bf16", "e2m1", 27648, 5120),
        # The norm of a decode-only iteration of four requests.
        _case("norm_b4_e4m3", "norm", "bf16", "e4m3", 4, 5120),
        # The decode-maximal benchmark batch (256 rows of a chunk, 64 decodes) with its residual stream in fp32.
        _case("norm_c256_b64_e2m1", "norm", "bf16", "e2m1", 320, 5120, stream="f32"),
        # A long prompt with the widest rows of the benchmark's layers.
        _case("norm_2048_wide_e4m3", "norm", "bf16", "e4m3", 2048, 12288),
        # The tiny fp32 layer's QKV product.
        _case("linear_tiny_f32", "linear", "f32", "e2m1", 72, 256, 768),
        # QKV of four decodes: the weights stream once.
        _case("linear_b4_qkv_e4m3", "linear", "bf16", "e4m3", 4, 5120, 15360),
        # The down projection of a full server's decode-only iteration, onto the fp32 residual stream.
        _case("linear_b48_down_e2m1", "linear", "bf16", "e2m1", 48, 13824, 5120, "resid_f32in"),
        # Gate and up projections of the decode-maximal batch.
        _case("linear_c256_b64_up_e4m3", "linear", "bf16", "e4m3", 320, 5120, 13824, "swiglu"),
        # Three prompts of ragged lengths: the output projection of the next larger layer.
        _case("linear_1955_o_e4m3", "linear", "bf16", "e4m3", 1955, 6656, 6656, "resid"),
        # The largest: gate and up projections of a whole long prompt.
        _case("linear_4096_up_e2m1", "linear", "bf16", "e2m1", 4096, 5120, 13824, "swiglu"),
    ]


def draw(rng):
    """One more case of the same ranges, no costlier than the largest listed one of its operator."""
    def span(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(["quantize", "norm", "linear", "linear"])
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        fmt = rng.choice(["e2m1", "e4m3"])
        cols = 8 * span(8, 2048)
        if op == "quantize":
            case = _case(None, op, dtype, fmt, span(1, 28000), cols)
        elif op == "norm":
            case = _case(None, op, dtype, fmt, span(1, 4096), 8 * span(8, 1536),
                         stream="f32" if dtype == "f32" or rng.random() < 0.3 else "bf16")
        else:
            case = _case(None, op, dtype, fmt, span(1, 4096), cols, span(16, 28000), rng.choice(KINDS))
        w, most = work(case), [work(c) for c in listed() if c["op"] == op]
        if w["bytes"] <= max(m["bytes"] for m in most) and w["flops"] <= max(m["flops"] for m in most):
            return case


def _held(fmt, rows, cols):
    """Bytes of rows held in a format: codes and one byte per block."""
    return rows * (cols * (0.5 if fmt == "e2m1" else 1.0) + -(-cols // BLOCK))


def work(case):
    """Bytes and operations of one pass: what is read and written once (the values shown count as written)."""
    es = 2 if case["dtype"] == "bf16" else 4
    rows, cols = case["rows"], case["cols"]
    held = _held(case["format"], rows, cols)
    if case["op"] == "quantize":
        return {"bytes": rows * cols * 2 * es + held, "flops": rows * cols * 3}
    if case["op"] == "norm":
        ss = 2 if case["stream"] == "bf16" else 4
        return {"bytes": rows * cols * (2 * ss + 2 * es) + cols * es + held, "flops": rows * cols * 8}
    n, kind = case["n"], case["kind"]
    wide = 2 * n if kind == "swiglu" else n
    extra = {"resid": es + 4, "resid_f32in": 4 + es}.get(kind, es)
    return {"bytes": held + _held("e2m1", wide, cols) + rows * n * extra, "flops": 2 * rows * wide * cols}


# ------------------------------------------------------------------ the operands

def _quantized(x, fmt):
    """Rows x [r, c] in 32 bits to (codes as values [r, blocks, 32], scales [r, blocks]); the last block filled with zeros."""
    r, c = x.shape
    nb = -(-c // BLOCK)
    if c % BLOCK:
        x = torch.cat([x, x.new_zeros((r, nb * BLOCK - c))], 1)
    x = x.view(r, nb, BLOCK)
    top = x.abs().amax(-1)
    whole = torch.isfinite(top)
    m, e = torch.frexp(torch.where(whole, top, torch.zeros_like(top)))          # top = m 2^e, m in [0.5, 1)
    m_top, e_top = math.frexp(TOP[fmt])
    e = torch.where(top > 0, e - e_top + (m > m_top).int(), -127).clamp(min=-127)
    y = torch.ldexp(torch.ldexp(x, (-e // 2)[..., None]), (-e - -e // 2)[..., None])   # two steps: 2^127 has no inverse
    if fmt == "e4m3":
        code = y.to(torch.float8_e4m3fn).float()
    else:
        a = y.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        code = torch.copysign(torch.round(a / step) * step, y)
    scale = torch.where(whole, torch.ldexp(torch.ones_like(top), e), torch.full_like(top, math.nan))
    return torch.where(whole[..., None], code, torch.zeros_like(code)), scale


def _values(code, scale, cols):
    r = code.shape[0]
    return (code * scale[..., None]).reshape(r, -1)[:, :cols]


def _packed(code, scale, fmt):
    """Codes and scales as a file holds them: e2m1 two to a byte (the even one low), e4m3 as they are; a byte per scale."""
    if fmt == "e4m3":
        held = code.flatten(1).to(torch.float8_e4m3fn)
    else:
        a = code.abs().flatten(1)
        idx = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
        idx = idx | (torch.signbit(code.flatten(1)).to(torch.uint8) << 3)
        held = idx[:, 0::2] | (idx[:, 1::2] << 4)
    return held, (torch.frexp(scale)[1] + 126).to(torch.uint8)


def _unpacked(held, scale, fmt, cols):
    """The values, in 32 bits."""
    if fmt == "e4m3":
        code = held.float()
    else:
        table = torch.tensor(GRID + tuple(-v for v in GRID), device=held.device)
        code = torch.stack([table[(held & 15).long()], table[(held >> 4).long()]], -1).flatten(1)
    s = torch.ldexp(torch.ones(scale.shape, device=scale.device), scale.int() - 127)
    return (code.view(code.shape[0], -1, BLOCK) * s[..., None]).flatten(1)[:, :cols]


def _rows(g, rows, cols):
    """Activations: N(0,1), one channel in a hundred stronger."""
    x = torch.randn((rows, cols), device="cuda", generator=g)
    return x * (1.0 + 9.0 * (torch.rand((cols,), device="cuda", generator=g) < 0.01))


def _inputs(case, seed):
    """Tensors of a case; a linear op's operands as packed codes and scales."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols, dt = case["rows"], case["cols"], DT[case["dtype"]]
    st = {"case": case}
    if case["op"] == "quantize":
        st["x"] = _rows(g, rows, cols).to(dt)
    elif case["op"] == "norm":
        st["x"] = (4 * _rows(g, rows, cols)).to(DT[case["stream"]])
        st["delta"] = torch.randn((rows, cols), device="cuda", generator=g).to(dt)
        st["gain"] = (1 + 0.1 * torch.randn((cols,), device="cuda", generator=g)).to(dt)
    else:
        wide = 2 * case["n"] if case["kind"] == "swiglu" else case["n"]
        st["a"], st["a_scale"] = _packed(*_quantized(_rows(g, rows, cols), case["format"]), case["format"])
        w = torch.randn((wide, cols), device="cuda", generator=g) * 0.02
        st["w"], st["w_scale"] = _packed(*_quantized(w, "e2m1"), "e2m1")
        if case["kind"].startswith("resid"):
            r = torch.randn((rows, case["n"]), device="cuda", generator=g)
            st["resid"] = r if case["kind"] == "resid_f32in" else r.to(dt)
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:
        _held_by_library(st)
    return st


# ------------------------------------------------------------------ the framework's calls

def _held_by_library(st):
    """The operands in the library's layout (weights are laid out once, rows by the op before), outputs and scratch memory."""
    from paper_2308_16369_amd import sarathi as S

    case, stream = st["case"], torch.cuda.current_stream().cuda_stream
    rows, cols, dt = case["rows"], case["cols"], DT[case["dtype"]]
    fmt = S.MX_E2M1 if case["format"] == "e2m1" else S.MX_E4M3
    st["fmt"], st["dt"] = fmt, S.BF16 if case["dtype"] == "bf16" else S.F32
    empty = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")  # noqa: E731
    if case["op"] != "linear":
        st["operand"] = empty(S.sarathi_mx_bytes(fmt, rows, cols))
        st["values"] = torch.empty((rows, cols), dtype=dt, device="cuda")
        if case["op"] == "norm":
            st["h"] = torch.empty_like(st["x"])
        return
    n, kind = case["n"], case["kind"]
    x = _unpacked(st.pop("a"), st.pop("a_scale"), case["format"], cols).contiguous()
    st["a"] = empty(S.sarathi_mx_bytes(fmt, rows, cols))
    S.sarathi_mx_quantize(S.F32, fmt, rows, cols, x.data_ptr(), cols, st["a"].data_ptr(), st["a"].numel(), stream)
    w = _unpacked(st.pop("w"), st.pop("w_scale"), "e2m1", cols).contiguous()
    one = S.sarathi_mx_bytes(S.MX_E2M1, n, cols)
    parts = w.shape[0] // n
    st["w"] = empty(parts * one)                                                # gate, then up
    for i in range(parts):
        S.sarathi_mx_quantize(S.F32, S.MX_E2M1, n, cols, w[i * n:].data_ptr(), cols, st["w"].data_ptr() + i * one, one, stream)
    st["out"] = torch.empty((rows, n), dtype=torch.float32 if kind == "resid" else dt, device="cuda")
    st["scratch"] = empty(S.sarathi_mx_linear_scratch_bytes(rows, n))
    st["kind"] = {"plain": S.LINEAR_PLAIN, "resid": S.LINEAR_RESID, "resid_f32in": S.LINEAR_RESID_F32IN,
                  "swiglu": S.LINEAR_SWIGLU, "gelu": S.LINEAR_GELU}[kind]


def _own(st):
    from paper_2308_16369_amd import sarathi as S

    case, stream = st["case"], torch.cuda.current_stream().cuda_stream
    rows, cols, fmt, dt = case["rows"], case["cols"], st["fmt"], st["dt"]
    if case["op"] == "linear":
        resid = st["resid"].data_ptr() if "resid" in st else 0
        S.sarathi_mx_linear(dt, st["kind"], fmt, rows, case["n"], cols, st["a"].data_ptr(), st["w"].data_ptr(), resid,
                            st["out"].data_ptr(), st["scratch"].data_ptr(), st["scratch"].numel(), stream)
        return {"y": st["out"]}
    operand, size = st["operand"].data_ptr(), st["operand"].numel()
    out = {}
    if case["op"] == "quantize":
        S.sarathi_mx_quantize(dt, fmt, rows, cols, st["x"].data_ptr(), cols, operand, size, stream)
    else:
        sdt = S.BF16 if case["stream"] == "bf16" else S.F32
        S.sarathi_mx_norm(sdt, dt, fmt, rows, cols, EPS, st["x"].data_ptr(), cols, st["delta"].data_ptr(), cols,
                          st["gain"].data_ptr(), st["h"].data_ptr(), cols, operand, size, stream)
        out["h"] = st["h"]
    S.sarathi_mx_dequantize(fmt, rows, cols, operand, size, dt, st["values"].data_ptr(), cols, stream)
    return {**out, "values": st["values"]}


# ------------------------------------------------------------------ the plain form

def _plain(st):
    case = st["case"]
    cols, dt = case["cols"], DT[case["dtype"]]
    if case["op"] == "quantize":
        return {"values": _values(*_quantized(st["x"].float(), case["format"]), cols).to(dt)}
    if case["op"] == "norm":
        h = st["x"].float() + st["delta"].float()
        y = h / torch.sqrt((h * h).mean(-1, keepdim=True) + EPS) * st["gain"].float()
        return {"h": h.to(st["x"].dtype), "values": _values(*_quantized(y, case["format"]), cols).to(dt)}
    kind = case["kind"]
    x = _unpacked(st["a"], st["a_scale"], case["format"], cols)
    z = torch.matmul(x, _unpacked(st["w"], st["w_scale"], "e2m1", cols).t())
    if kind == "swiglu":
        gate, up = z[:, :case["n"]], z[:, case["n"]:]
        z = gate / (1 + torch.exp(-gate)) * up
    elif kind == "gelu":
        z = 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    elif kind != "plain":
        z = z + st["resid"].float()
    return {"y": z if kind == "resid" else z.to(dt)}


def run(st):
    return _own(st) if own else _plain(st)


# ------------------------------------------------------------------ the definition in 64 bits

def _nearest(y, fmt):
    """y, in 64 bits, to the format's values: steps of the power of two that its magnitude has, not below the smallest normal's."""
    bits, low = (1, 0) if fmt == "e2m1" else (3, -6)
    power = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** low)))
    step = torch.exp2(power - bits)
    return torch.round(y / step) * step


def _exact_values(y, fmt):
    """Rows in 64 bits, as the values that their codes and scales stand for."""
    out = torch.empty_like(y)
    for c0 in range(0, y.shape[1], BLOCK * 64):
        part = y[:, c0:c0 + BLOCK * 64]
        cols = part.shape[1]
        part = torch.nn.functional.pad(part, (0, -cols % BLOCK)).view(y.shape[0], -1, BLOCK)
        need = part.abs().amax(-1, keepdim=True) / TOP[fmt]
        scale = torch.exp2(torch.ceil(torch.log2(need)).clamp(min=-127))
        scale = torch.where(scale < need, scale * 2, torch.where(scale / 2 >= need, scale / 2, scale)).clamp(min=2.0 ** -127)
        out[:, c0:c0 + cols] = (_nearest(part / scale, fmt) * scale).flatten(1)[:, :cols]
    return out


def _exact_operand(held, scale, fmt, cols):
    s = torch.exp2(scale.double() - 127).repeat_interleave(BLOCK, 1)[:, :cols]
    if fmt == "e4m3":
        return held.double()[:, :cols] * s
    nib = torch.empty((held.shape[0], 2 * held.shape[1]), dtype=torch.int16, device=held.device)
    nib[:, 0::2], nib[:, 1::2] = held % 16, held // 16
    nib = nib[:, :cols]
    mant, power = (nib % 2).double(), (nib // 2 % 4).double()
    mag = torch.where(power == 0, mant * 0.5, (1 + mant / 2) * torch.exp2(power - 1))
    return torch.where(nib >= 8, -mag, mag) * s


def exact(case, seed):
    st, fmt, cols = _inputs(case, seed), case["format"], case["cols"]
    if case["op"] == "quantize":
        return {"values": _exact_values(st["x"].double(), fmt)}
    if case["op"] == "norm":
        h = st["x"].double() + st["delta"].double()
        y = h * st["gain"].double() * (h.square().sum(-1, keepdim=True) / cols + EPS).rsqrt()
        return {"h": h, "values": _exact_values(y, fmt)}
    x = _exact_operand(st["a"], st["a_scale"], fmt, cols)
    n, kind = case["n"], case["kind"]
    w = _exact_operand(st["w"], st["w_scale"], "e2m1", cols)
    z = x @ w[:n].T
    if kind == "swiglu":
        z = z * torch.sigmoid(z) * (x @ w[n:].T)
    elif kind == "gelu":
        z = z * torch.special.ndtr(z)
    elif kind != "plain":
        z = st["resid"].double() + z
    return {"y": z}
