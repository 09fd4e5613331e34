"""The decoder layer and the model step over the 8-bit KV cache: every stage
against float64 from the stage before it, the step against layer-by-layer calls
bit for bit, captured replays, and the serving loop."""
import dataclasses

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import oracle  # noqa: E402
import workloads as wl  # noqa: E402
from gpu_harness import TOL, delta_err, rel_err  # noqa: E402
from kv8_harness import Batch, Cache, Spec, check_append, check_attention, cur, expected_rows, f64  # noqa: E402
from paper_2308_16369_amd import sarathi as S  # noqa: E402
from paper_2308_16369_amd import serve  # noqa: E402


class Model:
    """Layers with an 8-bit cache.  norm: "rms" (SwiGLU) or "layer" (GELU)."""

    def __init__(self, spec: Spec, hidden=192, ffn=320, norm="rms", seed=0):
        self.spec, self.hidden, self.ffn, self.norm = spec, hidden, ffn, norm
        rope = int(spec.rot > 0)
        self.cfg = S.make_cfg(hidden, spec.heads, spec.dim, ffn, n_layers=spec.layers,
                              norm=S.NORM_RMS if norm == "rms" else S.NORM_LAYER,
                              act=S.ACT_SWIGLU if norm == "rms" else S.ACT_GELU, rope=rope, rope_base=spec.base,
                              dtype=S.BF16 if spec.dtype == "bf16" else S.F32)
        g = torch.Generator(device="cuda").manual_seed(seed)
        qd, nqkv = spec.heads * spec.dim, (spec.heads + 2 * spec.kv_heads) * spec.dim
        dims = {"w_qkv": (nqkv, hidden), "w_o": (hidden, qd), "w_up": (2 * ffn if norm == "rms" else ffn, hidden),
                "w_down": (hidden, ffn), "norm1_g": (hidden,), "norm2_g": (hidden,), "q_gain": (spec.dim,),
                "k_gain": (spec.dim,)}
        if norm == "layer":
            dims.update(norm1_b=(hidden,), norm2_b=(hidden,))

        def draw(name, shape):
            x = torch.randn(shape, device="cuda", generator=g)
            return ((1 + 0.1 * x) if name.endswith(("_g", "gain")) else x * (0.1 if name.endswith("_b") else 0.06)).to(spec.tdt)

        self.w = [{k: draw(k, v) for k, v in dims.items()} for _ in range(spec.layers)]
        self.abi = [S.make_kv8_weights({k: t.data_ptr() for k, t in w.items()}) for w in self.w]

    def workspace(self, T, n_chunks):
        n = S.sarathi_kv8_workspace_bytes(self.cfg, self.spec.cfg(), T, n_chunks, self.spec.seq)
        assert n > 0, S.sarathi_last_error()
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda"), n

    def batch(self, b: Batch):
        return S.make_mixed_batch(list(b.chunks), [d[0] for d in b.decodes], [d[1] for d in b.decodes])

    def layer(self, cache, layer, b, x, ws, n):
        y = torch.empty_like(x)
        mb, keep = self.batch(b)
        S.sarathi_kv8_layer_forward(self.cfg, self.abi[layer], cache.kv, layer, mb, x.data_ptr(), y.data_ptr(), ws.data_ptr(),
                                    n, cur())
        torch.cuda.synchronize()
        return y

    def step(self, cache, b, x, ws, n):
        y = torch.empty_like(x)
        mb, keep = self.batch(b)
        S.sarathi_kv8_model_step(self.cfg, self.abi, cache.kv, mb, x.data_ptr(), y.data_ptr(), ws.data_ptr(), n, cur())
        torch.cuda.synchronize()
        return y


def view(ws, off, rows, cols, dt):
    es = 2 if dt == torch.bfloat16 else 4
    return ws[off:off + rows * cols * es].view(dt).view(rows, cols)


def rows(spec, T, hidden, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((T, hidden), device="cuda", generator=g).to(spec.tdt)


SPECS = [
    dict(heads=6, kv_heads=2, dim=64, block=32, rot=64, norm=True, fmt="int8"),
    dict(heads=4, kv_heads=4, dim=128, block=64, rot=128, fmt="e4m3"),
    dict(heads=4, kv_heads=1, dim=64, block=16, rot=32, layout="interleaved", scaling="bands", factor=4.0, mscale=1.1,
         fmt="int8"),
    dict(heads=3, kv_heads=3, dim=64, block=128, rot=0, fmt="e4m3"),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("i", range(len(SPECS)))
def test_layer_stages(dtype, i):
    """Two iterations of one layer; each stage from the values that the stage before it left on the device."""
    spec = Spec(dtype=dtype, layers=2, slots=4, seq=260, **SPECS[i])
    m, cache = Model(spec, norm="layer" if i == 3 else "rms"), Cache(spec)
    w = {k: f64(t) for k, t in m.w[1].items()}
    tol = TOL[dtype]
    nh, nkv, hd, H = spec.heads, spec.kv_heads, spec.dim, m.hidden
    for it, b in enumerate([Batch(chunks=[(2, 0, 75), (0, 0, 9)]), Batch(chunks=[(2, 75, 40)], decodes=[(0, 9), (3, 0)])]):
        T = b.T
        x = rows(spec, T, H, 5 + it)
        ws, n = m.workspace(T + 3, 2)            # a workspace for larger batches serves smaller ones
        before = cache.host()
        y = m.layer(cache, 1, b, x, ws, n)
        lay = S.sarathi_kv8_workspace_layout(m.cfg, spec.cfg(), T, len(b.chunks), spec.seq)
        qkv = view(ws, lay.qkv, T, (nh + 2 * nkv) * hd, spec.tdt)
        o = view(ws, lay.o, T, nh * hd, spec.tdt)
        hres = view(ws, lay.hres, T, H, torch.float32)
        act = view(ws, lay.m, T, m.ffn, spec.tdt)
        norm = (lambda v, k: oracle.rms_norm(v, w[k + "_g"], 1e-6)) if m.norm == "rms" else \
            (lambda v, k: oracle.layer_norm(v, w[k + "_g"], w[k + "_b"], 1e-6))
        proj = oracle.linear(norm(f64(x), "norm1"), w["w_qkv"])
        assert rel_err(f64(qkv)[:, nh * hd:], proj[:, nh * hd:]) <= tol
        pos = [p for _, p in b.rows()]
        gains = torch.stack([m.w[1]["q_gain"], m.w[1]["k_gain"]])
        q_ref = expected_rows(spec, torch.from_numpy(proj), gains, pos)[0]
        assert rel_err(f64(qkv)[:, :nh * hd].reshape(q_ref.shape), q_ref) <= tol
        _, k, v = expected_rows(spec, qkv, gains, pos)
        q = qkv[:, :nh * hd]
        check_append(spec, b, before, cache.host(), q, f64(q).reshape(T, nh, hd), k, v, layer=1)
        check_attention(spec, b, cache.values(), q.contiguous(), o, layer=1)
        h_ref = f64(x) + oracle.linear(f64(o), w["w_o"])
        assert rel_err(f64(hres) - f64(x), h_ref - f64(x)) <= tol
        up = oracle.linear(norm(f64(hres), "norm2"), w["w_up"])
        m_ref = oracle.silu(up[:, :m.ffn]) * up[:, m.ffn:] if m.norm == "rms" else oracle.gelu(up)
        assert rel_err(f64(act), m_ref) <= tol
        d_ref = oracle.linear(f64(act), w["w_down"])
        assert delta_err(f64(y), f64(hres) + d_ref, d_ref, dtype) <= tol


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_model_step_is_its_layers(dtype):
    spec = Spec(dtype=dtype, heads=6, kv_heads=2, dim=64, block=32, rot=64, norm=True, layers=3, slots=3, seq=200)
    m, a, b = Model(spec), Cache(spec), Cache(spec)
    for it, batch in enumerate([Batch(chunks=[(1, 0, 70)]), Batch(chunks=[(2, 0, 33)], decodes=[(1, 70)])]):
        x = rows(spec, batch.T, m.hidden, it)
        ws, n = m.workspace(batch.T, len(batch.chunks))
        y = m.step(a, batch, x, ws, n)
        z = x
        for layer in range(3):
            z = m.layer(b, layer, batch, z, ws, n)
        assert torch.equal(y, z) and torch.equal(a.mem, b.mem) and bool(torch.isfinite(y.float()).all())


def test_captured_step_replays():
    spec = Spec(heads=4, kv_heads=2, dim=128, block=64, rot=128, norm=True, layers=2, slots=3, seq=700)
    m, cache = Model(spec, hidden=256), Cache(spec)
    first = Batch(chunks=[(0, 0, 600), (2, 0, 100)])
    ws, n = m.workspace(first.T, 2)
    m.step(cache, first, rows(spec, first.T, 256, 1), ws, n)
    b = Batch(chunks=[(0, 600, 50)], decodes=[(2, 100), (1, 0)])
    x = rows(spec, b.T, 256, 2)
    start, y = cache.mem.clone(), torch.empty_like(x)
    mb, keep = m.batch(b)

    def call():
        S.sarathi_kv8_model_step(m.cfg, m.abi, cache.kv, mb, x.data_ptr(), y.data_ptr(), ws.data_ptr(), n, cur())

    call()
    torch.cuda.synchronize()
    want = y.clone(), cache.mem.clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(3):
        cache.mem.copy_(start)
        y.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(cache.mem, want[1])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_serving_runs_the_scheduled_steps(fmt):
    """run_schedule with an 8-bit cache leaves what its scheduler's iterations, called one by one, leave."""
    reqs = [(40, 5), (23, 7), (64, 0), (10, 12)]
    shape = dataclasses.replace(wl.TINY.shape, dtype="bf16")
    L, seq = 2, 64
    a, b = (serve.ServeModel(shape, L, 3, seq, 128, seed=4, max_chunks=2, kv8=fmt, kv8_block=32) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((len(reqs), seq, shape.hidden), device="cuda", generator=g).to(torch.bfloat16)
    got, want = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    serve.run_schedule(a, S.POLICY_DECODE_MAXIMAL, reqs, 3, 16, inputs=x, outputs=got)
    sched = S.Scheduler(S.POLICY_DECODE_MAXIMAL, max_batch=3, n_slots=3, max_seq_len=seq, chunk=16)
    for p, d in reqs:
        sched.submit(p, d)
    ws, n = torch.empty(b.ws_bytes, dtype=torch.uint8, device="cuda"), b.ws_bytes
    while (st := sched.next()).n_tokens:
        r = serve._rows(st)
        xi = x[r[0], r[1]]
        yi = torch.empty_like(xi)
        mb, keep = st.mixed_batch()
        S.sarathi_kv8_model_step(b.cfg, list(b.wabi), b.kv, mb, xi.data_ptr(), yi.data_ptr(), ws.data_ptr(), n, cur())
        want[r[0], r[1]] = yi
        sched.commit()
    torch.cuda.synchronize()
    done = torch.zeros(x.shape[:2], dtype=torch.bool)
    for i, (p, d) in enumerate(reqs):
        done[i, :p + d] = True
    assert torch.equal(got[done], want[done]) and bool(torch.isfinite(got[done].float()).all())
    assert bool(got[~done].isnan().all()) and torch.equal(a.kv_t, b.kv_t)
