"""The 8-bit KV cache on the host: sizes and layout, every refusal (found before
any launch: no GPU needed), and pins of its oracle."""
import ctypes as ct
import math

import numpy as np
import pytest

from oracle import kv8 as ref
from paper_2308_16369_amd import sarathi as S

FAKE = 0x100000   # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    return S.lib()


def cfg(**kw):
    base = dict(n_heads=8, n_kv_heads=2, head_dim=64, n_layers=2, block=32)
    base.update(kw)
    return S.make_kv8_cfg(**base)


def test_bytes_and_layout(lib):
    c = cfg()
    n = S.sarathi_kv8_bytes(c, 5, 100)
    codes = 2 * 5 * 2 * 2 * 100 * 64
    at = -(-codes // 256) * 256
    assert n == at + 4 * 2 * 5 * 2 * 2 * 4
    L = S.sarathi_kv8_alloc(c, 5, 100, FAKE, n).layout()
    assert (L.pos, L.head, L.kv, L.slot, L.layer) == (64, 6400, 12800, 25600, 128000)
    assert (L.scale_head, L.scale_kv, L.scale_slot, L.scale_layer, L.scale_offset) == (4, 8, 16, 80, at)


BAD_CFG = [
    (dict(head_dim=96), S.EUNSUPPORTED), (dict(dtype=2), S.EUNSUPPORTED), (dict(n_heads=0), S.EUNSUPPORTED),
    (dict(n_heads=5000, n_kv_heads=5000), S.EUNSUPPORTED), (dict(n_kv_heads=3), S.EINVAL), (dict(n_kv_heads=0), S.EINVAL),
    (dict(n_heads=129, n_kv_heads=1), S.EUNSUPPORTED), (dict(n_layers=0), S.EINVAL), (dict(format=2), S.EUNSUPPORTED),
    (dict(block=8), S.EUNSUPPORTED), (dict(block=48), S.EUNSUPPORTED), (dict(block=256), S.EUNSUPPORTED),
    (dict(softmax_scale=-1.0), S.EINVAL), (dict(softmax_scale=float("nan")), S.EINVAL),
    (dict(softmax_scale=float("inf")), S.EINVAL), (dict(qk_norm=2), S.EINVAL), (dict(qk_norm=1, qk_eps=0.0), S.EINVAL),
    (dict(rope_dim=-16), S.EINVAL), (dict(rope_dim=80), S.EINVAL), (dict(rope_dim=24), S.EUNSUPPORTED),
    (dict(rope_dim=64, rope_layout=2), S.EUNSUPPORTED), (dict(rope_dim=64, rope_scaling=4), S.EUNSUPPORTED),
    (dict(rope_dim=64, rope_base=1.0), S.EINVAL), (dict(rope_dim=64, rope_base=float("nan")), S.EINVAL),
    (dict(rope_dim=64, rope_scaling=S.ROPE_LINEAR, rope_factor=0.5), S.EINVAL),
    (dict(rope_dim=64, rope_scaling=S.ROPE_BANDS, rope_factor=4.0, rope_low=8.0, rope_high=8.0, rope_orig_len=64), S.EINVAL),
    (dict(rope_dim=64, rope_scaling=S.ROPE_BANDS, rope_factor=4.0, rope_orig_len=0), S.EINVAL),
    (dict(rope_dim=64, rope_mscale=-1.0), S.EINVAL),
]


@pytest.mark.parametrize("kw,code", BAD_CFG, ids=[str(i) for i in range(len(BAD_CFG))])
def test_bad_cfg(lib, kw, code):
    c = cfg(**kw)
    h = ct.c_void_p()
    assert lib.sarathi_kv8_alloc(ct.byref(c), 4, 128, FAKE, 1 << 40, ct.byref(h)) == code, S.sarathi_last_error()
    assert not h and S.sarathi_kv8_bytes(c, 4, 128) == 0 and S.sarathi_kv8_plan_bytes(c, 4, 1, 128) == 0


def test_alloc_refuses(lib):
    c = cfg()
    need, h = S.sarathi_kv8_bytes(c, 4, 128), ct.c_void_p()

    def call(ptr=FAKE, size=need, slots=4, seq=128, p=ct.byref(c), out=ct.byref(h)):
        return lib.sarathi_kv8_alloc(p, slots, seq, ptr, size, out)

    assert call(size=need - 1) == S.ENOSPC
    for kw in (dict(ptr=None), dict(ptr=FAKE + 8), dict(slots=0), dict(seq=0), dict(seq=(1 << 20) + 1), dict(out=None),
               dict(slots=(1 << 20) + 1), dict(p=None)):
        assert call(**kw) == S.EINVAL, kw
    lib.sarathi_kv8_free(None)
    lib.sarathi_kv8_plan_free(None)


def test_sizes_beyond_addressing(lib):
    """Sizes whose product passes 64 bits are refused, never wrapped."""
    c, h = cfg(n_heads=4096, n_kv_heads=4096, head_dim=128, n_layers=64), ct.c_void_p()
    assert S.sarathi_kv8_bytes(c, 1 << 20, 1 << 20) == 0
    assert lib.sarathi_kv8_alloc(ct.byref(c), 1 << 20, 1 << 20, FAKE, (1 << 64) - 1, ct.byref(h)) == S.EUNSUPPORTED and not h
    assert S.sarathi_kv8_bytes(c, (1 << 20) + 1, 64) == 0 and S.sarathi_kv8_bytes(c, 64, (1 << 20) + 1) == 0
    assert S.sarathi_kv8_plan_bytes(cfg(), (1 << 31) - 1, (1 << 31) - 1, 64) > (1 << 40)


BAD_BATCH = [
    ([], [], [], S.EINVAL), ([(4, 0, 1)], [], [], S.EINVAL), ([(-1, 0, 1)], [], [], S.EINVAL),
    ([(0, -1, 4)], [], [], S.ERANGE), ([(0, 0, 0)], [], [], S.ERANGE), ([(0, 100, 29)], [], [], S.ERANGE),
    ([], [0], [128], S.ERANGE), ([], [0], [-1], S.ERANGE), ([], [4], [3], S.EINVAL), ([(1, 0, 4)], [1], [3], S.EINVAL),
    ([], [2, 2], [3, 4], S.EINVAL), ([(1, 0, 4), (1, 4, 4)], [], [], S.EINVAL),
]


@pytest.mark.parametrize("chunks,slots,ctx,code", BAD_BATCH, ids=[str(i) for i in range(len(BAD_BATCH))])
def test_plan_refuses_batches(lib, chunks, slots, ctx, code):
    c = cfg()
    kv = S.sarathi_kv8_alloc(c, 4, 128, FAKE, S.sarathi_kv8_bytes(c, 4, 128))
    b, keep = S.make_mixed_batch(chunks, slots, ctx)
    with pytest.raises(S.SarathiError) as e:
        S.sarathi_kv8_plan_create(kv, b, FAKE, 1 << 40)
    assert e.value.code == code


def test_plan_refuses_arguments(lib):
    c = cfg()
    kv = S.sarathi_kv8_alloc(c, 4, 128, FAKE, S.sarathi_kv8_bytes(c, 4, 128))
    b, keep = S.make_mixed_batch([(0, 0, 8)], [1], [5])
    need, h = S.sarathi_kv8_plan_bytes(c, 9, 1, 128), ct.c_void_p()
    assert need > 0

    def call(k=kv.handle, batch=ct.byref(b), ws=FAKE, size=need, out=ct.byref(h)):
        return lib.sarathi_kv8_plan_create(k, batch, ws, size, None, out)

    assert call(size=need - 1) == S.ENOSPC
    for kw in (dict(k=None), dict(batch=None), dict(ws=None), dict(ws=FAKE + 4), dict(out=None)):
        assert call(**kw) == S.EINVAL, kw
    broken = S.sarathi_mixed_batch(1, None, None, None, 0, None, None)
    assert call(batch=ct.byref(broken)) == S.EINVAL
    assert call(batch=ct.byref(S.sarathi_mixed_batch(0, None, None, None, 1, None, None))) == S.EINVAL
    assert call(batch=ct.byref(S.sarathi_mixed_batch(-1, None, None, None, 0, None, None))) == S.EINVAL
    for args in ((0, 1, 128), (4, -1, 128), (4, 1, 0)):
        assert S.sarathi_kv8_plan_bytes(c, *args) == 0


def test_plan_bytes_grow_with_the_batch(lib):
    """A plan made for the most rows and chunks holds every smaller batch."""
    for kw in (dict(), dict(n_heads=1, n_kv_heads=1), dict(n_heads=100, n_kv_heads=1), dict(n_heads=64, n_kv_heads=64)):
        c = cfg(rope_dim=64, **kw)
        sizes = [S.sarathi_kv8_plan_bytes(c, t, k, 4096) for t, k in ((1, 0), (1, 1), (64, 1), (64, 4), (2048, 4))]
        assert sizes == sorted(sizes) and sizes[0] > 0


def test_operators_refuse_null_plan(lib):
    assert lib.sarathi_kv8_append(None, 0, FAKE, 768, None, None, FAKE, 512, None) == S.EINVAL
    assert lib.sarathi_kv8_attention(None, 0, FAKE, 512, FAKE, 512, None) == S.EINVAL
    assert lib.sarathi_kv8_read(None, 0, S.BF16, FAKE, 128, FAKE, 128, None) == S.EINVAL


# ---------------------------------------------------------------------------- oracle pins

def test_oracle_e4m3_values():
    torch = pytest.importorskip("torch")
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    got = ref.code_values("e4m3")
    assert np.array_equal(got, want, equal_nan=True) and np.nanmax(got) == 448


def test_oracle_half_step_is_half_the_gap():
    v = np.sort(ref.code_values("e4m3")[:127])
    mid = (v[1:] + v[:-1]) / 2
    assert np.array_equal(ref.half_step(v[:-1], "e4m3"), mid - v[:-1])


def test_oracle_scales():
    assert ref.scale_needed(127.0, "int8") == 1 and ref.scale_needed(0.0, "int8") == 0
    assert ref.scale_needed(448.0, "e4m3") == 1 and ref.scale_needed(448.5, "e4m3") == 2 and ref.scale_needed(0.0, "e4m3") == 0
    assert ref.scale_needed(1e-29, "int8") == 0


def test_oracle_thetas():
    t = ref.thetas(64, 10000.0)
    assert t[0] == 1 and np.allclose(t[1:] / t[:-1], 10000 ** (-1 / 32))
    assert np.allclose(ref.thetas(64, 10000.0, "linear", 4.0), t / 4)
    n = ref.thetas(64, 10000.0, "ntk", 4.0)
    assert n[0] == 1 and np.isclose(n[-1], t[-1] / 4)          # the slowest pair is stretched by the factor
    b = ref.thetas(64, 10000.0, "bands", 4.0, 1.0, 8.0, 256)
    fast, slow = 256 * t / (2 * math.pi) >= 8, 256 * t / (2 * math.pi) <= 1
    assert fast.any() and slow.any() and np.allclose(b[fast], t[fast]) and np.allclose(b[slow], t[slow] / 4)
    assert np.all((b <= t * (1 + 1e-12)) & (b >= t / 4 * (1 - 1e-12)))


def test_oracle_rotation_keeps_relative_positions():
    """q_m . k_n depends on m - n alone, and dims past the rotated ones are kept."""
    g = np.random.default_rng(0)
    q, k = g.standard_normal((2, 1, 1, 32))
    th = ref.thetas(16, 100.0)
    for layout in ("half", "interleaved"):
        dots = [float((ref.rotate(q, [m], th, layout)[0, 0, :16] * ref.rotate(k, [m - 3], th, layout)[0, 0, :16]).sum())
                for m in (3, 10, 77)]
        assert np.allclose(dots, dots[0])
        assert np.array_equal(ref.rotate(q, [5], th, layout)[..., 16:], q[..., 16:])
        assert np.isclose((ref.rotate(q, [9], th, layout, 2.0)[..., :16] ** 2).sum(), 4 * (q[..., :16] ** 2).sum())


def test_oracle_attend():
    v = np.arange(12.0).reshape(4, 3)
    o, a, mag = ref.attend(np.zeros(3), np.ones((4, 3)), v, 1.0)
    assert np.allclose(o, v.mean(0)) and np.allclose(a, o) and mag == 0
    o, _, _ = ref.attend(np.array([100.0, 0, 0]), np.eye(4)[:, :3], v, 1.0)
    assert np.allclose(o, v[0])


# ---------------------------------------------------------------------------- decoder layer

def layer_args(lib, **kw):
    kv_cfg = cfg(rope_dim=64)
    model = S.make_cfg(128, 8, 64, 256, n_layers=2)
    kv = S.sarathi_kv8_alloc(kv_cfg, 4, 128, FAKE, S.sarathi_kv8_bytes(kv_cfg, 4, 128))
    b, keep = S.make_mixed_batch([(0, 0, 8)], [1], [5])
    ws = S.sarathi_kv8_workspace_bytes(model, kv_cfg, 9, 1, 128)
    names = ["norm1_g", "w_qkv", "w_o", "norm2_g", "w_up", "w_down"]
    w = S.make_kv8_weights({n: FAKE for n in names})
    args = dict(cfg=ct.byref(model), w=ct.byref(w), kv=kv.handle, layer=0, batch=ct.byref(b), x=FAKE, y=FAKE + (1 << 20),
                ws=FAKE + (4 << 20), size=ws)
    args.update(kw)
    return args, (kv_cfg, model, kv, b, keep, w)


def test_layer_workspace(lib):
    kv_cfg, model = cfg(rope_dim=64), S.make_cfg(128, 8, 64, 256, n_layers=2)
    n = S.sarathi_kv8_workspace_bytes(model, kv_cfg, 9, 1, 128)
    L = S.sarathi_kv8_workspace_layout(model, kv_cfg, 9, 1, 128)
    assert L.total == n > 0 and [L.a, L.qkv, L.o, L.hres, L.m] == sorted([L.a, L.qkv, L.o, L.hres, L.m])
    assert L.o - L.qkv >= 9 * (8 + 2 * 2) * 64 * 2
    for other in (S.make_cfg(128, 4, 64, 256, n_layers=2), S.make_cfg(128, 8, 128, 256, n_layers=2),
                  S.make_cfg(128, 8, 64, 256, n_layers=3), S.make_cfg(128, 8, 64, 256, n_layers=2, dtype=S.F32),
                  S.make_cfg(128, 8, 64, 256, n_layers=2, rope=0),
                  S.make_cfg(128, 8, 64, 256, n_layers=2, rope_base=500000.0)):
        assert S.sarathi_kv8_workspace_bytes(other, kv_cfg, 9, 1, 128) == 0
        with pytest.raises(S.SarathiError):
            S.sarathi_kv8_workspace_layout(other, kv_cfg, 9, 1, 128)
    for bad in ((0, 1, 128), (9, -1, 128), (9, 1, 0)):
        assert S.sarathi_kv8_workspace_bytes(model, kv_cfg, *bad) == 0


def test_layer_refuses(lib):
    def call(step=False, **kw):
        a, keep = layer_args(lib, **kw)
        if step:
            return lib.sarathi_kv8_model_step(a["cfg"], a["w"], a["kv"], a["batch"], a["x"], a["y"], a["ws"], a["size"], None)
        return lib.sarathi_kv8_layer_forward(a["cfg"], a["w"], a["kv"], a["layer"], a["batch"], a["x"], a["y"], a["ws"],
                                             a["size"], None)

    a, keep = layer_args(lib)
    no_w = S.make_kv8_weights({"norm1_g": FAKE})
    off = S.make_kv8_weights({n: FAKE + 4 for n in ("norm1_g", "w_qkv", "w_o", "norm2_g", "w_up", "w_down")})
    other = S.make_cfg(128, 4, 64, 256, n_layers=2)
    empty = S.sarathi_mixed_batch(0, None, None, None, 0, None, None)
    for kw in (dict(cfg=None), dict(w=None), dict(kv=None), dict(layer=2), dict(layer=-1), dict(batch=None), dict(x=None),
               dict(y=None), dict(ws=None), dict(x=FAKE + 2), dict(ws=FAKE + (4 << 20) + 8), dict(y=FAKE),
               dict(y=FAKE + (4 << 20)), dict(x=FAKE + (4 << 20) + 64), dict(w=ct.byref(no_w)), dict(w=ct.byref(off)),
               dict(cfg=ct.byref(other)), dict(batch=ct.byref(empty))):
        assert call(**kw) == S.EINVAL, kw
    assert call(size=a["size"] - 1) == S.ENOSPC
    ws2 = (S.sarathi_kv8_layer_weights * 2)(keep[5], no_w)      # the second layer's weights are missing
    assert call(step=True, w=ws2) == S.EINVAL
    far, keep2 = S.make_mixed_batch([(0, 125, 8)], [], [])
    assert call(batch=ct.byref(far)) == S.ERANGE


def test_layer_needs_gains_with_norms(lib):
    kv_cfg = cfg(rope_dim=64, qk_norm=1)
    kv = S.sarathi_kv8_alloc(kv_cfg, 4, 128, FAKE, S.sarathi_kv8_bytes(kv_cfg, 4, 128))
    names = ["norm1_g", "w_qkv", "w_o", "norm2_g", "w_up", "w_down"]
    for extra in ({}, {"q_gain": FAKE}, {"q_gain": FAKE, "k_gain": FAKE + 2}):
        w = S.make_kv8_weights({**{n: FAKE for n in names}, **extra})
        a, keep = layer_args(lib, w=ct.byref(w), kv=kv.handle)
        assert lib.sarathi_kv8_layer_forward(a["cfg"], a["w"], a["kv"], 0, a["batch"], a["x"], a["y"], a["ws"], a["size"],
                                             None) == S.EINVAL
        assert "gain" in S.sarathi_last_error()


def test_serving_equation_counts_the_smaller_cache():
    import workloads as wl
    from paper_2308_16369_amd import serve

    shape, mem = wl.LLAMA13B_LAYER.shape, 288 * 10 ** 9
    full, half = (serve.equation_batch(shape, 40, 1024, mem, kv8_block=b) for b in (0, 64))
    assert half["kv_bytes_per_token"] == 40 * 2 * 40 * (128 + 4 / 64)
    assert 1.99 * full["B"] <= half["B"] + 1 <= 2 * full["B"] + 2
