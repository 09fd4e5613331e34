"""The 8-bit KV cache's operators against the float64 oracle: append (head
norms, rotary variants, scales and codes), attention and read, at the sizes
where they can go wrong."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from kv8_harness import (Batch, Cache, Spec, check_append, check_attention, cur, expected_rows, f64,  # noqa: E402
                         make_rows)
from oracle import kv8 as ref  # noqa: E402
from paper_2308_16369_amd import sarathi as S  # noqa: E402


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def append(cache, batch, qkv, gains, q_out=None, layer=0, plan=None):
    spec = cache.spec
    plan = plan or cache.plan(batch)
    q_out = torch.full((batch.T, spec.heads * spec.dim), 7.0, dtype=spec.tdt, device="cuda") if q_out is None else q_out
    S.sarathi_kv8_append(plan, layer, qkv.data_ptr(), qkv.stride(0), gains[0].data_ptr() if spec.norm else 0,
                         gains[1].data_ptr() if spec.norm else 0, q_out.data_ptr(), q_out.stride(0), cur())
    torch.cuda.synchronize()
    return q_out


def append_and_check(cache, batch, seed, layer=0):
    spec = cache.spec
    qkv, gains = make_rows(spec, batch.T, gen(seed), ld_extra=16)
    before = cache.host()
    kept = qkv.clone()
    q_out = append(cache, batch, qkv, gains, layer=layer)
    assert torch.equal(kept.view(torch.uint8), qkv.view(torch.uint8))
    q, k, v = expected_rows(spec, qkv, gains, [p for _, p in batch.rows()])
    check_append(spec, batch, before, cache.host(), q_out, q, k, v, layer=layer)
    assert cache.guards_intact()


# chunk starts and ends inside blocks, single rows, whole blocks, several of them, decodes at block borders
BATCHES = [
    Batch(chunks=[(1, 0, 1)]),
    Batch(chunks=[(2, 0, 150)], decodes=[(0, 0)]),
    Batch(chunks=[(0, 0, 33), (3, 0, 16)], decodes=[(1, 0), (2, 0)]),
]


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,heads,kv_heads,block", [(64, 4, 4, 16), (64, 6, 2, 128), (128, 5, 1, 32), (128, 3, 3, 64),
                                                      (128, 9, 3, 128), (64, 16, 2, 64), (128, 2, 2, 16)])
def test_append_fresh_and_grown(fmt, dtype, dim, heads, kv_heads, block):
    """Fresh blocks, then rows into started ones: scales grow, earlier codes are rounded to them."""
    spec = Spec(heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, fmt=fmt, block=block, rot=dim)
    cache = Cache(spec)
    for i, b in enumerate(BATCHES):
        append_and_check(cache, b, 10 * i)
    append_and_check(cache, Batch(chunks=[(2, 150, 41)], decodes=[(0, 33), (3, 16), (1, 1)]), 77)
    append_and_check(cache, Batch(chunks=[(1, 2, 70)], decodes=[(2, 191), (0, 34), (3, 17)]), 78)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dim,rot,scaling,norm", [(64, 64, "plain", True), (128, 128, "linear", False), (128, 32, "ntk", True),
                                                  (64, 16, "bands", False), (128, 96, "bands", True), (64, 48, "linear", True),
                                                  (128, 0, "plain", True), (128, 112, "plain", False)])
def test_append_rotary_and_norms(layout, dim, rot, scaling, norm):
    for dtype in ("f32", "bf16"):
        spec = Spec(heads=6, kv_heads=3, dim=dim, dtype=dtype, fmt="e4m3", block=32, rot=rot, layout=layout, scaling=scaling,
                    factor=1.0 if scaling == "plain" else 4.0, norm=norm, mscale=1.25 if scaling == "bands" else 0.0)
        cache = Cache(spec)
        append_and_check(cache, Batch(chunks=[(0, 0, 40)], decodes=[(2, 0)]), 3)
        append_and_check(cache, Batch(chunks=[(0, 40, 7)], decodes=[(2, 1)]), 4)


def test_append_far_positions():
    """Angles of positions near 2^20 (fp64 reduction) and a slot longer than 4 GiB of codes."""
    spec = Spec(heads=16, kv_heads=16, dim=128, dtype="f32", fmt="int8", block=64, rot=128, slots=2, seq=(1 << 20) - 3)
    c = spec.cfg()
    size = S.sarathi_kv8_bytes(c, spec.slots, spec.seq)
    assert size > 8 << 30
    mem = torch.empty(size, dtype=torch.uint8, device="cuda")
    kv = S.sarathi_kv8_alloc(c, spec.slots, spec.seq, mem.data_ptr(), size)
    lay = kv.layout()
    off, n = spec.seq - 20, 20
    batch, keep = S.make_mixed_batch([(1, off, n)], [], [])
    wsz = S.sarathi_kv8_plan_bytes(c, n, 1, spec.seq)
    ws = torch.empty(wsz, dtype=torch.uint8, device="cuda")
    plan = S.sarathi_kv8_plan_create(kv, batch, ws.data_ptr(), wsz, cur())
    qkv, gains = make_rows(spec, n, gen(5))
    # earlier positions of the first touched block: a zero scale
    at = lay.scale_offset // 4 + lay.scale_slot
    scales = mem.view(torch.float32)[at:at + 2 * lay.scale_kv].view(2, 16, lay.scale_head)
    scales.zero_()
    q_out = torch.empty((n, 16 * 128), dtype=torch.float32, device="cuda")
    S.sarathi_kv8_append(plan, 0, qkv.data_ptr(), qkv.stride(0), 0, 0, q_out.data_ptr(), 16 * 128, cur())
    k_out, v_out = torch.empty((2, n, 16 * 128), dtype=torch.float32, device="cuda")
    S.sarathi_kv8_read(plan, 0, S.F32, k_out.data_ptr(), 16 * 128, v_out.data_ptr(), 16 * 128, cur())
    torch.cuda.synchronize()
    q, k, v = expected_rows(spec, qkv, gains, range(off, off + n))
    assert np.max(np.abs(f64(q_out).reshape(q.shape) - q)) <= 2.0 ** -18 * np.abs(q).max()
    s = scales.cpu().numpy().astype(np.float64)[:, :, off // 64:]
    step = np.repeat(s, 64, -1)[:, :, off % 64:off % 64 + n]                     # [2, head, pos]
    for got, want, st in ((k_out, k, step[0]), (v_out, v, step[1])):
        err = np.abs(f64(got).reshape(want.shape) - want)
        assert np.all(err <= 0.5 * st.T[:, :, None] + 2.0 ** -18 * np.abs(want).max())


def test_append_sines_are_rounded_once():
    """fp32 heads of ones and zeros turn into the table's cosines and sines: half a step from the float64 ones (and
    the float64 angle's own roundings: three of a half 2^-52 of up to 2100 radians, below 1e-12)."""
    spec = Spec(heads=1, kv_heads=1, dim=128, dtype="f32", rot=128, layout="interleaved", slots=2, seq=2100)
    cache = Cache(spec)
    b = Batch(chunks=[(0, 0, 2099)], decodes=[(1, 1777)])
    qkv = torch.zeros((b.T, 3 * 128), device="cuda")
    qkv[:, 0:128:2] = 1
    q = f64(append(cache, b, qkv, [qkv, qkv]))
    ang = np.array([p for _, p in b.rows()], dtype=np.float64)[:, None] * np.asarray(spec.thetas())
    for got, want in ((q[:, 0::2], np.cos(ang)), (q[:, 1::2], np.sin(ang))):
        assert np.all(np.abs(got - want) <= 2.0 ** -24 * np.abs(want) + 1e-12)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_append_non_finite_zero_and_tiny(fmt):
    """Infinities become the largest code, NaN zero, neither moves the scale; zero and tiny blocks have scale 0."""
    spec = Spec(heads=2, kv_heads=2, dim=64, dtype="f32", fmt=fmt, block=16)
    cache = Cache(spec)
    qkv, gains = make_rows(spec, 40, gen(1))
    k0 = 2 * 64
    qkv[3, k0 + 5], qkv[3, k0 + 6], qkv[3, k0 + 7] = float("inf"), float("-inf"), float("nan")
    qkv[16:32, k0:k0 + 64] = 0
    qkv[32:40, k0:k0 + 64] = 1e-35
    append(cache, Batch(chunks=[(0, 0, 40)]), qkv, gains)
    codes, scales = cache.host()
    v = ref.code_values(fmt)[codes[0, 0, 0, 0]]
    top = np.nan_to_num(f64(qkv)[:16, k0:k0 + 64], nan=0, posinf=0, neginf=0)
    assert np.isclose(scales[0, 0, 0, 0, 0], ref.scale_needed(np.abs(top).max(), fmt), rtol=2e-7)
    assert (v[3, 5], v[3, 6], v[3, 7]) == (ref.QMAX[fmt], -ref.QMAX[fmt], 0.0)
    assert scales[0, 0, 0, 0, 1] == 0 and not v[16:32].any()
    assert scales[0, 0, 0, 0, 2] == 0 and not v[32:40].any()
    # a block of scale 0 takes in larger values later
    qkv2, _ = make_rows(spec, 1, gen(2))
    append(cache, Batch(decodes=[(0, 40)]), qkv2, gains)
    codes, scales = cache.host()
    v = ref.code_values(fmt)[codes[0, 0, 0, 0]]
    assert scales[0, 0, 0, 0, 2] > 0 and not v[32:40].any() and np.abs(v[40]).max() > 100


def test_append_in_place():
    spec = Spec(heads=6, kv_heads=2, dim=128, rot=128, norm=True, block=32)
    batch = Batch(chunks=[(0, 0, 37)], decodes=[(1, 0), (3, 0)])
    a, b = Cache(spec), Cache(spec)
    qkv, gains = make_rows(spec, batch.T, gen(9))
    q = append(a, batch, qkv, gains)
    inp = qkv.clone()
    append(b, batch, inp, gains, q_out=inp)
    nq = spec.heads * spec.dim
    assert torch.equal(inp[:, :nq], q) and torch.equal(inp[:, nq:], qkv[:, nq:])
    assert torch.equal(a.mem, b.mem)


def test_append_writes_one_layer():
    spec = Spec(layers=3, heads=4, kv_heads=4, dim=64, rot=64)
    cache = Cache(spec)
    append_and_check(cache, Batch(chunks=[(2, 0, 20)], decodes=[(0, 0)]), 5, layer=1)
    append_and_check(cache, Batch(chunks=[(2, 0, 20)], decodes=[(0, 0)]), 6, layer=2)


# ---------------------------------------------------------------------------- read

@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_read_is_code_times_scale(fmt, out):
    spec = Spec(heads=6, kv_heads=3, dim=64, fmt=fmt, layers=2)
    cache = Cache(spec)
    cache.fill(gen(3))
    batch = Batch(chunks=[(1, 0, 300), (3, 77, 5)], decodes=[(0, 299), (2, 0)])
    tdt = torch.bfloat16 if out == "bf16" else torch.float32
    cols = 3 * 64
    k, v = torch.full((2, batch.T, cols + 8), 5.0, dtype=tdt, device="cuda")
    S.sarathi_kv8_read(cache.plan(batch), 1, S.BF16 if out == "bf16" else S.F32, k.data_ptr(), cols + 8, v.data_ptr(),
                       cols + 8, cur())
    only = torch.full((batch.T, cols), 5.0, dtype=tdt, device="cuda")
    S.sarathi_kv8_read(cache.plan(batch), 1, S.BF16 if out == "bf16" else S.F32, 0, 0, only.data_ptr(), cols, cur())
    codes, scales = cache.views()
    val = codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float()
    val = val * scales.repeat_interleave(spec.block, -1)[..., :spec.seq, None]
    for i, (slot, pos) in enumerate(batch.rows()):
        want = val[1, slot, :, :, pos].reshape(2, -1).to(tdt)
        assert torch.equal(k[i, :cols], want[0]) and torch.equal(v[i, :cols], want[1]) and torch.equal(only[i], want[1])
    assert bool((k[:, cols:] == 5).all()) and bool((v[:, cols:] == 5).all())


# ---------------------------------------------------------------------------- attention

def attend(cache, batch, q, layer=0, extra=0, plan=None):
    spec = cache.spec
    out = torch.full((batch.T, spec.heads * spec.dim + extra), 3.0, dtype=spec.tdt, device="cuda")
    S.sarathi_kv8_attention(plan or cache.plan(batch), layer, q.data_ptr(), q.stride(0), out.data_ptr(), out.stride(0), cur())
    torch.cuda.synchronize()
    if extra:
        assert bool((out[:, -extra:] == 3).all())
    return out[:, :spec.heads * spec.dim]


def poison_unwritten(cache, batch, layer=0):
    """Positions past every sequence's last one: NaN codes and, where the block holds no valid position, NaN scales."""
    codes, scales = cache.views()
    last = {}
    for s, o, n in batch.seqs():
        last[s] = o + n
    for s in range(cache.spec.slots):
        end = last.get(s, 0)
        codes[layer, s, :, :, end:] = 255
        scales[layer, s, :, :, -(-end // cache.spec.block):] = float("nan")


ATTN_BATCHES = {
    "one key": Batch(chunks=[(0, 0, 1)], decodes=[(1, 0)]),
    "decodes": Batch(decodes=[(3, 15), (0, 16), (2, 31), (1, 299)]),
    "chunk from 0": Batch(chunks=[(2, 0, 130)]),
    "chunk in the middle": Batch(chunks=[(1, 63, 67)], decodes=[(0, 127), (2, 128)]),
    "several chunks": Batch(chunks=[(3, 0, 5), (0, 199, 33), (1, 255, 1)], decodes=[(2, 200)]),
}


@pytest.mark.parametrize("batch", ATTN_BATCHES, ids=lambda s: s.replace(" ", "_"))
@pytest.mark.parametrize("dtype,fmt", [("bf16", "int8"), ("bf16", "e4m3"), ("f32", "int8"), ("f32", "e4m3")])
@pytest.mark.parametrize("dim,heads,kv_heads,block", [(64, 4, 4, 16), (128, 5, 1, 32), (128, 4, 4, 128), (64, 24, 1, 64)])
def test_attention(batch, dtype, fmt, dim, heads, kv_heads, block):
    spec = Spec(heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, fmt=fmt, block=block)
    cache = Cache(spec)
    cache.fill(gen(11))
    b = ATTN_BATCHES[batch]
    poison_unwritten(cache, b)
    q = torch.randn((b.T, heads * dim + 24), device="cuda", generator=gen(12)).to(spec.tdt)
    out = attend(cache, b, q, extra=8)
    check_attention(spec, b, cache.values(), q[:, :heads * dim], out)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (40, 1), (128, 1), (34, 2), (3, 3)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_head_groups(heads, kv_heads, dtype):
    """Groups of one head, more than 16, and as many as a block has rows."""
    spec = Spec(heads=heads, kv_heads=kv_heads, dim=64, dtype=dtype, fmt="int8", block=32)
    cache = Cache(spec)
    cache.fill(gen(21))
    b = Batch(chunks=[(1, 30, 9)], decodes=[(0, 100), (2, 3)])
    q = torch.randn((b.T, heads * 64), device="cuda", generator=gen(22)).to(spec.tdt)
    check_attention(spec, b, cache.values(), q, attend(cache, b, q))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_split_keys(fmt, dtype):
    """Few rows over long contexts: decodes and chunk rows split over their keys and joined."""
    spec = Spec(heads=4, kv_heads=2, dim=128, dtype=dtype, fmt=fmt, block=64, seq=5000, slots=3)
    cache = Cache(spec)
    cache.fill(gen(31))
    b = Batch(chunks=[(1, 4500, 70)], decodes=[(0, 4998), (2, 1023)])
    poison_unwritten(cache, b)
    q = torch.randn((b.T, 4 * 128), device="cuda", generator=gen(32)).to(spec.tdt)
    check_attention(spec, b, cache.values(), q, attend(cache, b, q))


def test_attention_peaked_and_scaled():
    """Large scores (weights on one key), a softmax scale of one's own, scales that differ by 2^60 and zero blocks."""
    for dtype in ("bf16", "f32"):
        spec = Spec(heads=4, kv_heads=4, dim=64, dtype=dtype, fmt="e4m3", block=16, softmax_scale=0.5)
        cache = Cache(spec)
        cache.fill(gen(41))
        codes, scales = cache.views()
        scales[0, 0, 1, :, 3] *= 2.0 ** 60
        scales[0, 1, 1, :, 3] *= 2.0 ** -60
        codes[0, 2, :, :, 32:64] = 0
        scales[0, 2, :, :, 2:4] = 0
        b = Batch(chunks=[(0, 40, 90), (2, 0, 100)], decodes=[(1, 200), (3, 299)])
        q = torch.randn((b.T, 4 * 64), device="cuda", generator=gen(42)).to(spec.tdt)
        check_attention(spec, b, cache.values(), q, attend(cache, b, q))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_int8_scales_far_apart(dtype):
    """Value scales 2^60 apart, zero blocks, query heads of magnitude 2^-40 and with one strong element."""
    spec = Spec(heads=4, kv_heads=2, dim=64, dtype=dtype, fmt="int8", block=32)
    cache = Cache(spec)
    cache.fill(gen(43))
    codes, scales = cache.views()
    scales[0, 0, 1, :, 1] *= 2.0 ** 60
    scales[0, 1, 1, :, 2] *= 2.0 ** -60
    codes[0, 2, :, :, 64:96] = 0
    scales[0, 2, :, :, 2] = 0
    b = Batch(chunks=[(0, 40, 90)], decodes=[(1, 200), (3, 299), (2, 250)])
    q = torch.randn((b.T, 4 * 64), device="cuda", generator=gen(44))
    q[-2, 64:128] *= 2.0 ** -40
    q[-1, :64] *= 2.0 ** -20
    q[-1, 7] = 3.0
    q = q.to(spec.tdt)
    check_attention(spec, b, cache.values(), q, attend(cache, b, q))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_small_weights_keep_their_bits(dtype, fmt):
    """One key outweighs the others 2^22 times and has a zero value: the output is the others' alone."""
    spec = Spec(heads=2, kv_heads=1, dim=64, dtype=dtype, fmt=fmt, block=16)
    cache = Cache(spec)
    cache.fill(gen(45))
    codes, scales = cache.views()
    codes[:, :, 0] = 0                                     # keys: zero but the first, of ones
    codes[:, :, 0, :, 0] = 1 if fmt == "int8" else 0x38
    codes[:, :, 1, :, 0] = 0                               # its value
    # q of ones: score 64 scale / sqrt(64) = 22 log 2
    scales[:, :, 0] = 22 * 0.6931471805599453 / 8
    b = Batch(chunks=[(1, 60, 70)], decodes=[(0, 31), (2, 299)])
    q = torch.ones((b.T, 2 * 64), device="cuda", dtype=spec.tdt)
    check_attention(spec, b, cache.values(), q, attend(cache, b, q), scales=cache.host()[1])


@pytest.mark.parametrize("dim,fmt", [(64, "e4m3"), (128, "int8"), (128, "e4m3")])
def test_attention_many_blocks(dim, fmt):
    """So many heads times query blocks that a block's keys stay with one group of waves."""
    spec = Spec(heads=64, kv_heads=64, dim=dim, fmt=fmt, block=64, seq=620, slots=2)
    cache = Cache(spec)
    cache.fill(gen(46))
    b = Batch(chunks=[(1, 11, 600)])
    poison_unwritten(cache, b)
    q = torch.randn((b.T, 64 * dim), device="cuda", generator=gen(47)).to(spec.tdt)
    out, values = attend(cache, b, q), cache.values()
    for first, n in ((0, 6), (126, 5), (595, 5)):
        check_attention(spec, Batch(chunks=[(1, 11 + first, n)]), values, q[first:first + n], out[first:first + n])


def test_attention_non_finite_rows_stay_alone():
    """A NaN or infinite query row spoils its own output only."""
    spec = Spec(heads=4, kv_heads=2, dim=64, fmt="int8", block=16)
    cache = Cache(spec)
    cache.fill(gen(51))
    b = Batch(chunks=[(0, 10, 40)], decodes=[(1, 70), (2, 8)])
    q = torch.randn((b.T, 4 * 64), device="cuda", generator=gen(52)).to(spec.tdt)
    clean = attend(cache, b, q)
    bad = q.clone()
    bad[5, :64], bad[40, 64:128] = float("nan"), float("inf")
    out = attend(cache, b, bad)
    assert bool(out[5, :64].isnan().all()) and bool(out[40, 64:128].isnan().all())
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[5, :64] = False
    keep[40, 64:128] = False
    assert torch.equal(out[keep], clean[keep])


def test_attention_is_deterministic():
    spec = Spec(heads=8, kv_heads=2, dim=128, fmt="int8", block=32, seq=3000, slots=6)
    cache = Cache(spec)
    cache.fill(gen(61))
    b = Batch(chunks=[(1, 2000, 300)], decodes=[(0, 2999), (2, 17), (5, 1500)])
    q = torch.randn((b.T, 8 * 128), device="cuda", generator=gen(62)).to(spec.tdt)
    first = attend(cache, b, q)
    plan = cache.plan(b)
    for _ in range(3):
        assert torch.equal(first, attend(cache, b, q, plan=plan))


# ---------------------------------------------------------------------------- together

def test_chunked_prompt_then_decodes():
    """A prompt in chunks, then decodes: append and attention of every iteration, against float64 over the values
    that the cache holds, and the values against the rows they came from."""
    spec = Spec(heads=6, kv_heads=2, dim=64, dtype="bf16", fmt="int8", block=32, rot=64, norm=True, slots=2, seq=200)
    cache = Cache(spec)
    g = gen(71)
    done = {0: 0, 1: 0}
    steps = [Batch(chunks=[(0, 0, 50)]), Batch(chunks=[(0, 50, 45), (1, 0, 31)]), Batch(chunks=[(1, 31, 64)], decodes=[(0, 95)])]
    steps += [Batch(decodes=[(0, 96 + i), (1, 95 + i)]) for i in range(4)]
    for b in steps:
        qkv, gains = make_rows(spec, b.T, g)
        before = cache.host()
        q_out = append(cache, b, qkv, gains)
        q, k, v = expected_rows(spec, qkv, gains, [p for _, p in b.rows()])
        check_append(spec, b, before, cache.host(), q_out, q, k, v)
        check_attention(spec, b, cache.values(), q_out, attend(cache, b, q_out))
        for s, o, n in b.seqs():
            assert done[s] == o
            done[s] = o + n


def test_captured_calls_replay():
    """Plan, append, attention and read captured; replays among eager work equal the eager calls."""
    spec = Spec(heads=4, kv_heads=2, dim=128, fmt="e4m3", block=64, rot=128, norm=True, seq=700)
    b = Batch(chunks=[(1, 300, 70)], decodes=[(0, 650), (2, 13)])
    cache = Cache(spec)
    cache.fill(gen(81))
    start = cache.mem.clone()
    qkv, gains = make_rows(spec, b.T, gen(82))
    nq = spec.heads * spec.dim
    q, o = torch.empty((2, b.T, nq), dtype=spec.tdt, device="cuda")
    k, v = torch.empty((2, b.T, 2 * spec.dim), dtype=spec.tdt, device="cuda")
    size = S.sarathi_kv8_plan_bytes(cache.c, b.T, 1, spec.seq)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    mb, keep = S.make_mixed_batch(list(b.chunks), [0, 2], [650, 13])

    def call():
        plan = S.sarathi_kv8_plan_create(cache.kv, mb, ws.data_ptr(), size, cur())
        S.sarathi_kv8_append(plan, 0, qkv.data_ptr(), qkv.stride(0), gains[0].data_ptr(), gains[1].data_ptr(), q.data_ptr(),
                             nq, cur())
        S.sarathi_kv8_attention(plan, 0, q.data_ptr(), nq, o.data_ptr(), nq, cur())
        S.sarathi_kv8_read(plan, 0, S.BF16, k.data_ptr(), 256, v.data_ptr(), 256, cur())
        plan.free()

    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in (q, o, k, v, cache.mem)]
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    for _ in range(3):
        cache.mem.copy_(start)
        for t in (q, o, k, v):
            t.fill_(float("nan"))
        ws.random_(0, 255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((q, o, k, v, cache.mem), want):
            assert torch.equal(got.view(torch.uint8), w.view(torch.uint8))


def test_plans_on_two_streams():
    """Two plans in memory of their own, used on two streams at once, over one cache."""
    spec = Spec(heads=8, kv_heads=4, dim=128, fmt="int8", block=32, seq=2000, slots=4)
    cache = Cache(spec)
    cache.fill(gen(91))
    batches = [Batch(decodes=[(0, 1999), (1, 1500)]), Batch(chunks=[(2, 1000, 200)], decodes=[(3, 700)])]
    qs = [torch.randn((b.T, 8 * 128), device="cuda", generator=gen(92 + i)).to(spec.tdt) for i, b in enumerate(batches)]
    want = [attend(cache, b, q) for b, q in zip(batches, qs)]
    streams = [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    outs = [torch.empty_like(q) for q in qs]
    plans = [cache.plan(b, s.cuda_stream) for b, s in zip(batches, streams)]
    for _ in range(5):
        for p, q, o, s in zip(plans, qs, outs, streams):
            S.sarathi_kv8_attention(p, 0, q.data_ptr(), 8 * 128, o.data_ptr(), 8 * 128, s.cuda_stream)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


# ---------------------------------------------------------------------------- refusals with a plan in hand

def test_operators_refuse_arguments():
    spec = Spec(heads=4, kv_heads=2, dim=64, norm=True)
    cache = Cache(spec)
    plan = cache.plan(Batch(chunks=[(0, 0, 4)]))
    x = torch.zeros((8, 1024), dtype=torch.bfloat16, device="cuda")
    y = torch.zeros((8, 1024), dtype=torch.bfloat16, device="cuda")
    g = torch.ones(64, dtype=torch.bfloat16, device="cuda").data_ptr()
    px, py, lib = x.data_ptr(), y.data_ptr(), S.lib()
    kept = cache.mem.clone()

    def append(layer=0, qkv=px, ld=1024, qg=g, kg=g, q=py, ldq=1024):
        return lib.sarathi_kv8_append(plan.handle, layer, qkv, ld, qg, kg, q, ldq, cur())

    def attention(layer=0, q=px, ldq=1024, out=py, ldo=1024):
        return lib.sarathi_kv8_attention(plan.handle, layer, q, ldq, out, ldo, cur())

    def read(layer=0, dt=S.BF16, k=px, ldk=1024, v=py, ldv=1024):
        return lib.sarathi_kv8_read(plan.handle, layer, dt, k, ldk, v, ldv, cur())

    for kw in (dict(layer=1), dict(layer=-1), dict(qkv=None), dict(q=None), dict(ld=511), dict(ld=516), dict(ldq=255),
               dict(qkv=px + 2), dict(q=py + 8), dict(qg=None), dict(kg=None), dict(qg=g + 2), dict(q=px + 512),
               dict(q=px, ldq=512)):
        assert append(**kw) == S.EINVAL, kw
    for kw in (dict(layer=1), dict(q=None), dict(out=None), dict(ldq=248), dict(ldo=1020), dict(out=px), dict(out=px + 512),
               dict(q=px + 2)):
        assert attention(**kw) == S.EINVAL, kw
    for kw in (dict(layer=2), dict(k=None, v=None), dict(ldk=120), dict(ldv=1025), dict(v=px), dict(k=px + 4)):
        assert read(**kw) == S.EINVAL, kw
    assert read(dt=5) == S.EUNSUPPORTED
    torch.cuda.synchronize()
    assert torch.equal(kept, cache.mem) and not x.any() and not y.any()
