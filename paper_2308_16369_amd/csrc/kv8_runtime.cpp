// Host side of the 8-bit KV cache: argument checks (before anything is
// enqueued), the cache's layout, the batch plan and the operators' launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "host_error.h"
#include "kv8.h"
#include "runtime_internal.h"
#include "sarathi_kv8.h"

using namespace sarathi;

struct sarathi_kv8 {
  sarathi_kv8_cfg cfg;
  int n_slots, max_seq_len;
  char* mem;
  sarathi_kv8_layout st;
  double theta[KV8_MAX_PAIRS];   // angle per position of each rotated pair
};

struct sarathi_kv8_plan {
  sarathi_kv8_cfg cfg;
  char* mem;
  sarathi_kv8_layout st;
  int T;
  int n_chunk_units, n_units;    // touched blocks of chunks, then of decodes
  int n_pre, n_dec;              // attention items of chunks and decodes
  int groups;                    // 4-wave groups of a chunk-attention block
  int comb_row0, comb_rows;      // chunk rows that the combine pass visits: comb_row0 .. comb_rows - 1
  const int* row_slot;           // device
  const int* row_pos;
  const int* comb;
  const int* units;
  const int* chunks;
  const int* pre;
  const int* dec;
  const float2* tab;
  float* part;
  const int* joins;
  int n_joins;
};

namespace {

// Keys up to which a decode is one work item whatever the batch (two steps of
// each of a block's four waves), and the blocks that the decodes of a batch are
// split into where their keys allow it (three per CU, what runs at once).  Items
// are whole steps of all four waves, so a row's last item has what is left: of
// 1025 keys in items of 256, one key.
constexpr int DEC_MIN_KEYS = 256, DEC_STEP = 128;
constexpr long DEC_BLOCKS = 768;
// Chunk attention: key tiles of an item at least, the items that splitting adds
// to a batch at most, the four-wave groups that run at once (two per CU), a
// block's set-up, merge and output in tiles' times (of one and two groups), the
// time of a tile in a block of two groups, and the combine pass in tiles.
constexpr int PRE_MIN_TILES = 4;
constexpr long PRE_SPLIT_BLOCKS = 768, PRE_SLOTS = 512;
constexpr double PRE_FIXED_TILES = 2, PRE_FIXED_TILES_2 = 3, PRE_TILE_2 = 1.15, PRE_JOIN_TILES = 6;
constexpr int MAX_SLOTS = 1 << 20, MAX_SEQ = 1 << 20;
constexpr long MAX_GRID = (1l << 24) - 1;   // blocks of 256 threads in one launch

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
size_t esize(int dtype) { return dtype == SARATHI_BF16 ? 2 : 4; }
int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }

int hip_fail(hipError_t e, const char* what) { return fail(SARATHI_EHIP, "%s: %s", what, hipGetErrorString(e)); }

bool finite_pos(float x) { return x > 0.f && x < INFINITY; }

int check_kv8_cfg(const sarathi_kv8_cfg* c) {
  if (!c) return fail(SARATHI_EINVAL, "cfg is NULL");
  if (c->dtype != SARATHI_F32 && c->dtype != SARATHI_BF16)
    return fail(SARATHI_EUNSUPPORTED, "dtype %d not supported (F32 or BF16)", c->dtype);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(SARATHI_EUNSUPPORTED, "head_dim %d not supported (64 or 128)", c->head_dim);
  if (c->n_heads <= 0 || c->n_heads > 4096) return fail(SARATHI_EUNSUPPORTED, "n_heads %d out of range", c->n_heads);
  if (c->n_kv_heads <= 0 || c->n_heads % c->n_kv_heads)
    return fail(SARATHI_EINVAL, "n_kv_heads %d must divide n_heads %d", c->n_kv_heads, c->n_heads);
  if (c->n_heads / c->n_kv_heads > KV8_QB)
    return fail(SARATHI_EUNSUPPORTED, "%d query heads per key/value head (at most %d)", c->n_heads / c->n_kv_heads, KV8_QB);
  if (c->n_layers <= 0) return fail(SARATHI_EINVAL, "n_layers %d must be positive", c->n_layers);
  if (c->format != SARATHI_KV8_INT8 && c->format != SARATHI_KV8_E4M3) return fail(SARATHI_EUNSUPPORTED, "format %d", c->format);
  if (c->block != 16 && c->block != 32 && c->block != 64 && c->block != 128)
    return fail(SARATHI_EUNSUPPORTED, "block %d not supported (16, 32, 64 or 128)", c->block);
  if (c->softmax_scale != 0.f && !finite_pos(c->softmax_scale)) return fail(SARATHI_EINVAL, "softmax_scale must be > 0 (or 0)");
  if (c->qk_norm != 0 && c->qk_norm != 1) return fail(SARATHI_EINVAL, "qk_norm must be 0 or 1");
  if (c->qk_norm && !finite_pos(c->qk_eps)) return fail(SARATHI_EINVAL, "qk_eps must be > 0");
  if (c->rope_dim < 0 || c->rope_dim > c->head_dim) return fail(SARATHI_EINVAL, "rope_dim %d outside [0, head_dim]", c->rope_dim);
  if (c->rope_dim % 16) return fail(SARATHI_EUNSUPPORTED, "rope_dim %d must be a multiple of 16", c->rope_dim);
  if (c->rope_dim == 0) return SARATHI_OK;
  if (c->rope_layout != SARATHI_ROPE_HALF && c->rope_layout != SARATHI_ROPE_INTERLEAVED)
    return fail(SARATHI_EUNSUPPORTED, "rope_layout %d", c->rope_layout);
  if (c->rope_scaling < SARATHI_ROPE_PLAIN || c->rope_scaling > SARATHI_ROPE_BANDS)
    return fail(SARATHI_EUNSUPPORTED, "rope_scaling %d", c->rope_scaling);
  if (!(c->rope_base > 1.0f) || !finite_pos(c->rope_base)) return fail(SARATHI_EINVAL, "rope_base must be > 1");
  if (c->rope_scaling != SARATHI_ROPE_PLAIN && !(c->rope_factor >= 1.0f && c->rope_factor < INFINITY))
    return fail(SARATHI_EINVAL, "rope_factor must be >= 1");
  if (c->rope_scaling == SARATHI_ROPE_BANDS) {
    if (!(c->rope_low < c->rope_high) || !std::isfinite(c->rope_low) || !std::isfinite(c->rope_high))
      return fail(SARATHI_EINVAL, "rope_low must be below rope_high");
    if (c->rope_orig_len < 1) return fail(SARATHI_EINVAL, "rope_orig_len %d must be positive", c->rope_orig_len);
  }
  if (c->rope_mscale != 0.f && !finite_pos(c->rope_mscale)) return fail(SARATHI_EINVAL, "rope_mscale must be > 0 (or 0)");
  return SARATHI_OK;
}

void rope_thetas(const sarathi_kv8_cfg& c, double* theta) {
  const int r = c.rope_dim;
  const double f = c.rope_scaling == SARATHI_ROPE_PLAIN ? 1.0 : (double)c.rope_factor;
  double base = c.rope_base;
  if (c.rope_scaling == SARATHI_ROPE_NTK) base *= std::pow(f, (double)r / (r - 2));
  for (int i = 0; i < r / 2; ++i) {
    double t = std::pow(base, -2.0 * i / r);
    if (c.rope_scaling == SARATHI_ROPE_LINEAR) t /= f;
    if (c.rope_scaling == SARATHI_ROPE_BANDS) {
      const double turns = c.rope_orig_len * t / 6.283185307179586;
      const double w = std::min(1.0, std::max(0.0, (turns - c.rope_low) / ((double)c.rope_high - c.rope_low)));
      t *= w + (1.0 - w) / f;
    }
    theta[i] = t;
  }
}

sarathi_kv8_layout layout_of(const sarathi_kv8_cfg& c, int n_slots, int S) {
  sarathi_kv8_layout L{};
  L.pos = c.head_dim;
  L.head = (size_t)S * c.head_dim;
  L.kv = L.head * c.n_kv_heads;
  L.slot = L.kv * 2;
  L.layer = L.slot * n_slots;
  L.scale_head = ceil_div(S, c.block);
  L.scale_kv = L.scale_head * c.n_kv_heads;
  L.scale_slot = L.scale_kv * 2;
  L.scale_layer = L.scale_slot * n_slots;
  L.scale_offset = align256(L.layer * c.n_layers);
  return L;
}

// Chunk rows of an attention block, 16-head groups of a key/value head.
int rows_per_block(const sarathi_kv8_cfg& c) { return KV8_QB / (c.n_heads / c.n_kv_heads); }
int head_blocks(const sarathi_kv8_cfg& c) { return (c.n_heads / c.n_kv_heads + 15) / 16; }
// Attention items that splitting adds at most to one per query block / decode.
long extra_pre(const sarathi_kv8_cfg& c) { return PRE_SPLIT_BLOCKS / c.n_kv_heads; }
long extra_dec(const sarathi_kv8_cfg& c) { return DEC_BLOCKS / ((long)c.n_kv_heads * head_blocks(c)) + 1; }

struct PlanLayout {
  size_t rows, tab, meta, part, total;   // rows: row_slot[T], row_pos[T], comb[3 T]
  size_t meta_ints, part_rows;
};
PlanLayout plan_layout(const sarathi_kv8_cfg& c, int T, int n_chunks) {
  PlanLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = align256(off + bytes); return at; };
  const int rpb = rows_per_block(c);
  const long qblocks = (long)(T / rpb) + n_chunks;
  L.rows = take((size_t)T * 5 * 4);
  L.tab = take((size_t)T * (c.rope_dim / 2) * sizeof(float2));
  // spans and touched blocks have a row at least
  L.meta_ints = (size_t)T * KV8_SPAN_INTS + (size_t)T * 4 + 4 * (size_t)n_chunks + 4 * (size_t)(qblocks + extra_pre(c)) +
                KV8_DEC_INTS * (size_t)(T + extra_dec(c)) + KV8_JOIN_INTS * (size_t)T;
  L.meta = take(L.meta_ints * 4);
  L.part_rows = (size_t)(qblocks + extra_pre(c)) * rpb + T + extra_dec(c);
  L.part = take(L.part_rows * c.n_heads * (c.head_dim + PART_O) * 4);
  L.total = off;
  return L;
}

// The batch's work lists and the metadata that goes to the device.
struct HostPlan {
  std::vector<int> spans, units, chunks, pre, dec, joins;
  int n_chunk_units = 0;
  int groups = 1;                // 4-wave groups of a chunk-attention block
  size_t part_rows = 0;
  int comb_row0 = 0;
};

void plan_chunks(const sarathi_kv8_cfg& c, const BatchDesc& b, HostPlan* p) {
  const int rpb = rows_per_block(c);
  struct QB { int chunk, r0, rows, tiles; };
  std::vector<QB> qbs;
  int longest = 1;
  for (size_t ci = 0; ci < b.chunks.size(); ++ci) {
    const ChunkDesc& d = b.chunks[ci];
    for (int r = 0; r < d.len; r += rpb) {
      const int n = std::min(rpb, d.len - r);
      qbs.push_back({(int)ci, r, n, ceil_div(d.offset + r + n, KV8_KT)});
      longest = std::max(longest, qbs.back().tiles);
    }
  }
  // Every query block's tiles are cut into near-equal ranges of at most tau;
  // blocks of one four-wave group, or of two that take the tiles in turn.  The
  // choice that ends first: the longest range or the rounds of average ones,
  // with a block's set-up and output, and the combine pass where rows are split.
  // Two groups finish a block in about half the time without splitting its rows:
  // 512 rows over 2048 keys of 52 heads (208 blocks) took 54 us, one group with
  // rows split in two 64, when both were measured; three prompts of 347 to 910 rows of 32 / 8 heads 48
  // against 61; a 4096-token prompt of 32 / 8 heads (1024 blocks), which fills
  // the GPU either way, 189 against 179 of one group.
  int tau = longest;
  double best = 1e300;
  for (int groups = 1; groups <= (c.dtype == SARATHI_BF16 ? 2 : 1); ++groups) {
    const double fixed = groups == 2 ? PRE_FIXED_TILES_2 : PRE_FIXED_TILES, per_tile = groups == 2 ? PRE_TILE_2 : 1.0;
    const long slots = PRE_SLOTS / groups;
    for (int cand = longest;;) {
      long items = 0, tiles = 0;
      int most = 0;
      for (const QB& q : qbs) {
        const int ns = ceil_div(q.tiles, cand);
        items += ns;
        tiles += q.tiles;
        most = std::max(most, ceil_div(q.tiles, ns));
      }
      if (cand == longest || items <= (long)qbs.size() + extra_pre(c)) {
        const double mean = (double)tiles / std::max(1l, items) / groups;
        const double rounds = ceil_div(items * c.n_kv_heads, slots) * (mean + fixed);
        const double cost = std::max(rounds, ceil_div(most, groups) + fixed) * per_tile +
                            (items > (long)qbs.size() ? PRE_JOIN_TILES : 0);
        if (cost < best) {
          best = cost;
          tau = cand;
          p->groups = groups;
        }
      }
      cand -= std::max(1, cand / 5);
      if (cand < PRE_MIN_TILES) break;
    }
  }
  std::vector<int> row0(b.chunks.size());
  int r0 = 0;
  for (size_t ci = 0; ci < b.chunks.size(); ++ci) {
    const ChunkDesc& d = b.chunks[ci];
    row0[ci] = r0;
    p->chunks.insert(p->chunks.end(), {d.slot, d.offset, d.len, r0});
    // touched blocks of the cache
    for (int pos = d.offset; pos < d.offset + d.len;) {
      const int blk = pos / c.block, end = std::min(d.offset + d.len, (blk + 1) * c.block);
      p->units.insert(p->units.end(), {d.slot, blk, r0 + pos - d.offset, (pos - blk * c.block) << 16 | (end - blk * c.block)});
      pos = end;
    }
    r0 += d.len;
  }
  p->n_chunk_units = (int)p->units.size() / 4;
  struct Item { int v[4]; int tiles; };
  std::vector<Item> items;
  for (const QB& q : qbs) {
    const ChunkDesc& d = b.chunks[q.chunk];
    const int ns = ceil_div(q.tiles, tau);
    const int base = (int)p->part_rows;
    for (int s = 0; s < ns; ++s) {
      const int t0 = (int)((long)q.tiles * s / ns), t1 = (int)((long)q.tiles * (s + 1) / ns);
      items.push_back({{q.chunk, q.r0, ns > 1 ? base + s * rpb : -1, t0 << 16 | t1}, t1 - t0});
    }
    if (ns > 1) p->part_rows += (size_t)ns * rpb;
    for (int r = 0; r < q.rows; r += KV8_SPAN)
      p->spans.insert(p->spans.end(), {d.slot, d.offset + q.r0 + r, row0[q.chunk] + q.r0 + r, std::min(KV8_SPAN, q.rows - r),
                                       base + r, ns > 1 ? ns : 0, rpb});
  }
  // the longest ranges first: the short ones fill the last round
  std::stable_sort(items.begin(), items.end(), [](const Item& x, const Item& y) { return x.tiles > y.tiles; });
  for (const Item& i : items) p->pre.insert(p->pre.end(), i.v, i.v + 4);
}

void plan_decodes(const sarathi_kv8_cfg& c, const BatchDesc& b, int first_row, HostPlan* p) {
  long keys = 0;
  for (int i = 0; i < b.B; ++i) keys += b.dctx[i] + 1;
  const long per_key_range = (long)c.n_kv_heads * head_blocks(c);
  const long target = std::max<long>(DEC_MIN_KEYS, ceil_div(keys * per_key_range, DEC_BLOCKS));
  const int split = ceil_div(target, DEC_STEP) * DEC_STEP;
  // the longest rows first: their blocks start in the first round and short
  // ones fill the last (48 decodes of 512 to 2048 tokens: 105 us, in slot order 115)
  std::vector<int> order(b.B);
  for (int i = 0; i < b.B; ++i) order[i] = i;
  std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return b.dctx[x] > b.dctx[y]; });
  std::vector<int> span(KV8_SPAN_INTS * (size_t)b.B);
  for (int i : order) {
    const int n = b.dctx[i] + 1, want = ceil_div(n, split);
    const int len = ceil_div(ceil_div(n, want), DEC_STEP) * DEC_STEP, ns = ceil_div(n, len);
    for (int s = 0; s < ns; ++s)
      p->dec.insert(p->dec.end(), {first_row + i, b.dslots[i], s * len, std::min(n, (s + 1) * len),
                                   ns > 1 ? (int)p->part_rows + s : -1});
    const int v[KV8_SPAN_INTS] = {b.dslots[i], b.dctx[i], first_row + i, 1, 0, 0, 0};   // its own join
    std::copy(v, v + KV8_SPAN_INTS, span.begin() + KV8_SPAN_INTS * (size_t)i);
    if (ns > 1) {
      p->joins.insert(p->joins.end(), {first_row + i, ns, (int)p->part_rows});
      p->part_rows += ns;
    }
  }
  p->spans.insert(p->spans.end(), span.begin(), span.end());
  for (int i = 0; i < b.B; ++i) {
    const int blk = b.dctx[i] / c.block, p0 = b.dctx[i] - blk * c.block;
    p->units.insert(p->units.end(), {b.dslots[i], blk, first_row + i, p0 << 16 | (p0 + 1)});
  }
}

// The batch's work lists; SARATHI_* code.
int host_plan(const sarathi_kv8_cfg& c, const BatchDesc& b, HostPlan* p) {
  plan_chunks(c, b, p);
  plan_decodes(c, b, b.rows() - b.B, p);
  p->comb_row0 = b.rows();
  for (size_t i = 0; i < p->spans.size(); i += KV8_SPAN_INTS)
    if (p->spans[i + 5] > 0) p->comb_row0 = std::min(p->comb_row0, p->spans[i + 2]);
  const long T = b.rows(), units = (long)p->units.size() / 4;
  const long grids[] = {(long)p->pre.size() / 4 * c.n_kv_heads, (long)p->dec.size() / KV8_DEC_INTS * c.n_kv_heads * head_blocks(c),
                        T * ((c.n_heads + 3) / 4) + units * 2 * c.n_kv_heads, T * 2 * c.n_kv_heads * (c.head_dim / 16) / 256 + 1};
  for (long g : grids)
    if (g > MAX_GRID) return fail(SARATHI_EUNSUPPORTED, "batch of %ld rows x %d heads needs more than %ld blocks", T, c.n_heads, MAX_GRID);
  return SARATHI_OK;
}

struct Span {
  const char* a;
  size_t n;
};
Span rows_span(const void* p, int T, size_t ld, size_t cols, size_t es) {
  return {static_cast<const char*>(p), ((size_t)(T - 1) * ld + cols) * es};
}
bool overlap(const Span& x, const Span& y) { return x.a < y.a + y.n && y.a < x.a + x.n; }

int check_rows(const char* name, const void* p, size_t ld, size_t cols, size_t es) {
  if (!p) return fail(SARATHI_EINVAL, "%s is NULL", name);
  if (ld < cols) return fail(SARATHI_EINVAL, "%s: row stride %zu < %zu", name, ld, cols);
  if (!aligned16(p) || ld * es % 16) return fail(SARATHI_EINVAL, "%s: rows must be 16-byte aligned", name);
  return SARATHI_OK;
}
int check_plan(const sarathi_kv8_plan* plan, int layer) {
  if (!plan) return fail(SARATHI_EINVAL, "plan is NULL");
  if (layer < 0 || layer >= plan->cfg.n_layers) return fail(SARATHI_EINVAL, "layer %d outside [0, %d)", layer, plan->cfg.n_layers);
  return SARATHI_OK;
}

Kv8Layer layer_of(const sarathi_kv8_plan* p, int layer) {
  Kv8Layer L;
  L.codes = reinterpret_cast<uint8_t*>(p->mem) + p->st.layer * layer;
  L.scales = reinterpret_cast<float*>(p->mem + p->st.scale_offset) + p->st.scale_layer * layer;
  L.slot = p->st.slot; L.kv = p->st.kv; L.head = p->st.head;
  L.s_slot = p->st.scale_slot; L.s_kv = p->st.scale_kv; L.s_head = p->st.scale_head;
  L.log2_block = p->cfg.block == 16 ? 4 : p->cfg.block == 32 ? 5 : p->cfg.block == 64 ? 6 : 7;
  return L;
}

// Fills `plan` for a checked batch and enqueues its upload.
int plan_upload(const sarathi_kv8* kv, const BatchDesc& b, void* ws, size_t ws_bytes, hipStream_t s, sarathi_kv8_plan* plan) {
  const sarathi_kv8_cfg& c = kv->cfg;
  if (!ws) return fail(SARATHI_EINVAL, "workspace is NULL");
  if (!aligned16(ws)) return fail(SARATHI_EINVAL, "workspace must be 16-byte aligned");
  const int T = b.rows();
  const PlanLayout L = plan_layout(c, T, (int)b.chunks.size());
  if (ws_bytes < L.total) return fail(SARATHI_ENOSPC, "workspace of %zu bytes < %zu needed", ws_bytes, L.total);
  HostPlan h;
  int rc = host_plan(c, b, &h);
  if (rc) return rc;
  std::vector<int> meta;
  auto put = [&](const std::vector<int>& v) { const size_t at = meta.size(); meta.insert(meta.end(), v.begin(), v.end()); return at; };
  const size_t o_spans = put(h.spans), o_units = put(h.units), o_chunks = put(h.chunks), o_pre = put(h.pre), o_dec = put(h.dec),
               o_joins = put(h.joins);
  if (meta.size() > L.meta_ints || h.part_rows > L.part_rows)   // the bounds hold for every checked batch
    return fail(SARATHI_EINVAL, "internal: batch plan exceeds its workspace layout");
  char* base = static_cast<char*>(ws);
  int* rows = reinterpret_cast<int*>(base + L.rows);
  int* dm = reinterpret_cast<int*>(base + L.meta);
  plan->cfg = c; plan->mem = kv->mem; plan->st = kv->st;
  plan->T = T;
  plan->n_chunk_units = h.n_chunk_units; plan->n_units = (int)h.units.size() / 4;
  plan->n_pre = (int)h.pre.size() / 4; plan->groups = h.groups; plan->n_dec = (int)h.dec.size() / KV8_DEC_INTS;
  plan->comb_row0 = h.comb_row0; plan->comb_rows = T - b.B;
  plan->row_slot = rows; plan->row_pos = rows + T; plan->comb = rows + 2 * (size_t)T;
  plan->units = dm + o_units; plan->chunks = dm + o_chunks; plan->pre = dm + o_pre; plan->dec = dm + o_dec;
  plan->tab = reinterpret_cast<float2*>(base + L.tab);
  plan->part = reinterpret_cast<float*>(base + L.part);
  plan->joins = dm + o_joins; plan->n_joins = (int)h.joins.size() / KV8_JOIN_INTS;
  MetaChunk mc;
  for (size_t at = 0; at < meta.size(); at += META_CHUNK) {
    mc.count = (int)std::min<size_t>(META_CHUNK, meta.size() - at);
    std::memcpy(mc.values, meta.data() + at, mc.count * sizeof(int));
    hipError_t e = launch_meta_write(mc, dm + at, s);
    if (e != hipSuccess) return hip_fail(e, "plan upload");
  }
  Kv8RowsArgs ra{};
  ra.spans = dm + o_spans; ra.n_spans = (int)h.spans.size() / KV8_SPAN_INTS;
  ra.row_slot = rows; ra.row_pos = rows + T; ra.comb = rows + 2 * (size_t)T;
  ra.tab = reinterpret_cast<float2*>(base + L.tab); ra.pairs = c.rope_dim / 2;
  ra.mscale = c.rope_mscale == 0.f ? 1.f : c.rope_mscale;
  std::copy(kv->theta, kv->theta + KV8_MAX_PAIRS, ra.theta);
  hipError_t e = launch_kv8_rows(ra, s);
  return e == hipSuccess ? SARATHI_OK : hip_fail(e, "plan rows");
}

int run_append(const sarathi_kv8_plan* p, int layer, const void* qkv, size_t ld_qkv, const void* q_gain, const void* k_gain,
               void* q_out, size_t ld_q, hipStream_t s) {
  Kv8AppendArgs a{};
  a.qkv = qkv; a.ld_qkv = ld_qkv; a.q_out = q_out; a.ld_q = ld_q;
  if (p->cfg.qk_norm) { a.q_gain = q_gain; a.k_gain = k_gain; a.eps = p->cfg.qk_eps; }
  a.T = p->T; a.nh = p->cfg.n_heads; a.nkv = p->cfg.n_kv_heads;
  a.tab = p->tab; a.rot = p->cfg.rope_dim; a.interleaved = p->cfg.rope_layout == SARATHI_ROPE_INTERLEAVED;
  a.units = p->units; a.n_chunk = p->n_chunk_units; a.n_units = p->n_units;
  a.kv = layer_of(p, layer);
  const hipError_t e = launch_kv8_append(p->cfg.dtype, p->cfg.format, p->cfg.head_dim, p->cfg.block, a, s);
  return e == hipSuccess ? SARATHI_OK : hip_fail(e, "append");
}

int run_attention(const sarathi_kv8_plan* p, int layer, const void* q, size_t ld_q, void* out, size_t ld_out, hipStream_t s) {
  const sarathi_kv8_cfg& c = p->cfg;
  const float scale_log2 = (c.softmax_scale == 0.f ? 1.0f / std::sqrt((float)c.head_dim) : c.softmax_scale) * 1.4426950408889634f;
  hipError_t e;
  if (p->n_pre > 0) {
    Kv8ChunkArgs a{};
    a.q = q; a.ld_q = ld_q; a.out = out; a.ld_out = ld_out; a.chunks = p->chunks; a.work = p->pre; a.n_work = p->n_pre;
    a.nh = c.n_heads; a.nkv = c.n_kv_heads; a.groups = p->groups; a.part = p->part; a.scale_log2 = scale_log2;
    a.kv = layer_of(p, layer);
    e = launch_kv8_chunk(c.dtype, c.format, c.head_dim, a, s);
    if (e != hipSuccess) return hip_fail(e, "chunk attention");
  }
  if (p->n_dec > 0) {
    Kv8DecodeArgs a{};
    a.q = q; a.ld_q = ld_q; a.out = out; a.ld_out = ld_out; a.work = p->dec; a.n_work = p->n_dec;
    a.nh = c.n_heads; a.nkv = c.n_kv_heads; a.part = p->part; a.joins = p->joins; a.n_joins = p->n_joins; a.scale_log2 = scale_log2;
    a.kv = layer_of(p, layer);
    e = launch_kv8_decode(c.dtype, c.format, c.head_dim, a, s);
    if (e != hipSuccess) return hip_fail(e, "decode attention");
  }
  CombineArgs ca{};
  ca.part = p->part; ca.comb = p->comb; ca.row0 = p->comb_row0; ca.n_rows = p->comb_rows; ca.nh = c.n_heads; ca.hd = c.head_dim;
  ca.out = out; ca.ld_out = (int)ld_out;
  e = launch_attn_combine(c.dtype, ca, s);
  return e == hipSuccess ? SARATHI_OK : hip_fail(e, "attention combine");
}

// ---- decoder layer
struct LayerLayout {
  size_t a, qkv, o, hres, m, parts, ping0, ping1, plan, total;
};
LayerLayout layer_layout(const sarathi_model_cfg& c, const sarathi_kv8_cfg& k, int T, int n_chunks) {
  LayerLayout L{};
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = align256(off + bytes); return at; };
  const size_t es = esize(c.dtype), H = c.hidden, hd = k.head_dim;
  const size_t rows = T, nh = k.n_heads;
  L.a = take(rows * H * es);
  L.qkv = take(rows * (nh + 2 * (size_t)k.n_kv_heads) * hd * es);
  L.o = take(rows * nh * hd * es);
  L.hres = take(rows * H * 4);
  L.m = take(rows * c.ffn * es);
  L.parts = take((size_t)MAX_SPLIT * std::min(T, PARTS_ROWS) * H * 4);
  L.ping0 = take(rows * H * es);
  L.ping1 = take(rows * H * es);
  L.plan = take(plan_layout(k, T, n_chunks).total);
  L.total = off;
  return L;
}

// cfg on its own and against the cache's.
int check_layer_cfg(const sarathi_model_cfg* c, const sarathi_kv8_cfg* k) {
  int rc = check_cfg(c);
  if (!rc) rc = check_kv8_cfg(k);
  if (rc) return rc;
  if (c->n_heads != k->n_heads || c->head_dim != k->head_dim || c->n_layers != k->n_layers || c->dtype != k->dtype ||
      c->rope != (k->rope_dim > 0) || (c->rope && c->rope_base != k->rope_base))
    return fail(SARATHI_EINVAL, "cfg differs from the cfg of the 8-bit KV cache");
  return SARATHI_OK;
}

// One layer of a planned batch.  norm1_ready, next, next_norm1_done: as in the
// 16-bit layer (norm_1 folded into the previous layer's last reduction).
int layer_body(const sarathi_model_cfg* c, const LayerLayout& L, const sarathi_kv8_plan* plan,
               const sarathi_kv8_layer_weights* w, int layer, const void* x_in, void* x_out, char* ws, hipStream_t s,
               bool norm1_ready, const sarathi_kv8_layer_weights* next, bool* next_norm1_done) {
  const int T = plan->T, H = c->hidden, F = c->ffn, dt = c->dtype;
  const int QD = c->n_heads * c->head_dim, N = QD + 2 * plan->cfg.n_kv_heads * c->head_dim;
  const bool ln = c->norm == SARATHI_NORM_LAYER;
  float* hres = reinterpret_cast<float*>(ws + L.hres);
  float* parts = reinterpret_cast<float*>(ws + L.parts);
  const size_t parts_cap = (size_t)MAX_SPLIT * std::min(T, PARTS_ROWS) * H;
  hipError_t e;
  if (!norm1_ready) {
    e = launch_norm(dt, false, ln, x_in, w->base.norm1_g, w->base.norm1_b, ws + L.a, T, H, c->eps, s);
    if (e != hipSuccess) return hip_fail(e, "norm_1");
  }
  LinearArgs q{};
  q.kind = LIN_PLAIN; q.M = T; q.N = N; q.K = H; q.x = ws + L.a; q.w = w->base.w_qkv; q.out = ws + L.qkv;
  e = launch_linear(dt, q, s);
  if (e != hipSuccess) return hip_fail(e, "preproj");
  int rc = run_append(plan, layer, ws + L.qkv, N, w->q_gain, w->k_gain, ws + L.qkv, N, s);
  if (!rc) rc = run_attention(plan, layer, ws + L.qkv, N, ws + L.o, QD, s);
  if (rc) return rc;
  NormArgs n2{w->base.norm2_g, w->base.norm2_b, ws + L.a, c->eps, ln};
  bool norm2_done = false;
  LinearArgs po{};
  po.kind = LIN_RESID; po.M = T; po.N = H; po.K = QD; po.x = ws + L.o; po.w = w->base.w_o; po.resid = x_in; po.out = hres;
  po.parts = parts; po.parts_cap = parts_cap; po.norm = &n2; po.norm_done = &norm2_done;
  e = launch_linear(dt, po, s);
  if (e != hipSuccess) return hip_fail(e, "postproj");
  if (!norm2_done) {
    e = launch_norm(dt, true, ln, hres, w->base.norm2_g, w->base.norm2_b, ws + L.a, T, H, c->eps, s);
    if (e != hipSuccess) return hip_fail(e, "norm_2");
  }
  LinearArgs up{};
  up.kind = c->act == SARATHI_ACT_SWIGLU ? LIN_SWIGLU : LIN_GELU;
  up.M = T; up.N = F; up.K = H; up.x = ws + L.a; up.w = w->base.w_up; up.out = ws + L.m;
  e = launch_linear(dt, up, s);
  if (e != hipSuccess) return hip_fail(e, "ffn_ln1");
  LinearArgs dn{};
  dn.kind = LIN_RESID_F32IN; dn.M = T; dn.N = H; dn.K = F; dn.x = ws + L.m; dn.w = w->base.w_down; dn.resid = hres;
  dn.out = x_out; dn.parts = parts; dn.parts_cap = parts_cap;
  NormArgs n1{};
  if (next) {
    n1 = NormArgs{next->base.norm1_g, next->base.norm1_b, ws + L.a, c->eps, ln};
    dn.norm = &n1; dn.norm_done = next_norm1_done;
  }
  e = launch_linear(dt, dn, s);
  return e == hipSuccess ? SARATHI_OK : hip_fail(e, "ffn_ln2");
}

// Layers first .. first + n - 1 over one batch, each with its entry of w.
int run_layers(const sarathi_model_cfg* cfg, const sarathi_kv8_layer_weights* w, const sarathi_kv8* kv, int first, int n,
               const sarathi_mixed_batch* batch, const void* x_in, void* x_out, void* ws, size_t ws_bytes, hipStream_t s) {
  int rc = check_layer_cfg(cfg, &kv->cfg);
  if (rc) return rc;
  if (first < 0 || first + n > cfg->n_layers) return fail(SARATHI_EINVAL, "layer %d outside [0, %d)", first, cfg->n_layers);
  BatchDesc b;
  rc = from_mixed(batch, &b);
  if (!rc) rc = check_batch(b, kv->n_slots, kv->max_seq_len);
  if (rc) return rc;
  if (!w) return fail(SARATHI_EINVAL, "weights are NULL");
  for (int i = 0; i < n; ++i) {
    rc = check_weights(cfg, &w[i].base, first + i);
    if (rc) return rc;
    if (kv->cfg.qk_norm && (!w[i].q_gain || !w[i].k_gain || !aligned16(w[i].q_gain) || !aligned16(w[i].k_gain)))
      return fail(SARATHI_EINVAL, "layer %d: qk_norm needs 16-byte aligned q_gain and k_gain", first + i);
  }
  if (!x_in || !x_out || !ws) return fail(SARATHI_EINVAL, "x_in, x_out or the workspace is NULL");
  if (!aligned16(x_in) || !aligned16(x_out) || !aligned16(ws))
    return fail(SARATHI_EINVAL, "x_in, x_out and ws must be 16-byte aligned");
  const int T = b.rows();
  const LayerLayout L = layer_layout(*cfg, kv->cfg, T, (int)b.chunks.size());
  if (ws_bytes < L.total) return fail(SARATHI_ENOSPC, "workspace of %zu bytes < %zu needed", ws_bytes, L.total);
  const size_t xb = (size_t)T * cfg->hidden * esize(cfg->dtype);
  const Span xi{static_cast<const char*>(x_in), xb}, xo{static_cast<const char*>(x_out), xb}, wsp{static_cast<const char*>(ws), L.total};
  if (overlap(xi, xo) || overlap(xi, wsp) || overlap(xo, wsp))
    return fail(SARATHI_EINVAL, "x_in, x_out and the workspace must not overlap");
  char* base = static_cast<char*>(ws);
  sarathi_kv8_plan plan{};
  rc = plan_upload(kv, b, base + L.plan, L.total - L.plan, s, &plan);
  if (rc) return rc;
  char* ping[2] = {base + L.ping0, base + L.ping1};
  bool ready = false;
  for (int i = 0; i < n; ++i) {
    const void* in = i == 0 ? x_in : ping[i & 1];
    void* out = i == n - 1 ? x_out : ping[(i + 1) & 1];
    bool next_ready = false;
    rc = layer_body(cfg, L, &plan, w + i, first + i, in, out, base, s, ready, i + 1 < n ? w + i + 1 : nullptr, &next_ready);
    if (rc) return rc;
    ready = next_ready;
  }
  return SARATHI_OK;
}

// No C++ exception leaves a C entry (the host lists are the only allocations).
template <typename F>
int guarded(F&& f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail(SARATHI_ENOSPC, "out of host memory");
  } catch (...) {
    return fail(SARATHI_EINVAL, "internal: unexpected exception");
  }
}

}  // namespace

extern "C" {

size_t sarathi_kv8_bytes(const sarathi_kv8_cfg* cfg, int n_slots, int max_seq_len) {
  if (check_kv8_cfg(cfg) != SARATHI_OK) return 0;
  if (n_slots < 1 || n_slots > MAX_SLOTS || max_seq_len < 1 || max_seq_len > MAX_SEQ) {
    fail(SARATHI_EINVAL, "n_slots %d or max_seq_len %d out of range", n_slots, max_seq_len);
    return 0;
  }
  const sarathi_kv8_layout L = layout_of(*cfg, n_slots, max_seq_len);   // a layer: below 2^61 bytes
  if (L.layer > (size_t(1) << 62) / (size_t)cfg->n_layers) {
    fail(SARATHI_EUNSUPPORTED, "%d layers of %zu bytes", cfg->n_layers, L.layer);
    return 0;
  }
  return L.scale_offset + L.scale_layer * cfg->n_layers * sizeof(float);
}

int sarathi_kv8_alloc(const sarathi_kv8_cfg* cfg, int n_slots, int max_seq_len, void* dev_mem, size_t dev_bytes,
                      sarathi_kv8** out) {
  const int rc = check_kv8_cfg(cfg);
  if (rc) return rc;
  if (!out) return fail(SARATHI_EINVAL, "out is NULL");
  *out = nullptr;
  if (!dev_mem) return fail(SARATHI_EINVAL, "dev_mem is NULL");
  if (!aligned16(dev_mem)) return fail(SARATHI_EINVAL, "dev_mem must be 16-byte aligned");
  if (n_slots < 1 || n_slots > MAX_SLOTS) return fail(SARATHI_EINVAL, "n_slots %d out of range", n_slots);
  if (max_seq_len < 1 || max_seq_len > MAX_SEQ) return fail(SARATHI_EINVAL, "max_seq_len %d out of range", max_seq_len);
  const size_t need = sarathi_kv8_bytes(cfg, n_slots, max_seq_len);
  if (need == 0) return SARATHI_EUNSUPPORTED;   // more bytes than can be addressed
  if (dev_bytes < need) return fail(SARATHI_ENOSPC, "KV memory of %zu bytes < %zu needed", dev_bytes, need);
  sarathi_kv8* kv = new (std::nothrow) sarathi_kv8{};
  if (!kv) return fail(SARATHI_ENOSPC, "out of host memory");
  kv->cfg = *cfg;
  kv->n_slots = n_slots;
  kv->max_seq_len = max_seq_len;
  kv->mem = static_cast<char*>(dev_mem);
  kv->st = layout_of(*cfg, n_slots, max_seq_len);
  rope_thetas(*cfg, kv->theta);
  *out = kv;
  return SARATHI_OK;
}

void sarathi_kv8_free(sarathi_kv8* kv) { delete kv; }

int sarathi_kv8_get_layout(const sarathi_kv8* kv, sarathi_kv8_layout* out) {
  if (!kv || !out) return fail(SARATHI_EINVAL, "NULL argument");
  *out = kv->st;
  return SARATHI_OK;
}

size_t sarathi_kv8_plan_bytes(const sarathi_kv8_cfg* cfg, int max_tokens, int max_chunks, int max_seq_len) {
  if (check_kv8_cfg(cfg) != SARATHI_OK || max_tokens < 1 || max_chunks < 0 || max_seq_len < 1) return 0;
  return plan_layout(*cfg, max_tokens, max_chunks).total;
}

int sarathi_kv8_plan_create(const sarathi_kv8* kv, const sarathi_mixed_batch* batch, void* ws, size_t ws_bytes,
                            void* hip_stream, sarathi_kv8_plan** out) {
  if (!out) return fail(SARATHI_EINVAL, "out is NULL");
  *out = nullptr;
  if (!kv) return fail(SARATHI_EINVAL, "kv is NULL");
  return guarded([&]() -> int {
    BatchDesc b;
    int rc = from_mixed(batch, &b);
    if (!rc) rc = check_batch(b, kv->n_slots, kv->max_seq_len);
    if (rc) return rc;
    sarathi_kv8_plan plan{};
    rc = plan_upload(kv, b, ws, ws_bytes, static_cast<hipStream_t>(hip_stream), &plan);
    if (rc) return rc;
    *out = new sarathi_kv8_plan(plan);
    return SARATHI_OK;
  });
}

void sarathi_kv8_plan_free(sarathi_kv8_plan* plan) { delete plan; }

int sarathi_kv8_append(const sarathi_kv8_plan* plan, int layer, const void* qkv, size_t ld_qkv, const void* q_gain,
                       const void* k_gain, void* q_out, size_t ld_q, void* hip_stream) {
  int rc = check_plan(plan, layer);
  if (rc) return rc;
  const sarathi_kv8_cfg& c = plan->cfg;
  const size_t es = esize(c.dtype), qc = (size_t)c.n_heads * c.head_dim;
  const size_t cols = qc + 2 * (size_t)c.n_kv_heads * c.head_dim;
  if ((rc = check_rows("qkv", qkv, ld_qkv, cols, es)) || (rc = check_rows("q_out", q_out, ld_q, qc, es))) return rc;
  if (c.qk_norm && (!q_gain || !k_gain)) return fail(SARATHI_EINVAL, "qk_norm needs q_gain and k_gain");
  if (c.qk_norm && (!aligned16(q_gain) || !aligned16(k_gain))) return fail(SARATHI_EINVAL, "gains must be 16-byte aligned");
  if (!(q_out == qkv && ld_q == ld_qkv) &&
      overlap(rows_span(qkv, plan->T, ld_qkv, cols, es), rows_span(q_out, plan->T, ld_q, qc, es)))
    return fail(SARATHI_EINVAL, "q_out overlaps qkv (other than in place)");
  return run_append(plan, layer, qkv, ld_qkv, q_gain, k_gain, q_out, ld_q, static_cast<hipStream_t>(hip_stream));
}

int sarathi_kv8_attention(const sarathi_kv8_plan* plan, int layer, const void* q, size_t ld_q, void* out, size_t ld_out,
                          void* hip_stream) {
  int rc = check_plan(plan, layer);
  if (rc) return rc;
  const sarathi_kv8_cfg& c = plan->cfg;
  const size_t es = esize(c.dtype), qc = (size_t)c.n_heads * c.head_dim;
  if ((rc = check_rows("q", q, ld_q, qc, es)) || (rc = check_rows("out", out, ld_out, qc, es))) return rc;
  if (ld_out > (1u << 30)) return fail(SARATHI_EINVAL, "out: row stride %zu too large", ld_out);
  if (overlap(rows_span(q, plan->T, ld_q, qc, es), rows_span(out, plan->T, ld_out, qc, es)))
    return fail(SARATHI_EINVAL, "q and out must not overlap");
  return run_attention(plan, layer, q, ld_q, out, ld_out, static_cast<hipStream_t>(hip_stream));
}

int sarathi_kv8_read(const sarathi_kv8_plan* plan, int layer, int out_dtype, void* k_out, size_t ld_k, void* v_out,
                     size_t ld_v, void* hip_stream) {
  int rc = check_plan(plan, layer);
  if (rc) return rc;
  if (out_dtype != SARATHI_F32 && out_dtype != SARATHI_BF16) return fail(SARATHI_EUNSUPPORTED, "out_dtype %d", out_dtype);
  const sarathi_kv8_cfg& c = plan->cfg;
  const size_t es = esize(out_dtype), cols = (size_t)c.n_kv_heads * c.head_dim;
  if (!k_out && !v_out) return fail(SARATHI_EINVAL, "k_out and v_out are NULL");
  if (k_out && (rc = check_rows("k_out", k_out, ld_k, cols, es))) return rc;
  if (v_out && (rc = check_rows("v_out", v_out, ld_v, cols, es))) return rc;
  if (k_out && v_out && overlap(rows_span(k_out, plan->T, ld_k, cols, es), rows_span(v_out, plan->T, ld_v, cols, es)))
    return fail(SARATHI_EINVAL, "k_out and v_out must not overlap");
  Kv8ReadArgs a{};
  a.row_slot = plan->row_slot; a.row_pos = plan->row_pos; a.k_out = k_out; a.ld_k = ld_k; a.v_out = v_out; a.ld_v = ld_v;
  a.T = plan->T; a.nkv = c.n_kv_heads; a.hd = c.head_dim; a.kv = layer_of(plan, layer);
  const hipError_t e = launch_kv8_read(out_dtype, c.format, a, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? SARATHI_OK : hip_fail(e, "read");
}

size_t sarathi_kv8_workspace_bytes(const sarathi_model_cfg* cfg, const sarathi_kv8_cfg* kv_cfg, int max_tokens,
                                   int max_chunks, int max_seq_len) {
  if (check_layer_cfg(cfg, kv_cfg) != SARATHI_OK || max_tokens < 1 || max_chunks < 0 || max_seq_len < 1) return 0;
  return layer_layout(*cfg, *kv_cfg, max_tokens, max_chunks).total;
}

int sarathi_kv8_workspace_layout(const sarathi_model_cfg* cfg, const sarathi_kv8_cfg* kv_cfg, int n_tokens, int n_chunks,
                                 int max_seq_len, sarathi_ws_layout* out) {
  const int rc = check_layer_cfg(cfg, kv_cfg);
  if (rc) return rc;
  if (!out) return fail(SARATHI_EINVAL, "out is NULL");
  if (n_tokens < 1 || n_chunks < 0 || max_seq_len < 1) return fail(SARATHI_EINVAL, "bad sizes");
  const LayerLayout L = layer_layout(*cfg, *kv_cfg, n_tokens, n_chunks);
  out->a = L.a; out->qkv = L.qkv; out->o = L.o; out->hres = L.hres; out->m = L.m;
  out->ping[0] = L.ping0; out->ping[1] = L.ping1; out->total = L.total;
  return SARATHI_OK;
}

int sarathi_kv8_layer_forward(const sarathi_model_cfg* cfg, const sarathi_kv8_layer_weights* w, const sarathi_kv8* kv,
                              int layer, const sarathi_mixed_batch* batch, const void* x_in, void* x_out, void* ws,
                              size_t ws_bytes, void* hip_stream) {
  if (!kv) return fail(SARATHI_EINVAL, "kv is NULL");
  return guarded([&] {
    return run_layers(cfg, w, kv, layer, 1, batch, x_in, x_out, ws, ws_bytes, static_cast<hipStream_t>(hip_stream));
  });
}

int sarathi_kv8_model_step(const sarathi_model_cfg* cfg, const sarathi_kv8_layer_weights* w, const sarathi_kv8* kv,
                           const sarathi_mixed_batch* batch, const void* x_in, void* x_out, void* ws, size_t ws_bytes,
                           void* hip_stream) {
  if (!kv) return fail(SARATHI_EINVAL, "kv is NULL");
  return guarded([&] {
    return run_layers(cfg, w, kv, 0, kv->cfg.n_layers, batch, x_in, x_out, ws, ws_bytes, static_cast<hipStream_t>(hip_stream));
  });
}

}  // extern "C"
