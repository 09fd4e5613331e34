// Attention of prompt chunks over the 8-bit KV cache.
//
// Block = one key/value head, KV8_QB packed query rows (the rows of the chunk
// times the query heads that share the key/value head; four waves of 32 to a
// group) and a range of 64-key tiles.  A tile's codes are read once per group,
// converted to bf16 (exact) on the way into LDS, and multiplied there by its
// four waves:
//   S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_32x32x16_bf16, a lane (ql =
//   lane % 32, g = lane / 32) holding the scores of packed row ql for keys
//   8 (v / 4) + 4 g + v % 4 of each 32-key half; V^T comes from transposed LDS
//   reads.  A scale is constant over 16 keys: the key scale joins the softmax
//   scale in the exponent; of bf16 rows the value scale enters there as its
//   logarithm (the row sum divides it out again), so neither costs a
//   multiplication per score.
// Probabilities of bf16 rows are rounded to bf16 (with q and the codes exact, all
// that the products lose): outputs are off by 2.2e-3 of their magnitude, of which
// their own rounding is 1.7e-3.
// 512 rows over a prefix of 2048 (52 heads): 51 us, 0.62 PFLOP/s; a 4096-token
// prompt (32 / 8 heads) with three decodes: 181 us, 0.76 PFLOP/s.  The matrix
// cores are busy 21 and 32 % of the cycles: it is bound by the latency of a tile's
// chain (LDS reads, products, maximum, exponentials, products, barrier) and the
// vector instructions beside it (10 to 11 per matrix instruction).  Fragments are
// therefore read a step ahead of their products and the next tile is converted
// and stored beside the second products; either alone gained 0 to 1 %, both
// together 6 % on the first case and 2 % on the second.  Tried and no faster: the
// next tile's products under this one's exponentials, 32-key tiles with three
// waves per SIMD, 64 rows per wave (the accumulators then move between register
// files), and operands straight from global memory (440 us for the prompt).
#include "kv8_device.h"

namespace sarathi {

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

// 16 codes to 16 bf16.
template <bool INT8>
__device__ __forceinline__ void widen16(const uint4& w, u32x4& lo, u32x4& hi) {
  lo = __builtin_bit_cast(u32x4, codes8_bf16<INT8>(w.x, w.y));
  hi = __builtin_bit_cast(u32x4, codes8_bf16<INT8>(w.z, w.w));
}

// Swizzle of a tile row's 16-byte chunks: a bijection of the row mod 16 that
// moves aligned groups of four together (head_dim 128), so that both the row
// reads of K and the transposed reads of V fall on distinct LDS banks.
template <int D>
__device__ __forceinline__ int swz(int c, int r) {
  if (D == 128) return c ^ (((r & 3) << 2) | ((r >> 2) & 3));
  return c ^ (r & 7);
}

// Maximum that propagates NaN (fmaxf would first quieten every score).
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float lanes_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max_nan(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float lanes_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
__device__ __forceinline__ uint2 lds_tr16(const char* p) {
  const v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)p);
  return __builtin_bit_cast(uint2, v);
}

// NG: groups of four waves that take the item's tiles in turn, each with LDS
// stages of its own, and are merged at the end.
template <typename T, int D, bool INT8, int NG>
__global__ __launch_bounds__(256 * NG, sizeof(T) == 2 ? 2 : 1) void kv8_attn_chunk_kernel(Kv8ChunkArgs a) {
  constexpr int NT = sizeof(T) == 2 ? 1 : 3;
  constexpr int KT = KV8_KT, QB = KV8_QB;
  constexpr int DCH = D / 8;             // 16-byte chunks per bf16 tile row
  constexpr int TILE = KT * DCH;         // chunks per tile
  constexpr int LPR = D / 16;            // lanes that read a key row (16 codes each)
  constexpr int NI = KT * LPR / 256;     // 16-byte loads per thread and tile (K or V)
  extern __shared__ u32x4 lds[];         // [group][stage][K, V][TILE]; then the merge

  // blocks go to the eight XCDs in turn: each takes whole heads, whose keys and
  // values its L2 then serves to all of their query blocks
  const int per = gridDim.x / 8, bt = (int)(blockIdx.x % 8) * per + (int)(blockIdx.x / 8);
  if (bt >= a.n_work * a.nkv) return;
  const int item = bt % a.n_work, kvh = bt / a.n_work;
  const int* wk = a.work + 4 * item;
  const int* ch = a.chunks + 4 * wk[0];
  const int slot = ch[0], offset = ch[1], C = ch[2], row0 = ch[3];
  const int r0 = wk[1], part = wk[2];
  const int group = a.nh / a.nkv;
  const int nrows = min(QB / group, C - r0);       // the block's chunk rows
  const int tid = threadIdx.x & 255, lane = tid & 63, wave = tid >> 6;   // within the group
  const int grp = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
  const int g = lane >> 5, ql = lane & 31;
  u32x4* ring = lds + grp * 4 * TILE;

  const uint8_t* kbase = a.kv.codes + slot * a.kv.slot + kvh * a.kv.head;
  const uint8_t* vbase = kbase + a.kv.kv;
  const float* ksc = a.kv.scales + slot * a.kv.s_slot + kvh * a.kv.s_head;
  const float* vsc = ksc + a.kv.s_kv;

  const int kbeg = (wk[3] >> 16) * KT;
  const int kend = min(offset + r0 + nrows, (wk[3] & 0xffff) * KT);
  const int n_tiles = (kend - kbeg + KT - 1) / KT;
  const int n_iter = (n_tiles + NG - 1) / NG;        // the group's tile of iteration i: NG i + grp

  // the lane's packed row: chunk row r0 + rr, head
  const int pr = wave * 32 + ql;
  const int rr = min(pr / group, nrows - 1), head = kvh * group + pr % group;
  const bool real = pr < nrows * group;
  const int qpos = offset + r0 + rr;
  const int last_key = offset + r0 + min((wave * 32 + 31) / group, nrows - 1);
  const bool idle = wave * 32 >= nrows * group;
  bf16x8_t qf[D / 16][NT];
  {
    const T* q = reinterpret_cast<const T*>(a.q) + (size_t)(row0 + r0 + rr) * a.ld_q + (size_t)head * D;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      const T* p = q + ks * 16 + 8 * g;
      if constexpr (NT == 1) {
        qf[ks][0] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(p));
      } else {
        float x[8];
        Vec16<float>::unpack(*reinterpret_cast<const uint4*>(p), x);
        Vec16<float>::unpack(*reinterpret_cast<const uint4*>(p + 4), x + 4);
        split8<NT>(x, qf[ks]);
      }
    }
    // the fragments are here before the loop: waited for inside it, they would
    // take the prefetched tile with them (loads return in order)
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
      for (int n = 0; n < NT; ++n) asm volatile("" : "+v"(qf[ks][n]));
  }

  float m_run = -INFINITY, l_run = 0.f;
  floatx16 o_acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) o_acc[db][v] = 0.f;

  // Tile staging: a thread takes NI pieces of 16 codes of K and of V; positions
  // past the item's keys re-read its last one.
  uint4 kr[NI], vr[NI];
  float ks_next[4], vs_next[4];          // the fetched tile's scales of its four 16-key groups
  const int sr = tid / LPR, sc = tid % LPR;
  auto fetch = [&](int it) {
    const int k0 = kbeg + (NG * it + grp) * KT;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = min(k0 + 16 * i, kend - 1) >> a.kv.log2_block;
      ks_next[i] = ksc[b];
      vs_next[i] = vsc[b];
    }
    const uint8_t* kp = kbase + (size_t)k0 * D;
    const uint8_t* vp = vbase + (size_t)k0 * D;
    const int lim = (kend - 1 - k0) * D;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int off = min((sr + i * (256 / LPR)) * D, lim) + 16 * sc;
      kr[i] = *reinterpret_cast<const uint4*>(kp + off);
      vr[i] = *reinterpret_cast<const uint4*>(vp + off);
    }
  };
  auto stage_piece = [&](u32x4* tile, const uint4& x, int i) {
    const int r = sr + i * (256 / LPR);
    u32x4 lo, hi;
    widen16<INT8>(x, lo, hi);
    tile[r * DCH + swz<D>(2 * sc, r)] = lo;
    tile[r * DCH + swz<D>(2 * sc + 1, r)] = hi;
  };
  // piece j of the fetched tile (its NI pieces of K, then those of V)
  auto stage = [&](int buf, int j) {
    if (j < NI) stage_piece(ring + 2 * buf * TILE, kr[j % NI], j);
    else if (j < 2 * NI) stage_piece(ring + (2 * buf + 1) * TILE, vr[j % NI], j - NI);
  };

  // transposed-read offsets of V^T fragments (rows 4 g + e and + 8 of a 16-key step)
  const int G = lane >> 4, li = lane & 15;
  const int tr_e = li >> 2, tr_q = li & 3;
  const int tr_c16 = 2 * (G & 1) + (tr_q >> 1), tr_half = (tr_q & 1) * 8;
  int voff[2][D / 32], koff[D / 16];
#pragma unroll
  for (int hh = 0; hh < 2; ++hh)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const int r = 4 * g + tr_e + 8 * hh;
      voff[hh][db] = (r * DCH + swz<D>(4 * db + tr_c16, r)) * 16 + tr_half;
    }
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) koff[ks] = ql * DCH + swz<D>(2 * ks + g, ql);

  float ks4[4], vs4[4];
  float unit = KV8_UNIT;                 // of the row's sums (kv8_device.h)
  auto compute = [&](int it, int buf) {
    const int k0 = kbeg + (NG * it + grp) * KT;
    if (k0 > last_key || k0 >= kend || idle) {
#pragma unroll
      for (int j = 0; j < 2 * NI; ++j) stage(buf ^ 1, j);
      return;
    }
    // Fragments are read a step ahead of their products (the scheduling barriers
    // keep them there: left alone, the compiler saves registers by waiting for
    // every read just before its product, 16 LDS latencies in a row).
    floatx16 s[2];
    bf16x8_t kf[2][4];
    auto read_k = [&](bf16x8_t* f, int i) {                 // step i: 16-dim slices 2 i, 2 i + 1 of both halves
#pragma unroll
      for (int e = 0; e < 4; ++e)
        f[e] = __builtin_bit_cast(bf16x8_t, ring[2 * buf * TILE + (e & 1) * 32 * DCH + koff[2 * i + (e >> 1)]]);
      __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int v = 0; v < 16; ++v) s[kb][v] = 0.f;
    read_k(kf[0], 0);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      if (i + 1 < D / 32) read_k(kf[(i + 1) & 1], i + 1);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          s[e & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i & 1][e], qf[2 * i + (e >> 1)][n], s[e & 1], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    // V^T of a 16-key step
    const char* vt = reinterpret_cast<const char*>(ring + (2 * buf + 1) * TILE);
    bf16x8_t vf[2][D / 32];
    auto read_v = [&](bf16x8_t* f, int i) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const uint2 x = lds_tr16(vt + voff[0][db] + i * 16 * DCH * 16), y = lds_tr16(vt + voff[1][db] + i * 16 * DCH * 16);
        f[db] = __builtin_bit_cast(bf16x8_t, u32x4{x.x, x.y, y.x, y.y});
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    const bool full = k0 + KT <= kend && k0 + KT - 1 <= offset + r0 + wave * 32 / group;
    if (!full) {
      const int lim = min(qpos, kend - 1) - k0;
      // scales of keys that the row does not see stay out of its unit and its sums
#pragma unroll
      for (int i = 0; i < 4; ++i) vs4[i] = 16 * i <= lim ? vs4[i] : 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (kb * 32 + 8 * (v >> 2) + 4 * g + (v & 3) > lim) s[kb][v] = -INFINITY;
    }
    const bool change = kv8_unit_change(fmaxf(fmaxf(vs4[0], vs4[1]), fmaxf(vs4[2], vs4[3])), unit);
    // a zero scale belongs to zero codes, so 1 does as well
#pragma unroll
    for (int i = 0; i < 4; ++i) vs4[i] = vs4[i] > 0.f ? fmaxf(vs4[i], kv8_unit_floor(unit)) : 1.f;
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float t = s[i >> 1][8 * (i & 1)];
#pragma unroll
      for (int v = 1; v < 8; ++v) t = max_nan(t, s[i >> 1][8 * (i & 1) + v]);
      mx = max_nan(mx, t * ks4[i]);
    }
    mx = lanes_max(mx);
    if (__ballot(change || mx > m_run + 8.0f)) {
      const float m_new = fmaxf(m_run, mx);
      const float corr = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      const float corr_o = change ? corr * KV8_UNIT_STEP : corr;
#pragma unroll
      for (int db = 0; db < D / 32; ++db) o_acc[db] *= corr_o;
      l_run *= NT == 1 ? corr_o : corr;
      m_run = m_new;
    }
    const float m_use = (m_run == -INFINITY ? 0.f : m_run) - (NT == 1 ? unit : 0.f);
    bf16x8_t pf[2][NT];
    auto probs = [&](bf16x8_t* f, int i) {
      float p[8], sum = 0.f;
      if constexpr (NT == 1) {
        const float add = __builtin_amdgcn_logf(vs4[i]) - m_use;   // log2
#pragma unroll
        for (int v = 0; v < 8; ++v) p[v] = __builtin_amdgcn_exp2f(fmaf(s[i >> 1][8 * (i & 1) + v], ks4[i], add));
        split8<NT>(p, f);
        // the row sum takes the rounded probabilities that multiply V
        const u32x4 w = __builtin_bit_cast(u32x4, f[0]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t pair = w[e];
          sum = sum_bf16(pair, sum);
        }
        l_run = fmaf(sum, __builtin_amdgcn_rcpf(vs4[i]), l_run);
      } else {
        // the logarithm's roundings (2^-24 of its magnitude) would cost fp32 rows
        // bits: the value scale multiplies, and the row sum does without it
#pragma unroll
        for (int v = 0; v < 8; ++v) {
          p[v] = __builtin_amdgcn_exp2f(fmaf(s[i >> 1][8 * (i & 1) + v], ks4[i], -m_use));
          sum += p[v];
          p[v] *= vs4[i] * kv8_unit_pow2(unit);
        }
        split8<NT>(p, f);
        l_run += sum;
      }
    };
    read_v(vf[0], 0);
    probs(pf[0], 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i < 3) read_v(vf[(i + 1) & 1], i + 1);
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          o_acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i & 1][db], pf[i & 1][n], o_acc[db], 0, 0, 0);
      stage(buf ^ 1, i);                                        // the next tile's codes, beside the products
      if (i < 3) probs(pf[(i + 1) & 1], i + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  auto step = [&](int it, int buf) {
    // a zero key scale belongs to zero codes, so 1 does as well
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ks4[i] = (ks_next[i] > 0.f ? ks_next[i] : 1.f) * a.scale_log2;
      vs4[i] = vs_next[i];                 // as the row sees it: below
    }
    if (it + 1 < n_iter) fetch(it + 1);
    compute(it, buf);                      // (the last tile stages itself again, unread)
    __syncthreads();
  };
  fetch(0);
#pragma unroll
  for (int j = 0; j < 2 * NI; ++j) stage(0, j);
  __syncthreads();
  for (int it = 0; it < n_iter; it += 2) {
    step(it, 0);
    if (it + 1 < n_iter) step(it + 1, 1);
  }
  l_run = lanes_sum(l_run);
  {
    if constexpr (NT > 1) l_run *= kv8_unit_pow2(unit);
    const float f = kv8_unit_out(unit, m_run);
#pragma unroll
    for (int db = 0; db < D / 32; ++db) o_acc[db] *= f;
    l_run *= f;
  }
  if constexpr (NG == 2) {
    // the second group's result through LDS (the tiles are done with) to the first
    float* red_m = reinterpret_cast<float*>(lds);      // [QB] m, [QB] l, [QB][D + 4] o
    float* red_l = red_m + QB;
    float* red_o = red_l + QB + pr * (D + 4) + 4 * g;
    if (grp == 1) {
      if (g == 0) {
        red_m[pr] = m_run;
        red_l[pr] = l_run;
      }
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int v4 = 0; v4 < 4; ++v4)
          *reinterpret_cast<floatx4*>(red_o + db * 32 + 8 * v4) =
              floatx4{o_acc[db][4 * v4], o_acc[db][4 * v4 + 1], o_acc[db][4 * v4 + 2], o_acc[db][4 * v4 + 3]};
    }
    __syncthreads();
    if (grp == 1) return;
    const float m1 = red_m[pr], M = fmaxf(m_run, m1), Ms = M == -INFINITY ? 0.f : M;
    const float f0 = __builtin_amdgcn_exp2f(m_run - Ms), f1 = __builtin_amdgcn_exp2f(m1 - Ms);
    l_run = l_run * f0 + red_l[pr] * f1;
    m_run = M;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        const floatx4 x = *reinterpret_cast<const floatx4*>(red_o + db * 32 + 8 * v4);
#pragma unroll
        for (int i = 0; i < 4; ++i) o_acc[db][4 * v4 + i] = o_acc[db][4 * v4 + i] * f0 + x[i] * f1;
      }
  }
  if (!real) return;
  if (part < 0) {
    const float inv = 1.0f / l_run;
    T* out = reinterpret_cast<T*>(a.out) + (size_t)(row0 + r0 + rr) * a.ld_out + (size_t)head * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v4 = 0; v4 < 4; ++v4) {
        const int d = db * 32 + 8 * v4 + 4 * g;
        const floatx4 x = floatx4{o_acc[db][4 * v4], o_acc[db][4 * v4 + 1], o_acc[db][4 * v4 + 2], o_acc[db][4 * v4 + 3]} * inv;
        if constexpr (NT == 1) *reinterpret_cast<uint2*>(out + d) = make_uint2(pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3]));
        else *reinterpret_cast<floatx4*>(out + d) = x;
      }
    return;
  }
  float* dst = a.part + ((size_t)(part + rr) * a.nh + head) * (D + PART_O);
  if (g == 0) {
    dst[0] = m_run;
    dst[1] = l_run;
  }
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int v4 = 0; v4 < 4; ++v4)
      *reinterpret_cast<floatx4*>(dst + PART_O + db * 32 + 8 * v4 + 4 * g) =
          floatx4{o_acc[db][4 * v4], o_acc[db][4 * v4 + 1], o_acc[db][4 * v4 + 2], o_acc[db][4 * v4 + 3]};
}

template <typename T, int D, bool INT8, int NG>
static hipError_t run_chunk(const Kv8ChunkArgs& a, hipStream_t s) {
  constexpr int TILES = NG * 4 * KV8_KT * D * 2, MERGE = KV8_QB * (2 + D + 4) * 4;   // 128 KB at most
  constexpr int LDS = NG == 2 && MERGE > TILES ? MERGE : TILES;
  static std::atomic<uint64_t> done{0};
  const hipError_t e = ensure_dynamic_lds((const void*)kv8_attn_chunk_kernel<T, D, INT8, NG>, LDS, done);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)(((size_t)a.n_work * a.nkv + 7) / 8 * 8));
  hipLaunchKernelGGL((kv8_attn_chunk_kernel<T, D, INT8, NG>), grid, dim3(256 * NG), LDS, s, a);
  return hipGetLastError();
}

template <typename T, int D>
static hipError_t run_chunk_groups(int format, const Kv8ChunkArgs& a, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (a.groups == 2) return format == 0 ? run_chunk<T, D, true, 2>(a, s) : run_chunk<T, D, false, 2>(a, s);
  }
  return format == 0 ? run_chunk<T, D, true, 1>(a, s) : run_chunk<T, D, false, 1>(a, s);
}

hipError_t launch_kv8_chunk(int dtype, int format, int hd, const Kv8ChunkArgs& a, hipStream_t s) {
  if (a.n_work <= 0) return hipSuccess;
  if (dtype == 0) return hd == 128 ? run_chunk_groups<float, 128>(format, a, s) : run_chunk_groups<float, 64>(format, a, s);
  return hd == 128 ? run_chunk_groups<bf16, 128>(format, a, s) : run_chunk_groups<bf16, 64>(format, a, s);
}

}  // namespace sarathi
