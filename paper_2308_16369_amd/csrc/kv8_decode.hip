// Attention of the decodes of a batch over the 8-bit KV cache.
//
// Work item = (decode, a range of its keys), one block per item, key/value
// head and group of 16 query heads; four waves take steps of 32 keys in turn.
// A wave multiplies on v_mfma_f32_16x16x32_f16 (bf16 rows) or _bf16 (fp32 rows, in
// three terms) straight from registers, the codes converted exactly:
//   S^T = K Q^T: A = 16 keys x 32 dims, B = 32 dims x 16 query heads.  A lane
//     (c = lane % 16, gq = lane / 16) loads 16 bytes of key c at dims
//     64 i + 16 gq; the product's order over dims is the same permutation on
//     both sides.  It ends up with the scores of head c for keys 4 gq .. + 3.
//   O^T += V^T P^T: B = those probabilities as they are (32 keys: the lane's
//     four of either 16-key tile), A = V^T: the lane's eight keys at dim
//     (D / 16) c + db, which it loads as D / 16 neighbouring bytes of each of
//     its keys' rows.  It accumulates dims (D / 4) gq .. of head c.
// Query heads that share the key/value head fill the 16 columns; the unused
// ones cost matrix-core time only, which this kernel has to spare (it is bound
// by reading the cache).  A scale is constant over 16 keys: the key scale
// multiplies the scores with the softmax scale, the value scale the
// probabilities.
//
// 48 decodes of 512 to 2048 tokens (40 heads, int8): 104 us, 6.4 TB/s of codes
// (a plain non-temporal read: 7.1).  Two contexts of 98 and 131 thousand tokens
// (64 / 8 heads, e4m3): 67 us and 4.6 of the join.  With int8 codes converted to
// bf16, and rows in batch order, the first took 124 us: the conversions then
// outlasted the loads.  Nothing is staged in LDS, as no code is used by two waves.
#include "kv8_device.h"

namespace sarathi {

// Max / sum over the four 16-lane groups of the wave (the lanes of one head):
// v_permlane16/32_swap hand each lane its own and its partner's value.
__device__ __forceinline__ float groups_max(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float groups_sum(float v) {
  auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

template <typename T>
__device__ __forceinline__ void store_out4(const Kv8DecodeArgs& a, int row, int head, int D, int d, floatx4 x) {
  T* out = reinterpret_cast<T*>(a.out) + (size_t)row * a.ld_out + (size_t)head * D + d;
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(out) = make_uint2(pk_bf16(x[0], x[1]), pk_bf16(x[2], x[3]));
  else *reinterpret_cast<floatx4*>(out) = x;
}

// F16: bf16 rows (kv8_device.h).  OFFSET: of them, int8 codes, which enter as code + 128.
template <typename T, int D, bool INT8>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 3 : 2) void kv8_attn_rows_kernel(Kv8DecodeArgs a) {
  constexpr int NT = sizeof(T) == 2 ? 1 : 3;
  constexpr bool F16 = NT == 1, OFFSET = F16 && INT8;
  constexpr int KI = D / 64;             // 16-byte K loads per key row and lane
  constexpr int DB = D / 16;             // V bytes per key row and lane; tiles of O
  constexpr int VW = DB / 4;             // dwords of them
  constexpr int NW = 4;
  extern __shared__ float red[];         // [NW][16] m, [NW][16] l, [NW][heads][D] o

  const int group = a.nh / a.nkv, hblocks = (group + 15) / 16, per = a.nkv * hblocks;
  const int item = blockIdx.x / per, hx = blockIdx.x % per;
  const int kvh = hx / hblocks, hb = hx % hblocks;
  const int nheads = min(16, group - 16 * hb);
  const int head0 = kvh * group + 16 * hb;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int c = lane & 15, gq = lane >> 4;
  const int* wk = a.work + KV8_DEC_INTS * item;
  const int row = wk[0], slot = wk[1], kb = wk[2], ke = wk[3], part = wk[4];

  const uint8_t* kbase = a.kv.codes + slot * a.kv.slot + kvh * a.kv.head;
  const uint8_t* vbase = kbase + a.kv.kv;
  const float* ksc = a.kv.scales + slot * a.kv.s_slot + kvh * a.kv.s_head;
  const float* vsc = ksc + a.kv.s_kv;

  // scores: s = raw * (key scale * c_mul) + key scale * c_add
  float c_mul = a.scale_log2, c_add = 0.f;
  u32x4 qf[2 * KI][NT];
  {
    const T* q = reinterpret_cast<const T*>(a.q) + (size_t)row * a.ld_q + (size_t)(head0 + min(c, nheads - 1)) * D + 16 * gq;
    if constexpr (F16) {
      float x[2 * KI][8], top = 0.f, sum = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * KI; ++i) {
        Vec16<bf16>::unpack(*reinterpret_cast<const uint4*>(q + 64 * (i / 2) + 8 * (i & 1)), x[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[i][e]));
      }
      // a power of two that brings the row's largest magnitude to 2^14 .. 2^15
      const int ex = f16_exponent(groups_max(top), OFFSET ? 110 : 127);
      const float f = __builtin_ldexpf(1.f, -ex);
#pragma unroll
      for (int i = 0; i < 2 * KI; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = pk_f16(x[i][2 * e] * f, x[i][2 * e + 1] * f);
          qf[i][0][e] = w;
          if constexpr (OFFSET) sum = sum_f16(w, sum);
        }
      c_mul = __builtin_ldexpf(a.scale_log2, ex);
      if constexpr (OFFSET) {
        c_add = -128.f * groups_sum(sum) * c_mul;
        c_mul *= 16777216.f;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2 * KI; ++i) {
        const T* p = q + 64 * (i / 2) + 8 * (i & 1);
        float x[8];
        Vec16<float>::unpack(*reinterpret_cast<const uint4*>(p), x);
        Vec16<float>::unpack(*reinterpret_cast<const uint4*>(p + 4), x + 4);
        bf16x8_t t[NT];
        split8<NT>(x, t);
#pragma unroll
        for (int n = 0; n < NT; ++n) qf[i][n] = __builtin_bit_cast(u32x4, t[n]);
      }
    }
  }

  // m_run: the running maximum of head c's scores (the same in its four lanes),
  // l_run: this lane's share of the row sum, in units of 2^m_run.  F16: M_run,
  // the running maximum of score + log2(value scale) - 7; o and lp (the sum of
  // the rounded probabilities) are in units of 2^M_run.  The 7 puts the
  // probabilities (at most 2^15) at the top of f16's range: they keep 11 bits
  // down to 2^-21 of the largest and are dropped below 2^-32.
  float m_run = -INFINITY, M_run = -INFINITY, l_run = 0.f, lp = 0.f;
  float unit = KV8_UNIT;                 // of the sums of fp32 rows (kv8_device.h)
  floatx4 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = floatx4{0.f, 0.f, 0.f, 0.f};

  struct Tile {
    u32x4_nt k[2][KI];
    uint32_t v[8][VW];
    float ks[2], vs[2];
  };
  auto load_v = [&](uint32_t* v, const uint8_t* p) {
    if constexpr (VW == 2) {
      const u32x2_nt w = __builtin_nontemporal_load(reinterpret_cast<const u32x2_nt*>(p));
      v[0] = w[0]; v[1] = w[1];
    } else {
      v[0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
    }
  };
  // 32 keys from k0; positions past the item's end re-read its last key (masked below)
  auto load = [&](Tile& t, int k0) {
    if (k0 + 32 <= ke) {
      const uint8_t* kp = kbase + (size_t)(k0 + c) * D + 16 * gq;
      const uint8_t* vp = vbase + (size_t)(k0 + 4 * gq) * D + DB * c;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < KI; ++i)
          t.k[h][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt*>(kp + 16 * h * D + 64 * i));
#pragma unroll
      for (int e = 0; e < 8; ++e) load_v(t.v[e], vp + (16 * (e >> 2) + (e & 3)) * D);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < KI; ++i)
          t.k[h][i] = __builtin_nontemporal_load(
              reinterpret_cast<const u32x4_nt*>(kbase + (size_t)min(k0 + 16 * h + c, ke - 1) * D + 64 * i + 16 * gq));
#pragma unroll
      for (int e = 0; e < 8; ++e)
        load_v(t.v[e], vbase + (size_t)min(k0 + 16 * (e >> 2) + 4 * gq + (e & 3), ke - 1) * D + DB * c);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int b = min(k0 + 16 * h, ke - 1) >> a.kv.log2_block;
      t.ks[h] = ksc[b];
      t.vs[h] = vsc[b];
    }
  };
  auto step = [&](const Tile& t, int k0) {
    floatx4 s[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      s[h] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KI; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if constexpr (F16) {
            s[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes8_f16<INT8>(t.k[h][i][2 * u], t.k[h][i][2 * u + 1]),
                                                          __builtin_bit_cast(f16x8_t, qf[2 * i + u][0]), s[h], 0, 0, 0);
          } else {
            const bf16x8_t kf = codes8_bf16<INT8>(t.k[h][i][2 * u], t.k[h][i][2 * u + 1]);
#pragma unroll
            for (int n = 0; n < NT; ++n)
              s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, __builtin_bit_cast(bf16x8_t, qf[2 * i + u][n]), s[h], 0, 0, 0);
          }
        }
      const float mul = t.ks[h] * c_mul, add = t.ks[h] * c_add;
#pragma unroll
      for (int v = 0; v < 4; ++v) s[h][v] = OFFSET ? fmaf(s[h][v], mul, add) : s[h][v] * mul;
    }
    if (k0 + 32 > ke) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (k0 + 16 * h + 4 * gq + v >= ke) s[h][v] = -INFINITY;
    }
    // the running maxima move only when exceeded by more than 2^8
    // (probabilities stay below 256; sums and products keep their precision)
    const float mx0 = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3]));
    const float mx1 = fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3]));
    const float mx = groups_max(fmaxf(mx0, mx1));
    uint32_t w[4];
    bf16x8_t pf[NT];
    if constexpr (F16) {
      // value scales as logarithms; a zero scale belongs to zero codes: any small one does for the products
      const float lv0 = __builtin_amdgcn_logf(fmaxf(t.vs[0], KV8_TINY)), lv1 = __builtin_amdgcn_logf(fmaxf(t.vs[1], KV8_TINY));
      const float Mx = groups_max(fmaxf(mx0 + lv0, mx1 + lv1)) - 7.f;
      if (__ballot(mx > m_run + 8.0f || Mx > M_run + 8.0f)) {
        const float m_new = fmaxf(m_run, mx), M_new = fmaxf(M_run, Mx);
        l_run *= m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        const float corr = M_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M_run - M_new);
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] *= corr;
        lp *= corr;
        m_run = m_new;
        M_run = M_new;
      }
      const float d = M_run - m_run;
      // a group's probabilities are 2^(lv - d) of its weights.  Where that may take weights that count
      // (down to 2^-66) below fp32's range, the row sum takes them by themselves.
      const bool apart = __ballot(d - lv0 > 60.f || d - lv1 > 60.f) != 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float lv = h ? lv1 : lv0, add = lv - M_run;
        float p[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) p[v] = __builtin_amdgcn_exp2f(s[h][v] + add);
        if (apart) {
#pragma unroll
          for (int v = 0; v < 4; ++v) l_run += __builtin_amdgcn_exp2f(s[h][v] - m_run);
        } else {                           // back to units of 2^m_run and no value scale
          l_run = fmaf((p[0] + p[1]) + (p[2] + p[3]), __builtin_amdgcn_exp2f(d - lv), l_run);
        }
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const uint32_t pair = pk_f16(p[2 * v], p[2 * v + 1]);
          w[2 * h + v] = pair;
          if constexpr (OFFSET) lp = sum_f16(pair, lp);
        }
      }
    } else {
      const bool change = kv8_unit_change(fmaxf(t.vs[0], t.vs[1]), unit);
      if (__ballot(change || mx > m_run + 8.0f)) {
        const float m_new = fmaxf(m_run, mx);
        const float corr = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        const float corr_o = change ? corr * KV8_UNIT_STEP : corr;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] *= corr_o;
        l_run *= corr;
        m_run = m_new;
      }
      float p[8];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int v = 0; v < 4; ++v) p[4 * h + v] = __builtin_amdgcn_exp2f(s[h][v] - m_run);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        l_run += p[i];
        p[i] *= fmaxf(t.vs[i >> 2], kv8_unit_floor(unit)) * kv8_unit_pow2(unit);
      }
      split8<NT>(p, pf);
    }
#pragma unroll
    for (int x = 0; x < VW; ++x) {
      // bytes 4 x .. + 3 of the eight keys' rows, as four vectors over the keys
      uint32_t v[8];
      u32x4 y[4];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = t.v[e][x];
      transpose8<INT8, F16>(v, y);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const u32x4 vf = y[b];
        if constexpr (F16) {
          o[4 * x + b] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, vf),
                                                                __builtin_bit_cast(f16x8_t, u32x4{w[0], w[1], w[2], w[3]}),
                                                                o[4 * x + b], 0, 0, 0);
        } else {
#pragma unroll
          for (int n = 0; n < NT; ++n)
            o[4 * x + b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, vf), pf[n], o[4 * x + b], 0, 0, 0);
        }
      }
    }
  };

  // OFFSET: o and lp take the codes with their offset, whose sum outgrows the result
  // the more keys there are.  Taken out every CENTRE steps, it and the roundings
  // of the sums stay those of that many steps: over 2^20 keys in one item a mean
  // is off by 7e-5 of a code (by 1.3e-3 without), over 2^17 by 2e-4 (4e-4).
  constexpr int CENTRE = 16;
  auto centre = [&]() {
    const float bias = groups_sum(lp) * (128.f / 16777216.f);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int v = 0; v < 4; ++v) o[db][v] -= bias;
    lp = 0.f;
  };
  Tile t0, t1;
  const int k_first = kb + 32 * wave;
  int k = k_first;
  if (k < ke) load(t0, k);
  while (k < ke) {
    if (k + 32 * NW < ke) load(t1, k + 32 * NW);
    step(t0, k);
    k += 32 * NW;
    if (k >= ke) break;
    if (k + 32 * NW < ke) load(t0, k + 32 * NW);
    step(t1, k);
    k += 32 * NW;
    if constexpr (OFFSET) {
      if ((k - k_first) % (32 * NW * CENTRE) == 0) centre();
    }
  }
  l_run = groups_sum(l_run);
  if constexpr (F16) {
    // to units of 2^m_run; or m_run and l_run to those of 2^M_run, where o may leave
    // fp32's range in the others (m_run -inf: the wave had no keys, all zeros).
    // OFFSET: o = 2^24 (sum of p u) - 128 (sum of p) (since the last centre())
    const float up = m_run == -INFINITY ? 0.f : M_run - m_run, f = __builtin_amdgcn_exp2f(fminf(up, 0.f));
    const float bias = OFFSET ? 128.f * groups_sum(lp) : 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int v = 0; v < 4; ++v) o[db][v] = (OFFSET ? fmaf(o[db][v], 16777216.f, -bias) : o[db][v]) * f;
    l_run *= __builtin_amdgcn_exp2f(fminf(-up, 0.f));
    m_run = fmaxf(m_run, M_run);
  } else {
    l_run *= kv8_unit_pow2(unit);
    const float f = kv8_unit_out(unit, m_run);
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] *= f;
    l_run *= f;
  }

  // Merge of the waves.  Lane (c, gq) holds dims (D / 4) gq + DB v + db of head c in o[db][v].
  float* red_m = red;
  float* red_l = red + NW * 16;
  float* red_o = red + NW * 32;
  if (gq == 0) {
    red_m[wave * 16 + c] = m_run;
    red_l[wave * 16 + c] = l_run;
  }
  if (c < nheads) {
    float* dst = red_o + (wave * nheads + c) * D + (D / 4) * gq;
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
      for (int db = 0; db < DB; db += 4)
        *reinterpret_cast<float4*>(dst + DB * v + db) = make_float4(o[db][v], o[db + 1][v], o[db + 2][v], o[db + 3][v]);
  }
  __syncthreads();
  for (int i = tid; i < nheads * (D / 4); i += 256) {
    const int h = i / (D / 4), d = i % (D / 4) * 4;
    float M = red_m[h];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, red_m[w * 16 + h]);
    const float Ms = M == -INFINITY ? 0.f : M;
    float L = 0.f;
    floatx4 acc{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = __builtin_amdgcn_exp2f(red_m[w * 16 + h] - Ms);
      L = fmaf(f, red_l[w * 16 + h], L);
      acc += f * *reinterpret_cast<const floatx4*>(red_o + (w * nheads + h) * D + d);
    }
    if (part < 0) {
      store_out4<T>(a, row, head0 + h, D, d, acc * (1.0f / L));
    } else {
      float* dst = a.part + ((size_t)part * a.nh + head0 + h) * (D + PART_O);
      *reinterpret_cast<floatx4*>(dst + PART_O + d) = acc;
      if (d == 0) *reinterpret_cast<float2*>(dst) = make_float2(M, L);
    }
  }
}

// The join of the split decodes: one block per (row, head), D / 4 threads per
// partial row and 256 / (D / 4) of them at once, each thread merging every
// GR-th split (running maximum, sum and four columns, four splits' loads in
// flight), then the GR threads of a column in order: the result does not depend
// on which block finished first.  A launch of its own: counted in by the last
// block of the row instead, the fence that makes the other blocks' partials
// visible (one write-back of an XCD's L2 per block) cost 135 us for 640 blocks,
// this launch 3 to 4.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_join_kernel(Kv8DecodeArgs a) {
  constexpr int CG = D / 4, GR = 256 / CG, U = 4;
  __shared__ float jm[GR], jl[GR];
  __shared__ __align__(16) float jo[GR][D];
  const int* jn = a.joins + 3 * blockIdx.x;
  const int row = jn[0], n = jn[1], head = blockIdx.y;
  const int tid = threadIdx.x, col = tid % CG * 4, g = tid / CG;
  const float* src = a.part + ((size_t)jn[2] * a.nh + head) * (D + PART_O);
  const size_t stride = (size_t)a.nh * (D + PART_O);
  float m = -INFINITY, l = 0.f;
  floatx4 acc{0.f, 0.f, 0.f, 0.f};
  for (int j0 = g; j0 < n; j0 += GR * U) {
    float2 ml[U];
    floatx4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float* p = src + (size_t)min(j0 + u * GR, n - 1) * stride;
      ml[u] = *reinterpret_cast<const float2*>(p);
      x[u] = *reinterpret_cast<const floatx4*>(p + PART_O + col);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (j0 + u * GR < n) {
        const float mn = fmaxf(m, ml[u].x), ms = mn == -INFINITY ? 0.f : mn;
        const float f0 = __builtin_amdgcn_exp2f(m - ms), f1 = __builtin_amdgcn_exp2f(ml[u].x - ms);
        l = l * f0 + ml[u].y * f1;
        acc = acc * f0 + x[u] * f1;
        m = mn;
      }
    }
  }
  if (col == 0) {
    jm[g] = m;
    jl[g] = l;
  }
  *reinterpret_cast<floatx4*>(&jo[g][col]) = acc;
  __syncthreads();
  if (g > 0) return;
  float M = jm[0];
#pragma unroll
  for (int i = 1; i < GR; ++i) M = fmaxf(M, jm[i]);
  const float Ms = M == -INFINITY ? 0.f : M;
  float L = 0.f;
  acc = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < GR; ++i) {
    const float f = __builtin_amdgcn_exp2f(jm[i] - Ms);
    L = fmaf(f, jl[i], L);
    acc += f * *reinterpret_cast<const floatx4*>(&jo[i][col]);
  }
  store_out4<T>(a, row, head, D, col, acc * (1.0f / L));
}

template <typename T, int D>
static hipError_t run_decode(int format, const Kv8DecodeArgs& a, hipStream_t s) {
  const int group = a.nh / a.nkv, hblocks = (group + 15) / 16;
  const dim3 grid((unsigned)((size_t)a.n_work * a.nkv * hblocks));
  const size_t lds = (4 * 32 + (size_t)4 * (group < 16 ? group : 16) * D) * 4;   // at most 33 KB
  if (format == 0) hipLaunchKernelGGL((kv8_attn_rows_kernel<T, D, true>), grid, dim3(256), lds, s, a);
  else hipLaunchKernelGGL((kv8_attn_rows_kernel<T, D, false>), grid, dim3(256), lds, s, a);
  if (a.n_joins > 0) hipLaunchKernelGGL((kv8_join_kernel<T, D>), dim3(a.n_joins, a.nh), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv8_decode(int dtype, int format, int hd, const Kv8DecodeArgs& a, hipStream_t s) {
  if (a.n_work <= 0) return hipSuccess;
  if (dtype == 0) return hd == 128 ? run_decode<float, 128>(format, a, s) : run_decode<float, 64>(format, a, s);
  return hd == 128 ? run_decode<bf16, 128>(format, a, s) : run_decode<bf16, 64>(format, a, s);
}

}  // namespace sarathi
