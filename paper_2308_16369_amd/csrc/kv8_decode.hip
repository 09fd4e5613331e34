// Attention of the decodes of a batch over the 8-bit KV cache.
//
// Work item = (decode, a range of its keys), one block per item, key/value
// head and group of 16 query heads; four waves take steps of 32 keys in turn.
// A wave multiplies on v_mfma_f32_16x16x32_bf16 straight from registers, the
// codes converted to bf16 (exact for both formats):
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
#include "kv8.h"

namespace sarathi {

typedef unsigned int u32x4_nt __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2_nt __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pk_bf16(float a, float b) {   // nearest even; low half = a
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, bf16x2_t));
}

// Four codes (a dword) to bf16: lo = codes 0, 1; hi = codes 2, 3.
template <bool INT8>
__device__ __forceinline__ void codes_bf16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (INT8) {
    lo = pk_bf16((float)(signed char)w, (float)(signed char)(w >> 8));
    hi = pk_bf16((float)(signed char)(w >> 16), (float)(signed char)(w >> 24));
  } else {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
  }
}
template <bool INT8>
__device__ __forceinline__ bf16x8_t codes8_bf16(uint32_t a, uint32_t b) {
  u32x4 r;
  uint32_t x, y;
  codes_bf16<INT8>(a, x, y);
  r[0] = x; r[1] = y;
  codes_bf16<INT8>(b, x, y);
  r[2] = x; r[3] = y;
  return __builtin_bit_cast(bf16x8_t, r);
}

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

// x as NT bf16 terms of eight values each: bf16 rows are one exact term; fp32
// takes three (the remainders of the first two are exact in fp32), 24 bits.
template <int NT>
__device__ __forceinline__ void split8(const float* x, bf16x8_t* t) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = pk_bf16(r[2 * e], r[2 * e + 1]);
      r[2 * e] -= __uint_as_float(w[e] << 16);
      r[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
    }
    t[n] = __builtin_bit_cast(bf16x8_t, w);
  }
}

template <typename T, int D, bool INT8>
__global__ __launch_bounds__(256) void kv8_attn_rows_kernel(Kv8DecodeArgs a) {
  constexpr int NT = sizeof(T) == 2 ? 1 : 3;
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
  const int* wk = a.work + 5 * item;
  const int row = wk[0], slot = wk[1], kb = wk[2], ke = wk[3], part = wk[4];

  const uint8_t* kbase = a.kv.codes + slot * a.kv.slot + kvh * a.kv.head;
  const uint8_t* vbase = kbase + a.kv.kv;
  const float* ksc = a.kv.scales + slot * a.kv.s_slot + kvh * a.kv.s_head;
  const float* vsc = ksc + a.kv.s_kv;

  bf16x8_t qf[2 * KI][NT];
  {
    const T* q = reinterpret_cast<const T*>(a.q) + (size_t)row * a.ld_q + (size_t)(head0 + min(c, nheads - 1)) * D;
#pragma unroll
    for (int i = 0; i < 2 * KI; ++i) {
      const T* p = q + 64 * (i / 2) + 16 * gq + 8 * (i & 1);
      if constexpr (NT == 1) {
        qf[i][0] = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const u32x4*>(p));
      } else {
        float x[8];
        Vec16<float>::unpack(*reinterpret_cast<const uint4*>(p), x);
        Vec16<float>::unpack(*reinterpret_cast<const uint4*>(p + 4), x + 4);
        split8<NT>(x, qf[i]);
      }
    }
  }

  float m_run = -INFINITY, l_run = 0.f;   // m: of head c, the same in its four lanes; l: this lane's keys
  floatx4 o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = floatx4{0.f, 0.f, 0.f, 0.f};

  struct Tile {
    u32x4_nt k[2][KI];
    uint32_t v[8][VW];
    float ks[2], vs[2], vi[2];   // the two 16-key tiles' scales of K and V, and 1 / V's
  };
  // 32 keys from k0; positions past the item's end re-read its last key (masked below)
  auto load = [&](Tile& t, int k0) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < KI; ++i)
        t.k[h][i] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4_nt*>(kbase + (size_t)min(k0 + 16 * h + c, ke - 1) * D + 64 * i + 16 * gq));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint8_t* p = vbase + (size_t)min(k0 + 16 * (e >> 2) + 4 * gq + (e & 3), ke - 1) * D + DB * c;
      if constexpr (VW == 2) {
        const u32x2_nt w = __builtin_nontemporal_load(reinterpret_cast<const u32x2_nt*>(p));
        t.v[e][0] = w[0]; t.v[e][1] = w[1];
      } else {
        t.v[e][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(p));
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int b = min(k0 + 16 * h, ke - 1) >> a.kv.log2_block;
      t.ks[h] = ksc[b];
      const float y = vsc[b];
      t.vs[h] = y > 0.f ? y : 1.f;      // a zero scale belongs to zero codes
      t.vi[h] = 1.0f / t.vs[h];
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
          const bf16x8_t kf = codes8_bf16<INT8>(t.k[h][i][2 * u], t.k[h][i][2 * u + 1]);
#pragma unroll
          for (int n = 0; n < NT; ++n)
            s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[2 * i + u][n], s[h], 0, 0, 0);
        }
      s[h] *= t.ks[h] * a.scale_log2;
    }
    if (k0 + 32 > ke) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          if (k0 + 16 * h + 4 * gq + v >= ke) s[h][v] = -INFINITY;
    }
    // the running maximum moves only when a score exceeds it by more than 2^8
    // (probabilities stay below 256; sums and products keep their precision)
    float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                     fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    mx = groups_max(mx);
    if (__ballot(mx > m_run + 8.0f)) {
      const float m_new = fmaxf(m_run, mx);
      const float corr = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] *= corr;
      l_run *= corr;
      m_run = m_new;
    }
    float p[8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int v = 0; v < 4; ++v) p[4 * h + v] = __builtin_amdgcn_exp2f(s[h][v] - m_run);
    bf16x8_t pf[NT];
    if constexpr (NT == 1) {
      // the row sum takes the rounded probabilities that multiply V: the
      // weights add up to one, whatever their rounding
      const bf16x2_t ones = __builtin_convertvector((f32x2_t){1.f, 1.f}, bf16x2_t);
      u32x4 w;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          const uint32_t pair = pk_bf16(p[4 * h + 2 * v] * t.vs[h], p[4 * h + 2 * v + 1] * t.vs[h]);
          w[2 * h + v] = pair;
          sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pair), ones, sum, false);
        }
        l_run = fmaf(sum, t.vi[h], l_run);
      }
      pf[0] = __builtin_bit_cast(bf16x8_t, w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        l_run += p[i];
        p[i] *= t.vs[i >> 2];
      }
      split8<NT>(p, pf);
    }
#pragma unroll
    for (int w = 0; w < VW; ++w) {
      // bytes 4 w .. + 3 of the eight keys' rows, as four vectors over the keys
      uint32_t x[4][4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t lo0, hi0, lo1, hi1;
        codes_bf16<INT8>(t.v[2 * e][w], lo0, hi0);
        codes_bf16<INT8>(t.v[2 * e + 1][w], lo1, hi1);
        x[0][e] = __builtin_amdgcn_perm(lo1, lo0, 0x05040100);
        x[1][e] = __builtin_amdgcn_perm(lo1, lo0, 0x07060302);
        x[2][e] = __builtin_amdgcn_perm(hi1, hi0, 0x05040100);
        x[3][e] = __builtin_amdgcn_perm(hi1, hi0, 0x07060302);
      }
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, u32x4{x[b][0], x[b][1], x[b][2], x[b][3]});
#pragma unroll
        for (int n = 0; n < NT; ++n)
          o[4 * w + b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[n], o[4 * w + b], 0, 0, 0);
      }
    }
  };

  Tile t0, t1;
  int k = kb + 32 * wave;
  if (k < ke) load(t0, k);
  while (k < ke) {
    if (k + 32 * NW < ke) load(t1, k + 32 * NW);
    step(t0, k);
    k += 32 * NW;
    if (k >= ke) break;
    if (k + 32 * NW < ke) load(t0, k + 32 * NW);
    step(t1, k);
    k += 32 * NW;
  }
  l_run = groups_sum(l_run);

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
      acc *= 1.0f / L;
      T* out = reinterpret_cast<T*>(a.out) + (size_t)row * a.ld_out + (size_t)(head0 + h) * D + d;
      if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(out) = make_uint2(pk_bf16(acc[0], acc[1]), pk_bf16(acc[2], acc[3]));
      else *reinterpret_cast<floatx4*>(out) = acc;
    } else {
      float* dst = a.part + ((size_t)part * a.nh + head0 + h) * (D + PART_O);
      *reinterpret_cast<floatx4*>(dst + PART_O + d) = acc;
      if (d == 0) {
        dst[0] = M;
        dst[1] = L;
      }
    }
  }
}

template <typename T, int D>
static hipError_t run_decode(int format, const Kv8DecodeArgs& a, hipStream_t s) {
  const int group = a.nh / a.nkv, hblocks = (group + 15) / 16;
  const dim3 grid((unsigned)((size_t)a.n_work * a.nkv * hblocks));
  const size_t lds = (4 * 32 + (size_t)4 * (group < 16 ? group : 16) * D) * 4;   // at most 33 KB
  if (format == 0) hipLaunchKernelGGL((kv8_attn_rows_kernel<T, D, true>), grid, dim3(256), lds, s, a);
  else hipLaunchKernelGGL((kv8_attn_rows_kernel<T, D, false>), grid, dim3(256), lds, s, a);
  return hipGetLastError();
}

hipError_t launch_kv8_decode(int dtype, int format, int hd, const Kv8DecodeArgs& a, hipStream_t s) {
  if (a.n_work <= 0) return hipSuccess;
  if (dtype == 0) return hd == 128 ? run_decode<float, 128>(format, a, s) : run_decode<float, 64>(format, a, s);
  return hd == 128 ? run_decode<bf16, 128>(format, a, s) : run_decode<bf16, 64>(format, a, s);
}

}  // namespace sarathi
