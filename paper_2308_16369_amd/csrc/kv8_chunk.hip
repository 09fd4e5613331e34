// Attention of prompt chunks over the 8-bit KV cache.
//
// Block = one key/value head, KV8_QB packed query rows (the rows of the chunk
// times the query heads that share the key/value head; four waves of 32) and a
// range of 64-key tiles.  A tile's codes are read once per block, converted to
// bf16 (exact) on the way into LDS, and multiplied there by every wave:
//   S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_32x32x16_bf16, a lane (ql =
//   lane % 32, g = lane / 32) holding the scores of packed row ql for keys
//   8 (v / 4) + 4 g + v % 4 of each 32-key half; V^T comes from transposed LDS
//   reads.  A scale is constant over 16 keys: the key scale joins the softmax
//   scale in the exponent, the value scale enters there as its logarithm (the
//   row sum divides it out again), so neither costs a multiplication per score.
#include "kv8.h"

namespace sarathi {

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ uint32_t pk2_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, bf16x2_t));
}

// 16 codes to 16 bf16.
template <bool INT8>
__device__ __forceinline__ void widen16(const uint4& w, u32x4& lo, u32x4& hi) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t r[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (INT8) {
      r[2 * i] = pk2_bf16((float)(signed char)x[i], (float)(signed char)(x[i] >> 8));
      r[2 * i + 1] = pk2_bf16((float)(signed char)(x[i] >> 16), (float)(signed char)(x[i] >> 24));
    } else {
      r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], 1.0f, false));
      r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], 1.0f, true));
    }
  }
  lo = u32x4{r[0], r[1], r[2], r[3]};
  hi = u32x4{r[4], r[5], r[6], r[7]};
}

// Swizzle of a tile row's 16-byte chunks: a bijection of the row mod 16 that
// moves aligned groups of four together (head_dim 128), so that both the row
// reads of K and the transposed reads of V fall on distinct LDS banks.
template <int D>
__device__ __forceinline__ int swz(int c, int r) {
  if (D == 128) return c ^ (((r & 3) << 2) | ((r >> 2) & 3));
  return c ^ (r & 7);
}

__device__ __forceinline__ float lanes_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float lanes_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int NT>
__device__ __forceinline__ void terms8(const float* x, bf16x8_t* t) {
  float r[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = pk2_bf16(r[2 * e], r[2 * e + 1]);
      r[2 * e] -= __uint_as_float(w[e] << 16);
      r[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
    }
    t[n] = __builtin_bit_cast(bf16x8_t, w);
  }
}

typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
__device__ __forceinline__ uint2 lds_tr16(const char* p) {
  const v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)p);
  return __builtin_bit_cast(uint2, v);
}

template <typename T, int D, bool INT8>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void kv8_attn_chunk_kernel(Kv8ChunkArgs a) {
  constexpr int NT = sizeof(T) == 2 ? 1 : 3;
  constexpr int KT = KV8_KT, QB = KV8_QB;
  constexpr int DCH = D / 8;             // 16-byte chunks per bf16 tile row
  constexpr int TILE = KT * DCH;         // chunks per tile
  constexpr int LPR = D / 16;            // lanes that read a key row (16 codes each)
  constexpr int NI = KT * LPR / 256;     // 16-byte loads per thread and tile (K or V)
  __shared__ u32x4 ring[2][2][TILE];     // [stage][K, V]

  const int item = blockIdx.x / a.nkv, kvh = blockIdx.x % a.nkv;
  const int* wk = a.work + 4 * item;
  const int* ch = a.chunks + 4 * wk[0];
  const int slot = ch[0], offset = ch[1], C = ch[2], row0 = ch[3];
  const int r0 = wk[1], part = wk[2];
  const int group = a.nh / a.nkv;
  const int nrows = min(QB / group, C - r0);       // the block's chunk rows
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = lane >> 5, ql = lane & 31;

  const uint8_t* kbase = a.kv.codes + slot * a.kv.slot + kvh * a.kv.head;
  const uint8_t* vbase = kbase + a.kv.kv;
  const float* ksc = a.kv.scales + slot * a.kv.s_slot + kvh * a.kv.s_head;
  const float* vsc = ksc + a.kv.s_kv;

  const int kbeg = (wk[3] >> 16) * KT;
  const int kend = min(offset + r0 + nrows, (wk[3] & 0xffff) * KT);
  const int n_tiles = (kend - kbeg + KT - 1) / KT;

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
        terms8<NT>(x, qf[ks]);
      }
    }
  }

  float m_run = -INFINITY, l_run = 0.f;
  floatx16 o_acc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int v = 0; v < 16; ++v) o_acc[db][v] = 0.f;

  // tile staging: thread -> NI pieces of 16 codes of K and of V
  uint4 kr[NI], vr[NI];
  auto fetch = [&](int kt) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int at = i * 256 + tid, r = at / LPR, c = at % LPR;
      const size_t off = (size_t)min(kbeg + kt * KT + r, kend - 1) * D + 16 * c;
      kr[i] = *reinterpret_cast<const uint4*>(kbase + off);
      vr[i] = *reinterpret_cast<const uint4*>(vbase + off);
    }
  };
  auto stage = [&](int buf) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int at = i * 256 + tid, r = at / LPR, c = at % LPR;
      u32x4 lo, hi;
      widen16<INT8>(kr[i], lo, hi);
      ring[buf][0][r * DCH + swz<D>(2 * c, r)] = lo;
      ring[buf][0][r * DCH + swz<D>(2 * c + 1, r)] = hi;
      widen16<INT8>(vr[i], lo, hi);
      ring[buf][1][r * DCH + swz<D>(2 * c, r)] = lo;
      ring[buf][1][r * DCH + swz<D>(2 * c + 1, r)] = hi;
    }
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

  auto compute = [&](int kt, int buf) {
    const int k0 = kbeg + kt * KT;
    if (k0 > last_key || idle) return;
    // scales of the four 16-key groups; a zero scale belongs to zero codes, so 1 does as well
    float ks4[4], vs4[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = min(k0 + 16 * i, kend - 1) >> a.kv.log2_block;
      const float x = ksc[b], y = vsc[b];
      ks4[i] = (x > 0.f ? x : 1.f) * a.scale_log2;
      vs4[i] = y > 0.f ? y : 1.f;
    }
    floatx16 s[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int v = 0; v < 16; ++v) s[kb][v] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, ring[buf][0][kb * 32 * DCH + koff[ks]]);
#pragma unroll
        for (int n = 0; n < NT; ++n) s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks][n], s[kb], 0, 0, 0);
      }
    }
    const bool full = k0 + KT <= kend && k0 + KT - 1 <= offset + r0 + wave * 32 / group;
    if (!full) {
      const int lim = min(qpos, kend - 1) - k0;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (kb * 32 + 8 * (v >> 2) + 4 * g + (v & 3) > lim) s[kb][v] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float t = s[i >> 1][8 * (i & 1)];
#pragma unroll
      for (int v = 1; v < 8; ++v) t = fmaxf(t, s[i >> 1][8 * (i & 1) + v]);
      mx = fmaxf(mx, t * ks4[i]);
    }
    mx = lanes_max(mx);
    if (__ballot(mx > m_run + 8.0f)) {
      const float m_new = fmaxf(m_run, mx);
      const float corr = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) o_acc[db] *= corr;
      l_run *= corr;
      m_run = m_new;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    bf16x8_t pf[4][NT];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float add = __builtin_amdgcn_logf(vs4[i]) - m_use;   // log2
      float p[8], sum = 0.f;
#pragma unroll
      for (int v = 0; v < 8; ++v) p[v] = __builtin_amdgcn_exp2f(fmaf(s[i >> 1][8 * (i & 1) + v], ks4[i], add));
      terms8<NT>(p, pf[i]);
      if constexpr (NT == 1) {
        // the row sum takes the rounded probabilities that multiply V
        const u32x4 w = __builtin_bit_cast(u32x4, pf[i][0]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t pair = w[e];
          sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pair),
                                                __builtin_convertvector((f32x2_t){1.f, 1.f}, bf16x2_t), sum, false);
        }
      } else {
#pragma unroll
        for (int v = 0; v < 8; ++v) sum += p[v];
      }
      l_run = fmaf(sum, 1.0f / vs4[i], l_run);
    }
    const char* vt = reinterpret_cast<const char*>(ring[buf][1]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const uint2 x = lds_tr16(vt + voff[0][db] + i * 16 * DCH * 16), y = lds_tr16(vt + voff[1][db] + i * 16 * DCH * 16);
        const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, u32x4{x.x, x.y, y.x, y.y});
#pragma unroll
        for (int n = 0; n < NT; ++n)
          o_acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[i][n], o_acc[db], 0, 0, 0);
      }
  };

  fetch(0);
  stage(0);
  __syncthreads();
  for (int kt = 0; kt < n_tiles; ++kt) {
    if (kt + 1 < n_tiles) fetch(kt + 1);
    compute(kt, kt & 1);
    if (kt + 1 < n_tiles) stage((kt + 1) & 1);
    __syncthreads();
  }
  l_run = lanes_sum(l_run);
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
        if constexpr (NT == 1) *reinterpret_cast<uint2*>(out + d) = make_uint2(pk2_bf16(x[0], x[1]), pk2_bf16(x[2], x[3]));
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

template <typename T, int D>
static hipError_t run_chunk(int format, const Kv8ChunkArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((size_t)a.n_work * a.nkv));
  if (format == 0) hipLaunchKernelGGL((kv8_attn_chunk_kernel<T, D, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((kv8_attn_chunk_kernel<T, D, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_kv8_chunk(int dtype, int format, int hd, const Kv8ChunkArgs& a, hipStream_t s) {
  if (a.n_work <= 0) return hipSuccess;
  if (dtype == 0) return hd == 128 ? run_chunk<float, 128>(format, a, s) : run_chunk<float, 64>(format, a, s);
  return hd == 128 ? run_chunk<bf16, 128>(format, a, s) : run_chunk<bf16, 64>(format, a, s);
}

}  // namespace sarathi
