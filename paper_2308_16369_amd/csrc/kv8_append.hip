// The 8-bit KV cache's writers and reader: the append (head norms, rotary
// positions, quantisation) and the read of the held values.  All memory-bound.
#include "kv8.h"

namespace sarathi {

// ------------------------------------------------------------------ a plan's rows
// One block per span.  Angles, sines and cosines in fp64, rounded once: a sine
// of the angle rounded to fp32 is off by up to 2^-23 more, and rows near the
// middle of two codes then take the other one.  Made once for a batch and read
// by every layer's append.
__global__ __launch_bounds__(256) void kv8_rows_kernel(Kv8RowsArgs a) {
  const int* sp = a.spans + KV8_SPAN_INTS * blockIdx.x;
  const int slot = sp[0], pos = sp[1], row = sp[2], n = sp[3], part = sp[4], ns = sp[5], stride = sp[6];
  if ((int)threadIdx.x < n) {
    const int r = row + threadIdx.x;
    a.row_slot[r] = slot;
    a.row_pos[r] = pos + threadIdx.x;
    a.comb[3 * r] = part + threadIdx.x;
    a.comb[3 * r + 1] = ns;
    a.comb[3 * r + 2] = stride;
  }
  for (int t = threadIdx.x; t < n * a.pairs; t += 256) {
    const int j = t / a.pairs, i = t - j * a.pairs;
    const double ang = (double)(pos + j) * a.theta[i];
    const double red = ang - 6.283185307179586 * rint(ang * 0.15915494309189535);
    double sn, cs;
    sincos(red, &sn, &cs);
    a.tab[(size_t)(row + j) * a.pairs + i] = make_float2((float)(cs * a.mscale), (float)(sn * a.mscale));
  }
}

hipError_t launch_kv8_rows(const Kv8RowsArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(kv8_rows_kernel, dim3(a.n_spans), dim3(256), 0, s, a);
  return hipGetLastError();
}

// ------------------------------------------------------------------ append
// A head row of D elements sits in D / 8 neighbouring lanes, eight elements
// each (LPR lanes per row, RPW rows per wave).
// Bound by reading and writing its rows: 2048 rows of 52 heads (136 MB) in 33 us,
// 4.1 TB/s (a large copy: 4.7); a few decodes (64 rows of 40 / 8 heads, 4.6 us) by
// latency.  Rows of qkv are read once, so past the caches: with ordinary loads
// and stores the append and the read of that prompt took 9 % more.
typedef unsigned int u32x4_nt __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load16_nt(const void* p) {
  const u32x4_nt v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_nt*>(p));
  return make_uint4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void store16_nt(void* p, uint4 v) {
  __builtin_nontemporal_store((u32x4_nt){v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4_nt*>(p));
}
template <typename T, bool ONCE = true>
__device__ __forceinline__ void kv8_load8(const T* p, float* x) {
  auto get = [](const T* q) { return ONCE ? load16_nt(q) : *reinterpret_cast<const uint4*>(q); };
  Vec16<T>::unpack(get(p), x);
  if constexpr (sizeof(T) == 4) Vec16<T>::unpack(get(p + 4), x + 4);
}
typedef __bf16 kv8_bf16x2 __attribute__((ext_vector_type(2)));
typedef float kv8_f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t kv8_pack_bf16(float a, float b) {   // nearest even
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((kv8_f32x2){a, b}, kv8_bf16x2));
}
template <typename T, bool STREAM = false>
__device__ __forceinline__ void kv8_store8(T* p, const float* x) {
  auto put = [](T* q, uint4 v) { STREAM ? store16_nt(q, v) : (void)(*reinterpret_cast<uint4*>(q) = v); };
  if constexpr (sizeof(T) == 2) {
    put(p, make_uint4(kv8_pack_bf16(x[0], x[1]), kv8_pack_bf16(x[2], x[3]), kv8_pack_bf16(x[4], x[5]),
                      kv8_pack_bf16(x[6], x[7])));
  } else {
#pragma unroll
    for (int i = 0; i < 8; i += 4)
      put(p + i, make_uint4(__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]),
                            __float_as_uint(x[i + 3])));
  }
}

// Maximum that propagates NaN.
__device__ __forceinline__ float max_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
// Exchanges within 16 lanes (DPP row mirror, half mirror, quad permutes): a
// butterfly over them reaches all 16 lanes, from half mirror on all 8 of a half.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_amdgcn_update_dpp(0.f, v, CTRL, 0xf, 0xf, false);
}
template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
  if constexpr (LPR == 16) v += dpp<0x140>(v);
  v += dpp<0x141>(v);
  v += dpp<0x1B>(v);
  return v + dpp<0xB1>(v);
}
__device__ __forceinline__ float wave_max_nan(float v) {
  v = max_nan(v, dpp<0x140>(v));
  v = max_nan(v, dpp<0x141>(v));
  v = max_nan(v, dpp<0x1B>(v));
  v = max_nan(v, dpp<0xB1>(v));
  v = max_nan(v, __shfl_xor(v, 16, 64));
  return max_nan(v, __shfl_xor(v, 32, 64));
}

// Eight elements of a head row: norm (gain: this lane's eight gains, null for
// none), then the rotation by table row `tab`; j = the lane's place in the row.
template <int D>
__device__ __forceinline__ void norm_rotate(float* x, const float* gain, float eps, const float2* __restrict__ tab, int rot,
                                            int interleaved, int j) {
  constexpr int LPR = D / 8;
  if (gain) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
    const float inv = 1.0f / sqrtf(row_sum<LPR>(ss) * (1.0f / D) + eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= inv * gain[e];
  }
  if (rot == 0) return;
  const int d0 = 8 * j, half = rot / 2;
  const bool turns = d0 < rot;
  if (interleaved) {
    if (turns) {
      const float4* t = reinterpret_cast<const float4*>(tab + d0 / 2);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float4 cs = t[e];
        const float a = x[4 * e], b = x[4 * e + 1], c = x[4 * e + 2], d = x[4 * e + 3];
        x[4 * e] = a * cs.x - b * cs.y;
        x[4 * e + 1] = a * cs.y + b * cs.x;
        x[4 * e + 2] = c * cs.z - d * cs.w;
        x[4 * e + 3] = c * cs.w + d * cs.z;
      }
    }
    return;
  }
  // the partners' eight elements lie half / 8 lanes up or down
  const bool first = d0 < half;
  const int step = turns ? (first ? half / 8 : -(half / 8)) : 0;
  const int from = (threadIdx.x & 63) + step;
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = __shfl(x[e], from, 64);
  if (turns) {
    const float4* t = reinterpret_cast<const float4*>(tab + (first ? d0 : d0 - half));
    const float sg = first ? -1.f : 1.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float4 cs = t[e];
      x[2 * e] = x[2 * e] * cs.x + sg * y[2 * e] * cs.y;
      x[2 * e + 1] = x[2 * e + 1] * cs.z + sg * y[2 * e + 1] * cs.w;
    }
  }
}

// Largest magnitude of eight elements, NaN where one is.
__device__ __forceinline__ float top8(const float* x, float top) {
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max_nan(top, fabsf(x[e]));
  return top;
}
__device__ __forceinline__ bool is_finite(float top) { return top <= 3.4028234663852886e38f; }
// NaN to zero, infinities to the largest finite value of their sign; returns
// the magnitude that counts for the scale (0 for both).
__device__ __forceinline__ float tame8(float* x) {
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float m = fabsf(x[e]);
    if (is_finite(m)) top = fmaxf(top, m);
    else x[e] = m == INFINITY ? copysignf(3.4028234663852886e38f, x[e]) : 0.f;
  }
  return top;
}

// The scale that values of magnitude up to `top` need.
template <bool INT8>
__device__ __forceinline__ float scale_of(float top) {
  const float s = top / (INT8 ? KV8_INT8_MAX : KV8_E4M3_MAX);
  if (s < KV8_TINY) return 0.f;
  if (INT8) return s;
  return __uint_as_float((__float_as_uint(s) + 0x7fffffu) & 0xff800000u);   // the next power of two
}

// Eight codes of x * inv, |x * inv| at most the largest code but for the last
// bits, which the rounding takes away.  int8: adding 1.5 2^23 rounds the product
// to the nearest whole number (ties to even), which the sum's low byte then is.
template <bool INT8>
__device__ __forceinline__ uint2 encode8(const float* x, float inv) {
#pragma clang fp contract(off)
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float* y = x + 4 * h;
    if constexpr (INT8) {
      uint32_t b[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = __float_as_uint(y[e] * inv + 12582912.f);
      w[h] = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400) | __builtin_amdgcn_perm(b[3], b[2], 0x04000c0c);
    } else {
      const int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * inv, y[1] * inv, 0, false);
      w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2] * inv, y[3] * inv, v, true);
    }
  }
  return make_uint2(w[0], w[1]);
}
// The largest codes of the tamed infinities, whose x * inv lies far outside.
template <bool INT8>
__device__ __forceinline__ void clamp8(float* x, float now) {
  const float m = now * (INT8 ? KV8_INT8_MAX : KV8_E4M3_MAX);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = fminf(fmaxf(x[e], -m), m);
}
template <bool INT8>
__device__ __forceinline__ void decode4(uint32_t w, float* x) {
  if constexpr (INT8) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = (float)(signed char)(w >> (8 * e));
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
  }
}

// Codes of the block's positions before p0 to a scale `ratio` = old / new < 1;
// `lane` of `lanes` lanes.
template <int D, bool INT8>
__device__ __forceinline__ void rescale_old(uint8_t* codes, int p0, float ratio, int lane, int lanes) {
  for (int i = lane; i < p0 * (D / 8); i += lanes) {
    uint2* p = reinterpret_cast<uint2*>(codes + (size_t)i * 8);
    const uint2 w = *p;
    float x[8];
    decode4<INT8>(w.x, x);
    decode4<INT8>(w.y, x + 4);
    *p = encode8<INT8>(x, ratio);
  }
}

// One launch, three kinds of blocks (256 threads):
//   queries: a wave takes U * 64 / LPR heads of a row, all loads in flight; every
//     lane keeps the same eight dims, so the row's gains and table entries are
//     read once;
//   units of several rows (prompt chunks): one block per (unit, K or V, head)
//     holds the block's new rows in registers across the maximum;
//   units of one row (decodes): one wave each.
// NP: register passes that cover a block's rows.
template <typename T, int D, bool INT8, int NP>
__global__ __launch_bounds__(256, NP == 8 ? 4 : 6) void kv8_append_kernel(Kv8AppendArgs a, int q_blocks, int c_blocks, int hpw) {
  constexpr int U = 4;
  constexpr int LPR = D / 8, RPW = 64 / LPR, RPP = 4 * RPW;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int j = lane % LPR, g = lane / LPR;
  const T* qkv = reinterpret_cast<const T*>(a.qkv);
  const int pairs = a.rot / 2;
  const int blk = blockIdx.x;
  if (blk < q_blocks) {
    const int per_row = (a.nh + hpw - 1) / hpw;
    const long w = (long)blk * 4 + wave;
    const int row = (int)(w / per_row), h0 = (int)(w % per_row) * hpw;
    if (row >= a.T) return;
    float gain[8];
    if (a.q_gain) kv8_load8<T, false>(reinterpret_cast<const T*>(a.q_gain) + 8 * j, gain);
    const T* src = qkv + (size_t)row * a.ld_qkv + 8 * j;
    T* dst = reinterpret_cast<T*>(a.q_out) + (size_t)row * a.ld_q + 8 * j;
    const int h1 = min(a.nh, h0 + hpw);
    float x[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u)            // lanes past the last head repeat it, unwritten
      if (h0 + u * RPW < h1) kv8_load8(src + (size_t)min(h0 + u * RPW + g, h1 - 1) * D, x[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = h0 + u * RPW + g;
      if (h0 + u * RPW < h1) {
        norm_rotate<D>(x[u], a.q_gain ? gain : nullptr, a.eps, a.tab + (size_t)row * pairs, a.rot, a.interleaved, j);
        if (h < h1) kv8_store8(dst + (size_t)h * D, x[u]);
      }
    }
    return;
  }
  const int heads2 = 2 * a.nkv;
  if (blk < q_blocks + c_blocks) {
    const int at = blk - q_blocks;
    const int* u = a.units + 4 * (at / heads2);
    const int which = at % heads2 / a.nkv, h = at % heads2 % a.nkv;
    const int slot = u[0], b = u[1], row0 = u[2], p0 = u[3] >> 16, n = (u[3] & 0xffff) - p0;
    uint8_t* codes = a.kv.codes + slot * a.kv.slot + which * a.kv.kv + h * a.kv.head +
                     ((size_t)b << a.kv.log2_block) * D;
    float* scale = a.kv.scales + slot * a.kv.s_slot + which * a.kv.s_kv + h * a.kv.s_head + b;
    const float was = p0 > 0 ? *scale : 0.f;
    float gain[8];
    const bool norm = a.k_gain != nullptr && which == 0;
    if (norm) kv8_load8<T, false>(reinterpret_cast<const T*>(a.k_gain) + 8 * j, gain);
    const T* src = qkv + (size_t)row0 * a.ld_qkv + (size_t)(a.nh + which * a.nkv + h) * D + 8 * j;
    float x[NP][8], top = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = i * RPP + wave * RPW + g;
      if (i * RPP < n) kv8_load8(src + (size_t)min(r, n - 1) * a.ld_qkv, x[i]);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if (i * RPP < n) {
        const int r = min(i * RPP + wave * RPW + g, n - 1);
        if (which == 0)
          norm_rotate<D>(x[i], norm ? gain : nullptr, a.eps, a.tab + (size_t)(row0 + r) * pairs, a.rot, a.interleaved, j);
        top = top8(x[i], top);
      }
    }
    __shared__ float red[2][4];
    top = wave_max_nan(top);
    if (lane == 0) red[0][wave] = top;
    __syncthreads();
    top = max_nan(max_nan(red[0][0], red[0][1]), max_nan(red[0][2], red[0][3]));
    const bool tamed = !is_finite(top);
    if (tamed) {                           // the whole block: something is not finite
      top = 0.f;
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (i * RPP < n) top = fmaxf(top, tame8(x[i]));
      top = wave_max(top);
      if (lane == 0) red[1][wave] = top;
      __syncthreads();
      top = fmaxf(fmaxf(red[1][0], red[1][1]), fmaxf(red[1][2], red[1][3]));
    }
    const float now = fmaxf(was, scale_of<INT8>(top));
    if (tamed) {
#pragma unroll
      for (int i = 0; i < NP; ++i)
        if (i * RPP < n) clamp8<INT8>(x[i], now);
    }
    const float inv = now > 0.f ? 1.0f / now : 0.f;
    if (tid == 0) *scale = now;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = i * RPP + wave * RPW + g;
      if (r < n) *reinterpret_cast<uint2*>(codes + (size_t)(p0 + r) * D + 8 * j) = encode8<INT8>(x[i], inv);
    }
    if (now > was) rescale_old<D, INT8>(codes, p0, was * inv, tid, 256);
    return;
  }
  const long w = (long)(blk - q_blocks - c_blocks) * 4 + wave;
  const int at = (int)(w / heads2);
  if (at >= a.n_units - a.n_chunk) return;
  const int* u = a.units + 4 * (a.n_chunk + at);
  const int which = (int)(w % heads2) / a.nkv, h = (int)(w % heads2) % a.nkv;
  const int slot = u[0], b = u[1], row = u[2], p0 = u[3] >> 16;
  uint8_t* codes = a.kv.codes + slot * a.kv.slot + which * a.kv.kv + h * a.kv.head + ((size_t)b << a.kv.log2_block) * D;
  float* scale = a.kv.scales + slot * a.kv.s_slot + which * a.kv.s_kv + h * a.kv.s_head + b;
  const float was = p0 > 0 ? *scale : 0.f;
  float x[8], gain[8], top = 0.f;
  const bool norm = a.k_gain != nullptr && which == 0;
  kv8_load8(qkv + (size_t)row * a.ld_qkv + (size_t)(a.nh + which * a.nkv + h) * D + 8 * j, x);
  if (norm) kv8_load8<T, false>(reinterpret_cast<const T*>(a.k_gain) + 8 * j, gain);
  if (which == 0)
    norm_rotate<D>(x, norm ? gain : nullptr, a.eps, a.tab + (size_t)row * pairs, a.rot, a.interleaved, j);
  top = wave_max_nan(top8(x, 0.f));
  const bool tamed = !is_finite(top);
  if (tamed) top = wave_max(tame8(x));
  const float now = fmaxf(was, scale_of<INT8>(top));
  if (tamed) clamp8<INT8>(x, now);
  const float inv = now > 0.f ? 1.0f / now : 0.f;
  if (lane == 0) *scale = now;
  if (g == 0) *reinterpret_cast<uint2*>(codes + (size_t)p0 * D + 8 * j) = encode8<INT8>(x, inv);
  if (now > was) rescale_old<D, INT8>(codes, p0, was * inv, lane, 64);
}

template <typename T, int D, bool INT8>
static hipError_t append_launch(int block, const Kv8AppendArgs& a, hipStream_t s) {
  constexpr int RPP = 4 * 64 / (D / 8);
  // heads per wave: four rounds where that leaves waves enough to fill the GPU
  // (16 per CU), else fewer
  constexpr int RPW = 64 / (D / 8);
  int hpw = 4 * RPW;
  while (hpw > RPW && (long)a.T * ((a.nh + hpw - 1) / hpw) < 256 * 16) hpw /= 2;
  const long per_row = (a.nh + hpw - 1) / hpw;
  const int q_blocks = (int)((a.T * per_row + 3) / 4);
  const int c_blocks = a.n_chunk * 2 * a.nkv;
  const int d_blocks = (int)(((long)(a.n_units - a.n_chunk) * 2 * a.nkv + 3) / 4);
  const dim3 grid(q_blocks + c_blocks + d_blocks);
  const int np = (block + RPP - 1) / RPP;
  if (np <= 1) hipLaunchKernelGGL((kv8_append_kernel<T, D, INT8, 1>), grid, dim3(256), 0, s, a, q_blocks, c_blocks, hpw);
  else if (np <= 2) hipLaunchKernelGGL((kv8_append_kernel<T, D, INT8, 2>), grid, dim3(256), 0, s, a, q_blocks, c_blocks, hpw);
  else if (np <= 4) hipLaunchKernelGGL((kv8_append_kernel<T, D, INT8, 4>), grid, dim3(256), 0, s, a, q_blocks, c_blocks, hpw);
  else if constexpr (D == 128) hipLaunchKernelGGL((kv8_append_kernel<T, D, INT8, 8>), grid, dim3(256), 0, s, a, q_blocks, c_blocks, hpw);
  else return hipErrorNotSupported;   // block 128 of head_dim 64 needs four passes
  return hipGetLastError();
}

hipError_t launch_kv8_append(int dtype, int format, int hd, int block, const Kv8AppendArgs& a, hipStream_t s) {
  const bool i8 = format == 0;
  if (dtype == 0) {
    if (hd == 128) return i8 ? append_launch<float, 128, true>(block, a, s) : append_launch<float, 128, false>(block, a, s);
    return i8 ? append_launch<float, 64, true>(block, a, s) : append_launch<float, 64, false>(block, a, s);
  }
  if (hd == 128) return i8 ? append_launch<bf16, 128, true>(block, a, s) : append_launch<bf16, 128, false>(block, a, s);
  return i8 ? append_launch<bf16, 64, true>(block, a, s) : append_launch<bf16, 64, false>(block, a, s);
}

// ------------------------------------------------------------------ read
// One thread per 16 codes of a (row, K or V, head); the rows leave past the
// caches (2048 positions of 52 heads, 82 MB: 16.5 us so, 20 otherwise).
template <typename T, bool INT8>
__global__ __launch_bounds__(256) void kv8_read_kernel(Kv8ReadArgs a) {
  const int per = a.hd / 16;
  const size_t t = blockIdx.x * (size_t)256 + threadIdx.x;
  const size_t row = t / (size_t)(2 * a.nkv * per);
  if (row >= (size_t)a.T) return;
  const int rest = (int)(t - row * (2 * a.nkv * per));
  const int which = rest / (a.nkv * per), h = rest / per % a.nkv, c = rest % per;
  T* out = reinterpret_cast<T*>(which ? a.v_out : a.k_out);
  if (!out) return;
  const int slot = a.row_slot[row], pos = a.row_pos[row];
  const uint4 w = *reinterpret_cast<const uint4*>(a.kv.codes + slot * a.kv.slot + which * a.kv.kv + h * a.kv.head +
                                                  (size_t)pos * a.hd + 16 * c);
  const float s = a.kv.scales[slot * a.kv.s_slot + which * a.kv.s_kv + h * a.kv.s_head + (pos >> a.kv.log2_block)];
  float x[16];
  decode4<INT8>(w.x, x);
  decode4<INT8>(w.y, x + 4);
  decode4<INT8>(w.z, x + 8);
  decode4<INT8>(w.w, x + 12);
#pragma unroll
  for (int e = 0; e < 16; ++e) x[e] *= s;
  T* dst = out + row * (which ? a.ld_v : a.ld_k) + (size_t)h * a.hd + 16 * c;
  kv8_store8<T, true>(dst, x);
  kv8_store8<T, true>(dst + 8, x + 8);
}

hipError_t launch_kv8_read(int out_dtype, int format, const Kv8ReadArgs& a, hipStream_t s) {
  const size_t n = (size_t)a.T * 2 * a.nkv * (a.hd / 16);
  const dim3 grid((unsigned)((n + 255) / 256));
  if (out_dtype == 0) {
    if (format == 0) hipLaunchKernelGGL((kv8_read_kernel<float, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((kv8_read_kernel<float, false>), grid, dim3(256), 0, s, a);
  } else {
    if (format == 0) hipLaunchKernelGGL((kv8_read_kernel<bf16, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((kv8_read_kernel<bf16, false>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace sarathi
