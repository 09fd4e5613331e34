// Microscaled operands: quantise, dequantise, and the norm that writes one.
//
// A block of 32 elements with the largest magnitude m takes the scale 2^e, the
// smallest power of two with top 2^e >= m (top 6 or 448): the exponent of m,
// less that of top, plus one where m's mantissa passes top's.  Dividing by it is
// exact, so a code is the element itself rounded once.
//
// Eight elements to a lane, four lanes to a block; the largest magnitude is
// taken over the bit patterns, which puts infinities and NaN above every
// number.  Both ways are bound by the rows in memory (27648 x 5120 of bf16 to e2m1
// and back, one after the other: 152 us for 641 MB, 4.2 TB/s, where a copy reaches
// 4.7; either alone, over and over: 70 and 77 us, 5.1 and 4.6 TB/s, a copy 5.4).
#include <type_traits>

#include "common.h"
#include "mx.h"
#include "sarathi_mx.h"

namespace sarathi {

constexpr int E2M1 = SARATHI_MX_E2M1, E4M3 = SARATHI_MX_E4M3;

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t top_bits) {
  constexpr uint32_t OVER = FMT == E2M1 ? 0x3fffffu : 0x1fffffu;   // carries where the mantissa passes 1.5 (1.75)
  constexpr int EXP = FMT == E2M1 ? 2 : 8;
  const int e = (int)((top_bits + OVER) >> 23) - EXP;
  return top_bits >= 0x7f800000u ? 255u : (uint32_t)max(e, 0);
}

// The largest magnitude's bits of the 32 elements that this lane and its three neighbours hold.
__device__ __forceinline__ uint32_t block_top(const float* v) {
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(v[i]) & 0x7fffffffu);
  t = max(t, (uint32_t)__shfl_xor((int)t, 1, 64));
  return max(t, (uint32_t)__shfl_xor((int)t, 2, 64));
}

// The codes of a lane's eight elements (the conversion takes the scale's exponent field, so byte 0 is 2^-127).
__device__ __forceinline__ uint32_t codes_e2m1(const float* v, uint32_t byte) {
  const float s = __uint_as_float(byte << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
  return byte == 255u ? 0u : c;
}
__device__ __forceinline__ uint2 codes_e4m3(const float* v, uint32_t byte) {
  const float s = __uint_as_float(byte << 23);
  s16x2 a = {0, 0}, b = {0, 0};
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, v[0], v[1], s, false);
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, v[2], v[3], s, true);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, v[4], v[5], s, false);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, v[6], v[7], s, true);
  return byte == 255u ? make_uint2(0, 0) : make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
}

// Eight elements of columns 8 c .. (c counts within a row, padding included) of row r of a tile.
// `tile`: its codes; `scales`: its scales.  Every lane of the eight blocks of 256 columns takes part.
template <int FMT>
__device__ __forceinline__ void put8(char* tile, uint32_t* scales, int r, int c, const float* v, bool row_ok) {
  const uint32_t byte = scale_byte<FMT>(block_top(v));
  const int b = c >> 2;
  // bytes of the blocks of one parity into a dword: those of lanes 8, 16 and 24 away
  uint32_t word = byte << (8 * ((b & 7) >> 1));
  word |= (uint32_t)__shfl_xor((int)word, 8, 64);
  word |= (uint32_t)__shfl_xor((int)word, 16, 64);
  if (!row_ok) return;
  if constexpr (FMT == E2M1) {
    *reinterpret_cast<uint32_t*>(tile + ((size_t)b * 32 + r) * 16 + (c & 3) * 4) = codes_e2m1(v, byte);
  } else {
    *reinterpret_cast<uint2*>(tile + ((size_t)(c >> 1) * 32 + r) * 16 + (c & 1) * 8) = codes_e4m3(v, byte);
  }
  if ((c & 27) == 0) scales[((c >> 5) * 2 + (b & 1)) * 32 + r] = word;   // c % 32 is 0 or 4
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* v) {
#pragma unroll
  for (int o = 0; o < 8; o += Vec16<T>::N) Vec16<T>::unpack(*reinterpret_cast<const uint4*>(p + o), v + o);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* v);
template <> __device__ __forceinline__ void store8<float>(float* p, const float* v) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
template <> __device__ __forceinline__ void store8<bf16>(bf16* p, const float* v) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f2bf(v[2 * i]) | ((uint32_t)f2bf(v[2 * i + 1]) << 16);
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// ------------------------------------------------------------------ quantise, dequantise
// A block of four waves takes 32 rows of 256 columns; a wave two rows at a time, each read in one piece.
template <typename T, int FMT>
__global__ __launch_bounds__(256) void mx_quantize_kernel(MxQuantArgs a, int quads, size_t scale_offset) {
  const int quad = blockIdx.x % quads, tile = blockIdx.x / quads;
  const int c = threadIdx.x & 31, r0 = threadIdx.x >> 5;
  char* codes = a.operand + ((size_t)tile * quads + quad) * (32 * (FMT == E2M1 ? 128 : 256));
  uint32_t* scales = reinterpret_cast<uint32_t*>(a.operand + scale_offset) + ((size_t)tile * quads + quad) * 64;
  const int col = quad * MX_COLS + c * 8;
  const T* x = reinterpret_cast<const T*>(a.x) + (size_t)tile * 32 * a.ld + col;
  const int rows = min(32, a.rows - tile * 32);
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const int r = it * 8 + r0;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (r < rows && col < a.cols) load8(x + (size_t)r * a.ld, v);
    put8<FMT>(codes, scales, r, c, v, r < rows);
  }
}

template <typename T, int FMT>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(MxQuantArgs a, int quads, size_t scale_offset) {
  const int quad = blockIdx.x % quads, tile = blockIdx.x / quads;
  const int c = threadIdx.x & 31, r0 = threadIdx.x >> 5, b = c >> 2;
  const char* codes = a.operand + ((size_t)tile * quads + quad) * (32 * (FMT == E2M1 ? 128 : 256));
  const uint8_t* scales = reinterpret_cast<const uint8_t*>(a.operand + scale_offset) + ((size_t)tile * quads + quad) * 256;
  const int col = quad * MX_COLS + c * 8;
  if (col >= a.cols) return;
  T* out = reinterpret_cast<T*>(const_cast<void*>(a.x)) + (size_t)tile * 32 * a.ld + col;
  const int rows = min(32, a.rows - tile * 32);
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    const int r = it * 8 + r0;
    if (r >= rows) break;
    const uint32_t byte = scales[((b & 1) * 32 + r) * 4 + (b >> 1)];
    const float s = __uint_as_float(byte << 23);
    float v[8];
    f32x2 t;
    if constexpr (FMT == E2M1) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + (b * 32 + r) * 16 + (c & 3) * 4);
      t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 0); v[0] = t[0]; v[1] = t[1];
      t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 1); v[2] = t[0]; v[3] = t[1];
      t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 2); v[4] = t[0]; v[5] = t[1];
      t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, 3); v[6] = t[0]; v[7] = t[1];
    } else {
      const uint2 w = *reinterpret_cast<const uint2*>(codes + ((c >> 1) * 32 + r) * 16 + (c & 1) * 8);
      t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, s, false); v[0] = t[0]; v[1] = t[1];
      t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, s, true); v[2] = t[0]; v[3] = t[1];
      t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, s, false); v[4] = t[0]; v[5] = t[1];
      t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, s, true); v[6] = t[0]; v[7] = t[1];
    }
    if (byte == 255u) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(0x7fc00000u);
    }
    store8(out + (size_t)r * a.ld, v);
  }
}

template <typename T>
static hipError_t quantize_as(int format, const MxQuantArgs& a, hipStream_t s) {
  const int quads = mx_quads(a.cols), grid = quads * mx_tiles(a.rows);
  const size_t at = mx_scale_offset(format, a.rows, a.cols);
  if (format == E2M1) hipLaunchKernelGGL((mx_quantize_kernel<T, E2M1>), dim3(grid), dim3(256), 0, s, a, quads, at);
  else hipLaunchKernelGGL((mx_quantize_kernel<T, E4M3>), dim3(grid), dim3(256), 0, s, a, quads, at);
  return hipGetLastError();
}
hipError_t launch_mx_quantize(int dtype, int format, const MxQuantArgs& a, hipStream_t s) {
  return dtype == SARATHI_BF16 ? quantize_as<bf16>(format, a, s) : quantize_as<float>(format, a, s);
}

template <typename T>
static hipError_t dequantize_as(int format, const MxQuantArgs& a, hipStream_t s) {
  const int quads = mx_quads(a.cols), grid = quads * mx_tiles(a.rows);
  const size_t at = mx_scale_offset(format, a.rows, a.cols);
  if (format == E2M1) hipLaunchKernelGGL((mx_dequantize_kernel<T, E2M1>), dim3(grid), dim3(256), 0, s, a, quads, at);
  else hipLaunchKernelGGL((mx_dequantize_kernel<T, E4M3>), dim3(grid), dim3(256), 0, s, a, quads, at);
  return hipGetLastError();
}
hipError_t launch_mx_dequantize(int dtype, int format, const MxQuantArgs& a, hipStream_t s) {
  return dtype == SARATHI_BF16 ? dequantize_as<bf16>(format, a, s) : dequantize_as<float>(format, a, s);
}

// ------------------------------------------------------------------ norm
// One row per block, read once and kept in registers (eight elements to a lane,
// NC times).  Squares are added in fp64.  An element's fp32 value y = h r g (h = x +
// delta, r = 1 / sqrt(mean + eps)) carries four roundings, 2^-22 of it: up to four
// units in the last place.  Every border of two codes or scales has its low 19 bits
// zero, so one element in 60000 lies within four units of one; those are taken again
// in fp64, from x and delta as they are, and rounded to odd, so that a code is that of
// the value in 64 bits.  (Without it one element in a million takes a border's other
// side.)
// Bound by the rows, x and delta read, h and e4m3 codes written: 2048 x 12288 of
// bf16, 177 MB, in 47.5 us from memory (3.7 TB/s), 37.4 over and over (4.7 TB/s); the
// sum and the squares in fp64 are 2 of them.
//
// A row's output is 16-byte pieces 512 bytes apart, so the 32 rows of a tile
// run on one XCD, one after the other, and their pieces meet in its L2 before
// they leave it as whole lines.
template <typename T> struct Raw8 {   // eight elements as they lie in memory
  uint4 u[8 / Vec16<T>::N];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < 8 / Vec16<T>::N; ++i) u[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ float at(int e) const {
    const uint4& w = u[e / Vec16<T>::N];
    const int i = e % Vec16<T>::N / (sizeof(T) == 2 ? 2 : 1);
    const uint32_t b = i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
    return __uint_as_float(sizeof(T) == 4 ? b : e & 1 ? b & 0xffff0000u : b << 16);
  }
  // The compiler keeps nothing that was made of them (bf16: 10 registers of 72).
  __device__ __forceinline__ void anew() {
    if constexpr (sizeof(T) == 2) asm volatile("" : "+v"(u[0].x), "+v"(u[0].y), "+v"(u[0].z), "+v"(u[0].w));
  }
  __device__ __forceinline__ void clear() {   // -0, so that a sum is the other number
    constexpr uint32_t Z = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
#pragma unroll
    for (int i = 0; i < 8 / Vec16<T>::N; ++i) u[i] = make_uint4(Z, Z, Z, Z);
  }
};

// y to the nearest fp32 number or, where that is even and not y, to its neighbour on y's side.
__device__ __forceinline__ float round_odd(double y) {
  const float f = (float)y;
  const uint32_t u = __float_as_uint(f);
  const bool keep = (u & 1u) || (double)f == y || !(fabsf(f) < __uint_as_float(0x7f800000u));
  return keep ? f : __uint_as_float(fabs((double)f) < fabs(y) ? u + 1 : u - 1);
}

template <typename TS, typename T, int FMT, int NC>
__global__ __launch_bounds__(256) void mx_norm_kernel(MxNormArgs a, int quads, size_t scale_offset) {
  __shared__ double red[4];
  const int i = blockIdx.x / 8, tile = (i / 32) * 8 + blockIdx.x % 8, r = i % 32;
  const size_t row = (size_t)tile * 32 + r;
  if (row >= (size_t)a.rows) return;
  const TS* x = reinterpret_cast<const TS*>(a.x) + row * a.ld_x;
  const T* d = reinterpret_cast<const T*>(a.delta) + row * a.ld_delta;
  Raw8<TS> xr[NC];
  Raw8<T> dr[NC], g[NC];
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int col = (threadIdx.x + 256 * j) * 8;
    if (col >= a.cols) continue;
    xr[j].load(x + col);
    if (a.delta) dr[j].load(d + col);
    else dr[j].clear();
  }
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int col = (threadIdx.x + 256 * j) * 8;
    if (col < a.cols) g[j].load(reinterpret_cast<const T*>(a.gain) + col);
  }
  double ss = 0;
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int col = (threadIdx.x + 256 * j) * 8;
    if (col >= a.cols) continue;
    float h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      h[e] = xr[j].at(e) + dr[j].at(e);
      const double sum = (double)xr[j].at(e) + (double)dr[j].at(e);
      ss += sum * sum;
    }
    if (a.h) store8(reinterpret_cast<TS*>(a.h) + row * a.ld_h + col, h);
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) ss += __shfl_xor(ss, m, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
  __syncthreads();
  ss = red[0] + red[1] + red[2] + red[3];
  const double rs = 1.0 / sqrt(ss / a.cols + (double)a.eps);
  const float r32 = (float)rs;
  const uint32_t sure = r32 >= 0x1p-126f ? ~0u : 0u;   // 0: r is no normal number of fp32
  const float low = ss > 0 ? 0x1p-100f : -1.f;         // below: h r or a block of y may have lost bits (not in rows of zeros)
  char* codes = a.operand + (size_t)tile * quads * (32 * (FMT == E2M1 ? 128 : 256));
  uint32_t* scales = reinterpret_cast<uint32_t*>(a.operand + scale_offset) + (size_t)tile * quads * 64;
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int c = threadIdx.x + 256 * j;
    if (c >= quads * 32) continue;                  // whole groups of 32 lanes
    float y[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};   // padding, also in a row of NaN
    if (c * 8 < a.cols) {
      uint32_t off = sure;
      float least = INFINITY, most = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float t = (xr[j].at(e) + dr[j].at(e)) * r32;
        y[e] = t * g[j].at(e);
        least = fminf(least, fabsf(t));
        most = fmaxf(most, fabsf(y[e]));
        off = min(off, (__float_as_uint(y[e]) + 4) & 0x7ffffu);
      }
      if (off <= 8 || least < low || most < low) {
        xr[j].anew(), dr[j].anew(), g[j].anew();
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = round_odd(((double)xr[j].at(e) + (double)dr[j].at(e)) * rs * (double)g[j].at(e));
      }
    }
    put8<FMT>(codes, scales, r, c, y, true);
  }
}

template <typename TS, typename T, int FMT>
static hipError_t norm_as(const MxNormArgs& a, hipStream_t s) {
  const int quads = mx_quads(a.cols), nc = (quads * 32 + 255) / 256;
  const size_t at = mx_scale_offset(FMT, a.rows, a.cols);
  const dim3 grid((mx_tiles(a.rows) + 7) / 8 * 256);
  auto run = [&](auto n) {
    hipLaunchKernelGGL((mx_norm_kernel<TS, T, FMT, decltype(n)::value>), grid, dim3(256), 0, s, a, quads, at);
  };
  if (nc <= 1) run(std::integral_constant<int, 1>{});
  else if (nc <= 2) run(std::integral_constant<int, 2>{});
  else if (nc <= 3) run(std::integral_constant<int, 3>{});
  else if (nc <= 4) run(std::integral_constant<int, 4>{});
  else if (nc <= 6) run(std::integral_constant<int, 6>{});
  else if (nc <= 8) run(std::integral_constant<int, 8>{});
  else run(std::integral_constant<int, 12>{});
  return hipGetLastError();
}
template <typename TS, typename T>
static hipError_t norm_of(int format, const MxNormArgs& a, hipStream_t s) {
  return format == E2M1 ? norm_as<TS, T, E2M1>(a, s) : norm_as<TS, T, E4M3>(a, s);
}
hipError_t launch_mx_norm(int stream_dtype, int dtype, int format, const MxNormArgs& a, hipStream_t s) {
  if (stream_dtype == SARATHI_BF16) return norm_of<bf16, bf16>(format, a, s);
  return dtype == SARATHI_BF16 ? norm_of<float, bf16>(format, a, s) : norm_of<float, float>(format, a, s);
}

}  // namespace sarathi
