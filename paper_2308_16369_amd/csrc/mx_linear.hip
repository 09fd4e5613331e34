// Products of microscaled operands with the epilogues of the linear ops:
//   out = epilogue(sum_b 2^(sa_b + sw_b) sum_{k in block b} a_k w_k),
// on the matrix cores' scaled instruction, which takes both operands' codes and block scales.  Two kernels.  Up to 64 (128)
// rows the weights stream from memory into registers as fragments: bound by that stream (4 e4m3 rows of 15360 x 5120: 9.3 us
// a pass, 4.5 TB/s, of which 2 us are the launch).  More rows run as tiles fed through LDS: bound by the matrix cores and the
// power that they draw (the instruction alone, from registers, reaches 6.5 PFLOP/s of e2m1 on random codes, 8.8 on a single
// one; 4096 rows of 27648 x 5120 with SwiGLU run at 4.1 to 4.3, 267 to 284 us by the card and the length of the run), and for
// a few hundred rows by the chain of a stage (barrier, LDS reads, products) on one tile per CU.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "mx.h"
#include "sarathi_mx.h"

namespace sarathi {

constexpr int E2M1 = SARATHI_MX_E2M1, E4M3 = SARATHI_MX_E4M3;
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));

// One 32 x 32 x 64 product, W first: lane l holds W row l % 32 (x row l % 32), columns 32 (l / 32) .. + 31
// of the 64 in e2m1, and 16 (l / 32) .. + 15 of each 32 in e4m3; in either the scale of block l / 32 of its row, byte S
// of a dword.  The result holds column (x row) l % 32, rows (W rows) 8 g + 4 (l / 32) + i at 4 g + i.
//
// EXACT: the matrix cores add eight neighbouring products of e4m3 operands aligned to the largest, with 13 bits below
// it: a small product beside large ones that cancel is lost.  The codes of exponents 8 .. 15 and those of 0 .. 7 (bit 6 of a
// code) span 13 bits each beside e2m1's, so in two products these sums are exact.
template <int FMT, bool EXACT, int S>
__device__ __forceinline__ floatx16 mx_mfma(const u32x4& w, uint32_t ws, const u32x4* x, uint32_t xs, floatx16 c) {
  const i32x8 a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
  if constexpr (FMT == E2M1) {
    const i32x8 b = {(int)x[0][0], (int)x[0][1], (int)x[0][2], (int)x[0][3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, S, (int)ws, S, (int)xs);
  } else {
    i32x8 b;
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = (int)x[i / 4][i % 4];
    if constexpr (!EXACT) {
      return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 0, S, (int)ws, S, (int)xs);
    } else {
      i32x8 lo;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // 0xff in the bytes of the upper half: selectors 8 .. 11 repeat the top bits of bytes 1 and 3 of either operand
        const uint32_t u = (uint32_t)b[i], m = __builtin_amdgcn_perm(u << 9, u << 1, 0x090b080au);
        b[i] = (int)(u & m);
        lo[i] = (int)(u & ~m);
      }
      c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 0, S, (int)ws, S, (int)xs);
      return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, lo, c, 4, 0, S, (int)ws, S, (int)xs);
    }
  }
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pk_bf16(float a, float b) {   // nearest even; low half = a
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, bf16x2_t));
}

// silu(z) u with the hardware's reciprocal (a last place of fp32 off, where a division takes ten instructions).  It flushes
// subnormal results, which gates below -87.3 have, so it takes 2^-24 of its operand.
__device__ __forceinline__ float swiglu_f(float z, float u) {
  return z * (__builtin_amdgcn_rcpf(__builtin_fmaf(__expf(-z), 0x1p-24f, 0x1p-24f)) * 0x1p-24f) * u;
}

__device__ __forceinline__ bool adds_resid(const MxLinearArgs& p) {
  return p.kind == SARATHI_LINEAR_RESID || p.kind == SARATHI_LINEAR_RESID_F32IN;
}
// Four columns of a row of any N: the rows need not be aligned, the memory instructions take them so (one element at a
// time, 1956 rows of 4181 x 120 onto fp32 took 63 us).
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(4)));
// The residual at columns n .. n + 3 <= N - 1 of row m, as it lies in memory, and its values.
__device__ __forceinline__ bool resid_f32(const MxLinearArgs& p) {
  return p.dtype == SARATHI_F32 || p.kind == SARATHI_LINEAR_RESID_F32IN;
}
// Two pieces of eight bytes whatever the type (bf16: the same one twice): with a branch between the types' loads the compiler
// drains every request before each of the second type's (1955 rows of 6656 x 6656, e2m1, onto bf16: 67.7 us, 61.2 without).
__device__ __forceinline__ uint4 load_resid4(const MxLinearArgs& p, int m, int n) {
  const bool f32 = resid_f32(p);
  const char* r = reinterpret_cast<const char*>(p.resid) + (((size_t)m * p.N + n) << (f32 ? 2 : 1));
  const u32x2_any a = *reinterpret_cast<const u32x2_any*>(r), b = *reinterpret_cast<const u32x2_any*>(r + (f32 ? 8 : 0));
  return make_uint4(a[0], a[1], b[0], b[1]);
}
__device__ __forceinline__ float4 resid4(const MxLinearArgs& p, const uint4& r) {
  if (resid_f32(p)) return __builtin_bit_cast(float4, r);
  return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u), __uint_as_float(r.y << 16),
                     __uint_as_float(r.y & 0xffff0000u));
}
// Columns n .. n + 3 <= N - 1 of row m of the output, rounded to its type.
__device__ __forceinline__ void put4(const MxLinearArgs& p, int m, int n, const float4& v) {
  const size_t at = (size_t)m * p.N + n;
  if (p.dtype == SARATHI_F32 || p.kind == SARATHI_LINEAR_RESID)
    *reinterpret_cast<u32x4_any*>(reinterpret_cast<float*>(p.out) + at) = __builtin_bit_cast(u32x4, v);
  else
    *reinterpret_cast<u32x2_any*>(reinterpret_cast<bf16*>(p.out) + at) = u32x2_any{pk_bf16(v.x, v.y), pk_bf16(v.z, v.w)};
}
// The last columns of a row, fewer than four, with the residual added.
__device__ __forceinline__ void put_last(const MxLinearArgs& p, int m, int n, float4 v) {
#pragma unroll 1
  for (int i = 0; i < 4 && n + i < p.N; ++i) {
    const size_t at = (size_t)m * p.N + n + i;
    float z = v.x;
    v = make_float4(v.y, v.z, v.w, v.x);
    if (adds_resid(p))
      z += resid_f32(p)
               ? reinterpret_cast<const float*>(p.resid)[at]
               : bf2f(reinterpret_cast<const bf16*>(p.resid)[at]);
    if (p.dtype == SARATHI_F32 || p.kind == SARATHI_LINEAR_RESID) reinterpret_cast<float*>(p.out)[at] = z;
    else reinterpret_cast<bf16*>(p.out)[at] = f2bf(z);
  }
}
__device__ __forceinline__ float4 add4(const float4& a, const float4& b) {
  return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
}
// One such piece from sums v.
__device__ __forceinline__ void mx_store4(const MxLinearArgs& p, int m, int n, const float4& v) {
  if (m >= p.M || n >= p.N) return;
  if (n + 4 > p.N) put_last(p, m, n, v);
  else put4(p, m, n, adds_resid(p) ? add4(v, resid4(p, load_resid4(p, m, n))) : v);
}

// W tile t of a product's columns (SwiGLU: even ones are tiles of the gate, odd ones those of up): bytes from the first
// one's codes and scales.
__device__ __forceinline__ int w_tile(const MxLinearArgs& p, int t, size_t& up) {
  const int last = (p.N + 31) / 32 - 1;
  const bool glu = p.kind == SARATHI_LINEAR_SWIGLU;
  up = glu && (t & 1) ? p.up : 0;
  return min(glu ? t >> 1 : t, last);
}

template <int I, int N, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<I + 1, N>(f);
  }
}

// ============================================================================ few rows
// The weights stream once, from memory into registers, as fragments: FN W tiles to a block (SwiGLU: a gate tile and its up
// tile), all FM tiles of x (L2 holds them), NW waves each with every NW-th quad of columns, requested one quad ahead.  The
// waves' sums are joined through LDS in a fixed order, the upper half of the waves first.
template <int FMT, bool EXACT, int NW, int FN, int FM>
__global__ __launch_bounds__(64 * NW) void mx_stream_kernel(MxLinearArgs p) {
  constexpr int XU = FMT == E2M1 ? 1 : 2;             // 16-byte units of a lane per 64 columns
  constexpr int TILES = FN * FM;
  __shared__ float4 join[NW / 2 * TILES * 4 * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const u32x4* w[FN];
  const uint32_t* ws[FN];
#pragma unroll
  for (int f = 0; f < FN; ++f) {
    size_t up;
    const int t = w_tile(p, FN * blockIdx.x + f, up);
    w[f] = reinterpret_cast<const u32x4*>(p.w + up) + (size_t)t * p.quads * 256 + lane;
    ws[f] = reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(p.w_scale) + up) + (size_t)t * p.quads * 64 + lane;
  }
  const u32x4* x[FM];
  const uint32_t* xs[FM];
#pragma unroll
  for (int f = 0; f < FM; ++f) {
    const int at = (lane & 32) + min(lane & 31, p.M - 1 - f * 32);   // rows past the last: the last one's
    x[f] = reinterpret_cast<const u32x4*>(p.a) + (size_t)f * p.quads * 256 * XU + at;
    xs[f] = p.a_scale + (size_t)f * p.quads * 64 + at;
  }
  floatx16 acc[FN][FM];
#pragma unroll
  for (int f = 0; f < FN; ++f)
#pragma unroll
    for (int g = 0; g < FM; ++g)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[f][g][i] = 0.f;

  u32x4 wf[4][FN], xf[4][FM][XU];
  uint32_t wsc[2][FN], xsc[2][FM];
  auto load = [&](int q, int k) {
#pragma unroll
    for (int f = 0; f < FN; ++f) wf[k][f] = w[f][(size_t)q * 256 + k * 64];
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
      for (int u = 0; u < XU; ++u) xf[k][f][u] = x[f][((size_t)q * 4 + k) * 64 * XU + u * 64];
  };
  auto load_scales = [&](int q, int b) {
#pragma unroll
    for (int f = 0; f < FN; ++f) wsc[b][f] = ws[f][(size_t)q * 64];
#pragma unroll
    for (int f = 0; f < FM; ++f) xsc[b][f] = xs[f][(size_t)q * 64];
  };
  if (wave < p.quads) {
    load_scales(wave, 0);
#pragma unroll
    for (int k = 0; k < 4; ++k) load(wave, k);
    for (int q = wave; q < p.quads; q += NW) {
      const int next = min(q + NW, p.quads - 1);      // past the last: read again, not used
      load_scales(next, 1);
      static_for<0, 4>([&](auto kc) {
        constexpr int K = decltype(kc)::value;
#pragma unroll
        for (int f = 0; f < FN; ++f)
#pragma unroll
          for (int g = 0; g < FM; ++g)
            acc[f][g] = mx_mfma<FMT, EXACT, K>(wf[K][f], wsc[0][f], xf[K][g], xsc[0][g], acc[f][g]);
        load(next, K);
        __builtin_amdgcn_sched_barrier(0);
      });
#pragma unroll
      for (int f = 0; f < FN; ++f) wsc[0][f] = wsc[1][f];
#pragma unroll
      for (int f = 0; f < FM; ++f) xsc[0][f] = xsc[1][f];
    }
  }

  // join[wave of a half][tile, group of four][lane]
  auto put = [&](int at) {
#pragma unroll
    for (int f = 0; f < FN; ++f)
#pragma unroll
      for (int g = 0; g < FM; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          join[((at * TILES + f * FM + g) * 4 + i) * 64 + lane] =
              make_float4(acc[f][g][4 * i], acc[f][g][4 * i + 1], acc[f][g][4 * i + 2], acc[f][g][4 * i + 3]);
  };
  if (wave >= NW / 2) put(wave - NW / 2);
  __syncthreads();
  if (wave < NW / 2) {
#pragma unroll
    for (int f = 0; f < FN; ++f)
#pragma unroll
      for (int g = 0; g < FM; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 t = join[((wave * TILES + f * FM + g) * 4 + i) * 64 + lane];
          acc[f][g][4 * i] += t.x; acc[f][g][4 * i + 1] += t.y; acc[f][g][4 * i + 2] += t.z; acc[f][g][4 * i + 3] += t.w;
        }
    put(wave);                                        // where it has just read
  }
  __syncthreads();
  const bool glu = p.kind == SARATHI_LINEAR_SWIGLU;
  auto sum = [&](int part) {
    float4 v = join[part * 64 + lane];
#pragma unroll
    for (int h = 1; h < NW / 2; ++h) {
      const float4 t = join[(h * TILES * 4 + part) * 64 + lane];
      v = make_float4(v.x + t.x, v.y + t.y, v.z + t.z, v.w + t.w);
    }
    return v;
  };
  for (int part = wave; part < (glu ? FM * 4 : TILES * 4); part += NW) {   // 32 rows of x by eight W rows
    const int f = part / (FM * 4), g = part / 4 % FM, i = part % 4;
    float4 v = sum(part);
    if (glu) {
      const float4 u = sum(FM * 4 + part);
      v = make_float4(swiglu_f(v.x, u.x), swiglu_f(v.y, u.y), swiglu_f(v.z, u.z), swiglu_f(v.w, u.w));
    } else if (p.kind == SARATHI_LINEAR_GELU) {
      v = make_float4(gelu_f(v.x), gelu_f(v.y), gelu_f(v.z), gelu_f(v.w));
    }
    const int tile = glu ? (int)blockIdx.x : FN * (int)blockIdx.x + f;
    mx_store4(p, g * 32 + (lane & 31), tile * 32 + 8 * i + 4 * (lane >> 5), v);
  }
}

// ============================================================================ many rows
// WGN x WGM waves of FN W tiles by FM tiles of x; a block per CU runs its tiles one after the other.  A stage holds CS
// steps of 64 columns of a tile's operands, copied to LDS by DMA as they lie in memory: 1 KB per tile and step of e2m1, 2
// of e4m3, lane after lane as the instruction takes them, so reads are free of bank conflicts.  NS stages in a ring.  A
// wave multiplies a step while it reads the next one from LDS.  Before the products of a stage's last step:
//   wait for the next stage (and the reads of this one, which the step before ended with), barrier;
// then every wave has read stage s, so its place takes stage s + NS: requests run NS - 1 stages ahead, across the tiles
// of the block, so a tile starts with its operands there, and its output leaves while the next one's arrive.  Requests
// past the last stage re-read it into places that nothing reads.  The scales, a dword per lane, tile and 256 columns, go
// the same way (the compiler drains the DMA for any other load in the loop): requested four such quads ahead, before the
// stage's own requests, and read from LDS with the quad's first fragments.
//
// SwiGLU: W tiles come in pairs, gate and up.  With FN = 2 a wave has both of a pair; with FN = 1 it takes 16 rows of each
// as one fragment, so that either way a lane holds both sums of an output element.
template <int OFF>
__device__ __forceinline__ u32x4 lds_read16(uint32_t addr) {   // the compiler would wait for the DMA it may overlap
  u32x4 v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "i"(OFF));
  return v;
}
template <int OFF>
__device__ __forceinline__ void lds_write16(uint32_t addr, const u32x4& v) {
  asm volatile("ds_write_b128 %0, %1 offset:%2" ::"v"(addr), "v"(v), "i"(OFF) : "memory");
}
__device__ __forceinline__ uint32_t lds_read4(uint32_t addr) {
  uint32_t v;
  asm volatile("ds_read_b32 %0, %1" : "=v"(v) : "v"(addr));
  return v;
}
template <typename V, int N>
__device__ __forceinline__ void pin_regs(V (&r)[N]) {      // no use of r moves above this point
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+v"(r[i]));
}
template <int FMT, int WGN, int WGM, int FN, int FM>
struct MxTile {
  static constexpr int XU = FMT == E2M1 ? 1 : 2;
  static constexpr int TN = WGN * FN, TM = WGM * FM, NW = WGN * WGM;
  static constexpr int STEP = (TN + TM * XU) * 1024;                         // bytes
  // Large tiles gain from requests in small pieces; the smallest from fewer barriers (320 rows of 5120 x 5120, e2m1, 4 x 2
  // tiles: 15.5 us with four steps to a stage, 18.4 with one).
  static constexpr int CS = STEP <= 6 * 1024 ? 4 : 1, STAGE = CS * STEP, SPQ = 4 / CS;   // stages of a quad
  static constexpr int SCALES = (TN + TM) * 256, SR = 4;                     // of a quad; quads in the ring
  static constexpr int UNITS = STAGE / 1024, PER = (UNITS + NW - 1) / NW;    // 1 KB requests of a stage, of a wave
  static constexpr int SPER = (TN + TM + NW - 1) / NW;                       // requests of a quad's scales, of a wave
  static constexpr int PAD = 36;                                             // floats of a row of the epilogue's tile
  static constexpr int OUT = NW * 32 * PAD * 4;
  static constexpr int most(int a, int b) { return a < b ? a : b; }
  // Whole quads, so that a stage's place goes by its place in the quad (4 or 8).  In turn on one card: 4096 rows of 27648 x
  // 5120, e2m1, six stages 290 us, four 269 to 283; of 5120 x 13824, e4m3, 238 and 227.
  static constexpr int FIT = most(most((160 * 1024 - SR * SCALES - OUT) / STAGE, (56 - 3 * SPER) / PER), most(8, SR * SPQ));
  static constexpr int NS = FIT / 4 * 4;
  static constexpr int LDS = SR * SCALES + NS * STAGE + OUT;
  // requests of scales with the n stages before stage j of a quad (one with each quad's first, before the stage's own)
  static constexpr int scale_requests(int j, int n) { return j > 0 ? (n >= j ? (n - j) / SPQ + 1 : 0) : n / SPQ; }
};

template <int FMT, bool EXACT, bool GLU, int WGN, int WGM, int FN, int FM>
__global__ __launch_bounds__(64 * WGN * WGM, 1) void mx_tile_kernel(MxLinearArgs p, int tiles_m, int tiles_n, int splits) {
  using T = MxTile<FMT, WGN, WGM, FN, FM>;
  constexpr int XU = T::XU, TN = T::TN, TM = T::TM, NW = T::NW, NS = T::NS, CS = T::CS, STEP = T::STEP, STAGE = T::STAGE;
  constexpr int UNITS = T::UNITS, PER = T::PER, SPER = T::SPER, SR = T::SR;
  constexpr int NR = FN + FM * XU, NM = FN * FM;                             // LDS reads and products of a step
  static_assert(NS >= 3 && NS <= T::SPQ * SR, "ring");
  extern __shared__ uint4 lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = wave % WGN, wm = wave / WGN;

  // XCD-aware order: block b runs on XCD b % 8, each XCD takes consecutive tiles, its blocks in turn; eight x tiles by one
  // panel of W, then the next panel, so that what runs at once shares both
  const int n_tiles = tiles_m * tiles_n * splits, per = (n_tiles + 7) / 8, stride = gridDim.x / 8;
  const int t_first = (blockIdx.x % 8) * per + blockIdx.x / 8, t_end = min((int)(blockIdx.x % 8 + 1) * per, n_tiles);
  if (t_first >= t_end) return;
  struct Place {
    int tm, tn, split, q0, quads;                    // the tile, its share of the columns
  };
  auto place = [&](int t) {
    constexpr int GM = 8;
    Place a{0, 0, 0, 0, p.quads};
    if (splits > 1) {
      a.split = t / (tiles_m * tiles_n);
      t -= a.split * (tiles_m * tiles_n);
      a.q0 = p.quads * a.split / splits;
      a.quads = p.quads * (a.split + 1) / splits - a.q0;
    }
    const int group = tiles_m > GM ? t / (GM * tiles_n) : 0, gm = min(GM, tiles_m - group * GM);
    t -= group * (GM * tiles_n);
    a.tn = t / gm;
    a.tm = group * GM + t - a.tn * gm;
    return a;
  };

  // requests: unit j * NW + wave of a stage: [step][W tiles, then x tiles (e4m3: two units)]
  const char* src[PER];
  int r_tile = t_first - stride, r_quads = 0, r_slot = 0;
  auto aim = [&](int t) {                            // the requests' tile
    const Place a = place(t);
    r_quads = a.quads;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int u = min(j * NW + wave, UNITS - 1), k = u / (STEP / 1024), i = u % (STEP / 1024);
      if (i < TN) {
        size_t up;
        const int wt = w_tile(p, a.tn * TN + i, up);
        src[j] = p.w + up + ((size_t)wt * p.quads + a.q0) * 4096 + k * 1024;
      } else {
        const int xt = min(a.tm * TM + (i - TN) / XU, (p.M + 31) / 32 - 1);
        src[j] = p.a + ((size_t)xt * p.quads + a.q0) * 4096 * XU + (k * XU + (i - TN) % XU) * 1024;
      }
    }
  };
  auto request = [&](int j) {
    const int u = min(j * NW + wave, UNITS - 1);
    dma16(src[j] + lane * 16, lds + (SR * T::SCALES + r_slot * STAGE + u * 1024) / 16);
    src[j] += u % (STEP / 1024) < TN ? CS * 1024 : CS * 1024 * XU;
  };
  auto next_quad = [&]() {                           // before a quad's first request: the next tile's after a tile's last
    if (r_quads == 0) {
      if (r_tile + stride < t_end) r_tile += stride;
      aim(r_tile);
    }
    --r_quads;
  };
  const char* ssrc[SPER];
  int s_tile = t_first - stride, s_quads = 0, s_slot = 0;
  auto aim_scales = [&](int t) {
    const Place a = place(t);
    s_quads = a.quads;
#pragma unroll
    for (int j = 0; j < SPER; ++j) {
      const int u = min(j * NW + wave, TN + TM - 1);
      size_t up = 0;
      const int i = u < TN ? w_tile(p, a.tn * TN + u, up) : min(a.tm * TM + u - TN, (p.M + 31) / 32 - 1);
      ssrc[j] = reinterpret_cast<const char*>(u < TN ? p.w_scale : p.a_scale) + up + ((size_t)i * p.quads + a.q0) * 256;
    }
  };
  auto request_scales = [&]() {
    if (s_quads == 0) {
      if (s_tile + stride < t_end) s_tile += stride;
      aim_scales(s_tile);
    }
    --s_quads;
#pragma unroll
    for (int j = 0; j < SPER; ++j) {
      dma4(ssrc[j] + lane * 4, lds + (s_slot * T::SCALES + min(j * NW + wave, TN + TM - 1) * 256) / 16);
      ssrc[j] += 256;
    }
    s_slot = (s_slot + 1) % SR;
  };

  floatx16 acc[FN][FM];
  // this lane's place in the W tiles, in fragments of a tile (16 bytes of codes, 4 of scales), and in the x tiles
  const int wplace = FN == 1 && GLU ? ((wn & ~1) + (lane >> 4 & 1)) * 64 + (lane & 32) + (lane & 15) + 16 * (wn & 1)
                                    : wn * FN * 64 + lane;
  const int xplace = (TN + wm * FM * XU) * 64 + lane, xsplace = (TN + wm * FM) * 64 + lane;
  const uint32_t s0 = (uint32_t)(uintptr_t)lds, l0 = s0 + SR * T::SCALES;
  const uint32_t wl = l0 + wplace * 16, xl = l0 + xplace * 16;
  u32x4 fr[2][NR];                                   // fragments of a step: W, then x
  auto read = [&](auto buf, auto k, uint32_t at, auto r) {   // fragment r of step k of the stage at `at`
    constexpr int B = decltype(buf)::value, K = decltype(k)::value, R = decltype(r)::value;
    if constexpr (R < FN) fr[B][R] = lds_read16<K * STEP + R * 1024>(wl + at);
    else fr[B][R] = lds_read16<K * STEP + (R - FN) * 1024>(xl + at);
  };
  uint32_t sc[FN + FM], sc_next[FN + FM];            // the quad's scales: W, then x
  int sc_slot = 0;
  auto read_scales = [&](uint32_t* d) {
    const uint32_t b = s0 + sc_slot * T::SCALES;
#pragma unroll
    for (int f = 0; f < FN + FM; ++f) d[f] = lds_read4(b + (f < FN ? wplace + f * 64 : xsplace + (f - FN) * 64) * 4);
    sc_slot = (sc_slot + 1) % SR;
  };
  using C0 = std::integral_constant<int, 0>;
  using C1 = std::integral_constant<int, 1>;
  auto landed = [&]() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };

  // The loop's order, from stage -SPQ SR on: at stage s, requests of stage s + NS; at a quad's first, scales SR quads
  // ahead.  (Not unrolled: the copies' code, fetched once each, took 7 to 12 us of a launch.)
#pragma unroll 1
  for (int t = -T::SPQ * SR; t < 0; ++t) {
    if (t % T::SPQ == 0) request_scales();
    if (t < -NS) continue;
    if ((t + NS) % T::SPQ == 0) next_quad();
#pragma unroll
    for (int j = 0; j < PER; ++j) request(j);
    r_slot = r_slot + 1 == NS ? 0 : r_slot + 1;
  }
  wait_vmcnt<(NS - 1) * PER + (NS - 1) / T::SPQ * SPER>();   // quad 0's scales and stage 0
  lds_barrier();
  read_scales(sc);
  static_for<0, NR>([&](auto r) { read(C0{}, C0{}, 0, r); });
  landed();
  pin_regs(sc);
  pin_regs(fr[0]);

  int slot = 0;
  auto step = [&](auto jc) {                         // J of a quad's four
    constexpr int J = decltype(jc)::value, B = J & 1, SP = J / CS;   // the stage's place in its quad
    constexpr bool LAST = J % CS == CS - 1;
    const int next = slot + 1 == NS ? 0 : slot + 1;
    const uint32_t at = (LAST ? next : slot) * STAGE;
    if constexpr (LAST) {
      // the next stage: younger are the requests of NS - 2 stages, with those of scales before some
      wait_vmcnt<(NS - 2) * PER + T::scale_requests(SP, NS - 2) * SPER>();
      lds_barrier();
      if constexpr (SP == 0) request_scales();
      if constexpr ((SP + NS) % T::SPQ == 0) next_quad();
    }
    static_for<0, NM>([&](auto i) {
      constexpr int I = decltype(i)::value, fm = I / FN, fn = I % FN;
      acc[fn][fm] = mx_mfma<FMT, EXACT, J>(fr[B][fn], sc[fn], &fr[B][FN + fm * XU], sc[FN + fm], acc[fn][fm]);
      // the next step's reads in the first three quarters of the products, requests beside all of them
      constexpr int SPREAD = (NM * 3 + 3) / 4, R0 = I * NR / SPREAD, R1 = (I + 1) * NR / SPREAD;
      static_for<(R0 < NR ? R0 : NR), (R1 < NR ? R1 : NR)>([&](auto r) {
        read(std::integral_constant<int, 1 - B>{}, std::integral_constant<int, LAST ? 0 : J % CS + 1>{}, at, r);
      });
      if constexpr (LAST) static_for<I * PER / NM, (I + 1) * PER / NM>([&](auto j) { request(decltype(j)::value); });
      if constexpr (J == 3 && I == 0) read_scales(sc_next);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (LAST) slot = r_slot = next;          // the places run together
    landed();
    pin_regs(fr[1 - B]);
    if constexpr (J == 3) {
      pin_regs(sc_next);
#pragma unroll
      for (int f = 0; f < FN + FM; ++f) sc[f] = sc_next[f];
    }
  };

  const uint32_t out = (uint32_t)(uintptr_t)lds + SR * T::SCALES + NS * STAGE + wave * (32 * T::PAD * 4);
  for (int t = t_first; t < t_end; t += stride) {
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int j = 0; j < FM; ++j)
#pragma unroll
        for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.f;
    const Place at = place(t);
    for (int q = 0; q < at.quads; ++q) static_for<0, 4>([&](auto j) { step(j); });

    // The output: SwiGLU in place, then a piece of 32 rows by 32 (FN = 1, SwiGLU: 16) columns at a time through the
    // wave's part of LDS, so that it leaves in larger pieces of its rows.  One copy of the code that stores a piece: the
    // whole of it unrolled is fetched anew for every tile (10 to 20 thousand cycles).  LDS by hand here too, or the
    // compiler would wait for the stores of one piece before the next.
    constexpr int FO = GLU ? (FN + 1) / 2 : FN, PIECES = FO * FM;   // output tiles of the wave, side by side
    constexpr int W = FN == 1 && GLU ? 16 : 32, PR = 256 / W, ROWS = 32 / PR;   // columns of one; rows that leave at once
    if constexpr (GLU) {
#pragma unroll
      for (int g = 0; g < FM; ++g)
#pragma unroll
        for (int f = 0; f < FO; ++f)
#pragma unroll
          for (int k = 0; k < W / 2; ++k)
            acc[f][g][k] = FN == 1 ? swiglu_f(acc[0][g][k], acc[0][g][k + 8 & 15])
                                   : swiglu_f(acc[2 * f % FN][g][k], acc[(2 * f + 1) % FN][g][k]);
    }
    int le = threadIdx.x & 63;                       // the lane anew: what follows from it needs no register in the loop
    asm volatile("" : "+v"(le));
    const int r0 = le / (W / 4), c0 = le % (W / 4) * 4;
    const int m0 = (at.tm * TM + wm * FM) * 32 + r0, n0 = (at.tn * WGN + wn) * FO * W + c0;
    const uint32_t put_at = out + ((le & 31) * T::PAD + 4 * (le >> 5)) * 4, get_at = out + (r0 * T::PAD + c0) * 4;
    const bool add = !GLU && splits == 1 && adds_resid(p) && p.N >= 4;
    // The piece's residual, requested a piece ahead (1955 rows of 6656 x 6656, bf16 onto fp32, e2m1: 59 us, 69 without); the
    // 256 x 256 tiles of e4m3 rows with single products have no registers left for it.
    constexpr bool AHEAD = PIECES > 1 && (FMT == E2M1 || EXACT || PIECES < 8);
    uint4 raw[ROWS];
    auto fetch = [&](int piece) {
      const int m = m0 + piece / FO * 32, n = min(n0 + piece % FO * W, p.N - 4);
#pragma unroll
      for (int i = 0; i < ROWS; ++i) raw[i] = load_resid4(p, min(m + i * PR, p.M - 1), n);
    };
    if (AHEAD && add) fetch(0);
#pragma unroll 1
    for (int piece = 0; piece < PIECES; ++piece) {
      static_for<0, PIECES>([&](auto ic) {
        constexpr int I = decltype(ic)::value;
        if (piece != I) return;
        static_for<0, W / 8>([&](auto gc) {
          constexpr int G = decltype(gc)::value;
          const floatx16& a = acc[I % FO][I / FO];
          const float v[4] = {a[4 * G], a[4 * G + 1], a[4 * G + 2], a[4 * G + 3]};
          lds_write16<G * 32>(put_at, __builtin_bit_cast(u32x4, v));
        });
      });
      u32x4 v[ROWS];
      static_for<0, ROWS>([&](auto rc) { v[decltype(rc)::value] = lds_read16<decltype(rc)::value * PR * T::PAD * 4>(get_at); });
      landed();
      pin_regs(v);
      const int m = m0 + piece / FO * 32, n = n0 + piece % FO * W;
      if (add) {
        if (!AHEAD) fetch(piece);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
          const u32x4 y = __builtin_bit_cast(u32x4, add4(__builtin_bit_cast(float4, v[i]), resid4(p, raw[i])));
          if (n + 4 <= p.N) v[i] = y;
        }
        if (AHEAD && piece + 1 < PIECES) fetch(piece + 1);
      } else if (!GLU && splits == 1 && p.kind == SARATHI_LINEAR_GELU) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[i][e] = __float_as_uint(gelu_f(__uint_as_float(v[i][e])));
      }
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const int row = m + i * PR;
        if (row >= p.M || n >= p.N) continue;
        const float4 y = __builtin_bit_cast(float4, v[i]);
        if (!GLU && splits > 1) *reinterpret_cast<float4*>(p.parts + ((size_t)at.split * p.M + row) * mx_part_cols(p.N) + n) = y;
        else if (n + 4 > p.N) put_last(p, row, n, y);
        else put4(p, row, n, y);
      }
    }
  }
  wait_vmcnt<0>();                                   // requests past the last tile still fill the stages
}

// The partial sums of `splits` shares of the columns, added in order; four columns to a thread.
__global__ __launch_bounds__(256) void mx_join_kernel(MxLinearArgs p, int splits) {
  const size_t cols = mx_part_cols(p.N);
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, size = (size_t)p.M * cols;
  if (i * 4 >= size) return;
  float4 v = reinterpret_cast<const float4*>(p.parts)[i];
  for (int s = 1; s < splits; ++s) {
    const float4 t = *reinterpret_cast<const float4*>(p.parts + s * size + i * 4);
    v = make_float4(v.x + t.x, v.y + t.y, v.z + t.z, v.w + t.w);
  }
  if (p.kind == SARATHI_LINEAR_GELU) v = make_float4(gelu_f(v.x), gelu_f(v.y), gelu_f(v.z), gelu_f(v.w));
  mx_store4(p, (int)(i * 4 / cols), (int)(i * 4 % cols), v);
}

// Most that split columns can use: at most 256 tiles run, of 64 K output elements at most; eight splits.
constexpr int MX_MAX_SPLITS = 8;
size_t mx_linear_parts(int M, int N) {
  if (M <= 2 * MX_ROWS) return 0;
  return std::min((size_t)MX_MAX_SPLITS * M * mx_part_cols(N), (size_t)256 * 65536);
}

template <int FMT, bool EXACT, bool GLU, int WGN, int WGM, int FN, int FM>
static hipError_t run_tile_as(const MxLinearArgs& a, int splits, hipStream_t s) {
  using T = MxTile<FMT, WGN, WGM, FN, FM>;
  const auto kernel = mx_tile_kernel<FMT, EXACT, GLU, WGN, WGM, FN, FM>;
  static_assert(T::LDS <= 160 * 1024, "LDS of a CU");
  static std::atomic<uint64_t> lds_set{0};           // devices on which this instance's LDS limit is raised
  hipError_t e = ensure_dynamic_lds((const void*)kernel, T::LDS, lds_set);
  if (e != hipSuccess) return e;
  const int w_tiles = (GLU ? 2 : 1) * mx_tiles(a.N);
  const int tiles_n = (w_tiles + T::TN - 1) / T::TN, tiles_m = (mx_tiles(a.M) + T::TM - 1) / T::TM;
  const int grid = std::min((tiles_n * tiles_m * splits + 7) / 8 * 8, 256);   // a block per CU
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(64 * T::NW), T::LDS, s, a, tiles_m, tiles_n, splits);
  e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  hipLaunchKernelGGL(mx_join_kernel, dim3((unsigned)(((size_t)a.M * mx_part_cols(a.N) / 4 + 255) / 256)), dim3(256), 0, s, a, splits);
  return hipGetLastError();
}

template <int FMT, bool EXACT, int WGN, int WGM, int FN, int FM>
static hipError_t run_tile(const MxLinearArgs& a, int splits, hipStream_t s, MxLinearPlan* plan) {
  if (plan) {
    *plan = {WGM * FM * MX_ROWS, WGN * FN * MX_ROWS, splits};
    return hipSuccess;
  }
  return a.kind == SARATHI_LINEAR_SWIGLU ? run_tile_as<FMT, EXACT, true, WGN, WGM, FN, FM>(a, 1, s)
                                         : run_tile_as<FMT, EXACT, false, WGN, WGM, FN, FM>(a, splits, s);
}

template <int FMT, bool EXACT, int NW, int FN, int FM>
static hipError_t run_stream(const MxLinearArgs& a, hipStream_t s, MxLinearPlan* plan) {
  if (plan) {
    *plan = {FM * MX_ROWS, FN * MX_ROWS, 1};
    return hipSuccess;
  }
  const int w_tiles = (a.kind == SARATHI_LINEAR_SWIGLU ? 2 : 1) * mx_tiles(a.N);
  hipLaunchKernelGGL((mx_stream_kernel<FMT, EXACT, NW, FN, FM>), dim3((w_tiles + FN - 1) / FN), dim3(64 * NW), 0, s, a);
  return hipGetLastError();
}

// The tiles of the second kernel (W tiles by x tiles) and what 64 columns of one cost with every CU busy, in us (on one card,
// others differ by 5 %; from 4096 rows of 13824 x 5120, a round of one tile per CU: e2m1 12.1, 15.5, 27, 28, 31, 37 us in the order below, e4m3 14.5, 20.5,
// 31, 39.6 and 53.7, with exact sums 22, 33, 52 and 97; 2.5 of them the output's).  0: not built, another tile is
// faster everywhere (the split of an x fragment for exact sums is shared by FN W tiles).  Where tiles leave CUs idle, the
// columns are split: shorter tiles, but the partial sums are written and read back, and a launch of their own joins them.
struct TileCost {
  int tn, tm;
  float e2m1, e4m3, exact;
};
constexpr TileCost kTiles[] = {{4, 2, 0.120f, 0.150f, 0.245f}, {4, 4, 0.160f, 0.225f, 0.385f}, {8, 4, 0.305f, 0.36f, 0.62f},
                               {4, 10, 0.32f, 0.465f, 0},      {8, 6, 0.355f, 0, 0},          {8, 8, 0.43f, 0.64f, 1.18f}};

struct TilePick {
  int tile, splits;
};
static TilePick pick_tile(const MxLinearArgs& a, int w_tiles, int x_tiles, int format, bool exact) {
  TilePick best{0, 1};
  float least = INFINITY;
  const size_t size = (size_t)a.M * mx_part_cols(a.N);
  // (partial sums of SwiGLU would be two for each output, and its W tiles are many)
  const bool can_split = a.parts && a.kind != SARATHI_LINEAR_SWIGLU;
  for (int i = 0; i < (int)(sizeof(kTiles) / sizeof(kTiles[0])); ++i) {
    const TileCost& t = kTiles[i];
    const float cost = exact ? t.exact : format == E2M1 ? t.e2m1 : t.e4m3;
    if (cost == 0) continue;
    const long tiles = (long)((w_tiles + t.tn - 1) / t.tn) * ((x_tiles + t.tm - 1) / t.tm);
    for (int n = 1; n <= MX_MAX_SPLITS; ++n) {
      if (n > 1 && (!can_split || n * tiles > 256 || a.quads < 4 * n || n * size > a.parts_cap)) break;
      float us = (float)((tiles * n + 255) / 256) * (2.5f + ((a.quads + n - 1) / n) * 4 * cost);
      if (n > 1) us += 4.0f + n * size * 8e-6f / 5.0f;   // the launch; partial sums written and read, 5 TB/s
      if (us < least) least = us, best = {i, n};
    }
  }
  return best;
}

template <int FMT, bool EXACT>
static hipError_t linear_as(const MxLinearArgs& a, hipStream_t s, MxLinearPlan* plan) {
  const bool glu = a.kind == SARATHI_LINEAR_SWIGLU;
  const int x_tiles = mx_tiles(a.M), w_tiles = (glu ? 2 : 1) * mx_tiles(a.N);
  // Up to 64 rows stream; up to 128 where the W tiles would leave CUs idle in the other kernel (128 rows of 5120 x 5120,
  // e4m3: 12.3 us, 14.2 there; 96 rows of 5120 x 4096 9.4 and 12.8), but not where it splits many columns of few W tiles (128
  // rows of 2600 x 13824: e4m3 23.3 us streamed, 15.9 split; e2m1 15.5 and 15.0).
  const bool few = w_tiles <= 256, many = a.quads * (long)x_tiles > (FMT == E2M1 ? 170 : 110);
  const TilePick pick = pick_tile(a, w_tiles, x_tiles, FMT, EXACT);
  const bool split = few && many && pick.splits > 1;
  if (x_tiles <= 2 || (x_tiles <= 4 && few && !split)) {
    // Up to 64 rows the sums of eight are exact whatever the output's type.  The weights' stream hides most of the second
    // products: onto bf16, 4 rows of 15360 x 5120 take 9.6 us (11.0 with single ones), of 2 x 13824 x 5120 with SwiGLU 15.6
    // (14.4), 64 rows of the two 17.1 (15.9) and 23.8 (21.7); most is lost where few blocks split many columns' x: 48 rows of
    // 5120 x 13824 17.0 (13.8).  In the other kernel exact sums take 1.7 to 2.4 times as long.
    constexpr bool SUMS = FMT == E4M3;
    switch (x_tiles) {
      case 1:
        if (glu) return run_stream<FMT, SUMS, 8, 2, 1>(a, s, plan);
        return w_tiles <= 256 ? run_stream<FMT, SUMS, 16, 1, 1>(a, s, plan) : run_stream<FMT, SUMS, 8, 1, 1>(a, s, plan);
      case 2:
        if (glu) return run_stream<FMT, SUMS, 8, 2, 2>(a, s, plan);
        if constexpr (FMT == E2M1)                    // (e4m3: the registers of 16 waves do not hold a quad)
          if (w_tiles <= 256) return run_stream<FMT, SUMS, 16, 1, 2>(a, s, plan);
        return run_stream<FMT, SUMS, 8, 1, 2>(a, s, plan);
      case 3: return glu ? run_stream<FMT, EXACT, 4, 2, 3>(a, s, plan) : run_stream<FMT, EXACT, 8, 1, 3>(a, s, plan);
      default: return glu ? run_stream<FMT, EXACT, 4, 2, 4>(a, s, plan) : run_stream<FMT, EXACT, 4, 1, 4>(a, s, plan);
    }
  }
  switch (pick.tile) {
    case 0: return run_tile<FMT, EXACT, 4, 2, 1, 1>(a, pick.splits, s, plan);
    case 1: return run_tile<FMT, EXACT, 2, 4, 2, 1>(a, pick.splits, s, plan);
    case 2: return run_tile<FMT, EXACT, 2, 4, 4, 1>(a, pick.splits, s, plan);
    case 3:
      if constexpr (!EXACT) return run_tile<FMT, EXACT, 4, 2, 1, 5>(a, pick.splits, s, plan);
    case 4:
      if constexpr (FMT == E2M1) return run_tile<FMT, EXACT, 4, 2, 2, 3>(a, pick.splits, s, plan);
    default: return run_tile<FMT, EXACT, 2, 4, 4, 2>(a, pick.splits, s, plan);
  }
}

hipError_t launch_mx_linear(int a_format, const MxLinearArgs& a, hipStream_t s, MxLinearPlan* plan) {
  const bool f32_out = a.dtype == SARATHI_F32 || a.kind == SARATHI_LINEAR_RESID;
  if (a_format == E2M1) return linear_as<E2M1, false>(a, s, plan);
  return f32_out ? linear_as<E4M3, true>(a, s, plan) : linear_as<E4M3, false>(a, s, plan);
}

}  // namespace sarathi
