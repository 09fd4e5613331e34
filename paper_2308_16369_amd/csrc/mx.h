// Microscaled operands: their layout in memory and the launches of their
// operators.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace sarathi {

constexpr int MX_ROWS = 32;     // rows of a tile: those of a matrix instruction
constexpr int MX_COLS = 256;    // columns are padded to these: a dword of scales per row and parity of the block
constexpr int MX_BLOCK = 32;    // elements of a scale
constexpr int MX_NORM_COLS = 24576;

inline int mx_tiles(int rows) { return (int)(((long)rows + MX_ROWS - 1) / MX_ROWS); }
inline int mx_quads(int cols) { return (int)(((long)cols + MX_COLS - 1) / MX_COLS); }
// codes of one row tile: 32 rows of 128 (e2m1) or 256 bytes per 256 columns
inline size_t mx_tile_bytes(int format, int cols) { return (size_t)mx_quads(cols) * MX_ROWS * (format ? 256 : 128); }
// columns of partial sums: rows of whole float4
__host__ __device__ inline size_t mx_part_cols(int N) { return ((size_t)N + 3) & ~(size_t)3; }
inline size_t mx_scale_offset(int format, int rows, int cols) { return mx_tiles(rows) * mx_tile_bytes(format, cols); }
inline size_t mx_bytes(int format, int rows, int cols) {
  return mx_scale_offset(format, rows, cols) + (size_t)mx_tiles(rows) * mx_quads(cols) * 256;
}

struct MxQuantArgs {
  int rows, cols;
  const void* x;      // dequantise: the output
  size_t ld;
  char* operand;
};
hipError_t launch_mx_quantize(int dtype, int format, const MxQuantArgs& a, hipStream_t s);
hipError_t launch_mx_dequantize(int dtype, int format, const MxQuantArgs& a, hipStream_t s);

struct MxNormArgs {
  int rows, cols;
  float eps;
  const void* x;
  const void* delta;   // or NULL
  const void* gain;
  void* h;             // or NULL
  size_t ld_x, ld_delta, ld_h;
  char* operand;
};
hipError_t launch_mx_norm(int stream_dtype, int dtype, int format, const MxNormArgs& a, hipStream_t s);

struct MxLinearArgs {
  int kind;
  int dtype;
  int M, N, quads;         // quads: 256 columns each
  const char* a;           // codes
  const char* w;
  const uint32_t* a_scale;
  const uint32_t* w_scale;
  size_t up;               // SwiGLU: bytes from gate to up, codes and scales alike
  const void* resid;
  void* out;
  float* parts;            // [split][M][mx_part_cols(N)], or NULL
  size_t parts_cap;        // floats
};
struct MxLinearPlan {
  int bm, bn, splits;      // rows of x and W rows of a block, shares of the columns
};
// With `plan`, nothing is launched: what would run.
hipError_t launch_mx_linear(int a_format, const MxLinearArgs& a, hipStream_t s, MxLinearPlan* plan = nullptr);
size_t mx_linear_parts(int M, int N);   // floats that the launch can use

}  // namespace sarathi
