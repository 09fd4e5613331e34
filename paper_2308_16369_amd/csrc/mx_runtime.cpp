// Host side of the microscaled operands: argument checks (before anything is
// enqueued) and the operators' launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "host_error.h"
#include "mx.h"
#include "sarathi_mx.h"

using namespace sarathi;

namespace {

// A launch holds fewer than 2^32 threads.
constexpr long MAX_TILES = (1l << 24) - 1;         // blocks of 256 threads
constexpr long MAX_W_TILES = (1l << 23) - 1;       // of 512: the product of few rows, a block per W tile
constexpr int MAX_NORM_ROWS = (1 << 24) - 256;     // of 256: a row to a block, in groups of 256

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
size_t esize(int dtype) { return dtype == SARATHI_BF16 ? 2 : 4; }
int hip_fail(hipError_t e, const char* what) { return fail(SARATHI_EHIP, "%s: %s", what, hipGetErrorString(e)); }

bool known_dtype(int d) { return d == SARATHI_F32 || d == SARATHI_BF16; }
bool known_format(int f) { return f == SARATHI_MX_E2M1 || f == SARATHI_MX_E4M3; }
bool sizes_fit(int rows, int cols) {
  return rows >= 1 && cols >= 1 && cols <= (1 << 28) && (long)mx_tiles(rows) * mx_quads(cols) <= MAX_TILES;
}

int check_operand(int format, int rows, int cols) {
  if (!known_format(format)) return fail(SARATHI_EUNSUPPORTED, "format %d", format);
  if (rows < 1 || cols < 1) return fail(SARATHI_EINVAL, "rows %d and cols %d must be positive", rows, cols);
  if (!sizes_fit(rows, cols)) return fail(SARATHI_EUNSUPPORTED, "%d x %d is more than %ld tiles", rows, cols, MAX_TILES);
  if (cols % 8) return fail(SARATHI_EUNSUPPORTED, "cols %d must be a multiple of 8", cols);
  return SARATHI_OK;
}

// Rows [rows, ld] of esize es: aligned, strides that hold a row.
int check_rows(const void* p, size_t ld, int cols, size_t es, const char* what) {
  if (!p) return fail(SARATHI_EINVAL, "%s is NULL", what);
  if (!aligned16(p) || ld * es % 16) return fail(SARATHI_EINVAL, "rows of %s must be 16-byte aligned", what);
  if (ld < (size_t)cols) return fail(SARATHI_EINVAL, "the stride %zu of %s is below cols %d", ld, what, cols);
  if (ld > (size_t)1 << 32) return fail(SARATHI_EINVAL, "the stride %zu of %s is above 2^32", ld, what);
  return SARATHI_OK;
}
size_t span(int rows, size_t ld, int cols, size_t es) { return ((size_t)(rows - 1) * ld + cols) * es; }

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

int check_memory(int format, int rows, int cols, const void* operand, size_t bytes) {
  if (!operand) return fail(SARATHI_EINVAL, "operand is NULL");
  if (!aligned16(operand)) return fail(SARATHI_EINVAL, "operand must be 16-byte aligned");
  const size_t need = mx_bytes(format, rows, cols);
  if (bytes < need) return fail(SARATHI_ENOSPC, "operand needs %zu bytes, got %zu", need, bytes);
  return SARATHI_OK;
}

int check_linear(int dtype, int kind, int a_format, int M, int N, int K) {
  if (!known_dtype(dtype)) return fail(SARATHI_EUNSUPPORTED, "dtype %d", dtype);
  if (kind < SARATHI_LINEAR_PLAIN || kind > SARATHI_LINEAR_GELU) return fail(SARATHI_EINVAL, "kind %d", kind);
  if (!known_format(a_format)) return fail(SARATHI_EUNSUPPORTED, "a_format %d", a_format);
  if (M < 1 || N < 1 || K < 1) return fail(SARATHI_EINVAL, "M, N, K must be positive");
  if (K % 8) return fail(SARATHI_EUNSUPPORTED, "K %d must be a multiple of 8", K);
  if (!sizes_fit(M, K) || !sizes_fit(N, K) || (long)mx_tiles(M) * mx_tiles(N) > MAX_TILES)
    return fail(SARATHI_EUNSUPPORTED, "%d x %d x %d is more than %ld tiles", M, N, K, MAX_TILES);
  if (mx_tiles(N) > MAX_W_TILES) return fail(SARATHI_EUNSUPPORTED, "N %d is more than %ld tiles", N, MAX_W_TILES);
  return SARATHI_OK;
}

}  // namespace

extern "C" {

size_t sarathi_mx_bytes(int format, int rows, int cols) {
  return known_format(format) && sizes_fit(rows, cols) && cols % 8 == 0 ? mx_bytes(format, rows, cols) : 0;
}

int sarathi_mx_get_layout(int format, int rows, int cols, sarathi_mx_layout* out) {
  if (!out) return fail(SARATHI_EINVAL, "out is NULL");
  const int rc = check_operand(format, rows, cols);
  if (rc) return rc;
  sarathi_mx_layout l{};
  l.tile = mx_tile_bytes(format, cols);
  l.unit = MX_ROWS * 16;
  l.row = 16;
  l.scale_cols = 256;
  l.scale_tile = (size_t)mx_quads(cols) * l.scale_cols;
  l.scale_half = MX_ROWS * 4;
  l.scale_row = 4;
  l.scale_offset = mx_scale_offset(format, rows, cols);
  l.total = mx_bytes(format, rows, cols);
  *out = l;
  return SARATHI_OK;
}

int sarathi_mx_quantize(int dtype, int format, int rows, int cols, const void* x, size_t ld_x, void* operand,
                        size_t operand_bytes, void* hip_stream) {
  if (!known_dtype(dtype)) return fail(SARATHI_EUNSUPPORTED, "dtype %d", dtype);
  int rc = check_operand(format, rows, cols);
  if (!rc) rc = check_rows(x, ld_x, cols, esize(dtype), "x");
  if (!rc) rc = check_memory(format, rows, cols, operand, operand_bytes);
  if (rc) return rc;
  if (overlap(x, span(rows, ld_x, cols, esize(dtype)), operand, mx_bytes(format, rows, cols)))
    return fail(SARATHI_EINVAL, "operand overlaps x");
  const MxQuantArgs a{rows, cols, x, ld_x, static_cast<char*>(operand)};
  const hipError_t e = launch_mx_quantize(dtype, format, a, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? SARATHI_OK : hip_fail(e, "mx_quantize");
}

int sarathi_mx_dequantize(int format, int rows, int cols, const void* operand, size_t operand_bytes, int out_dtype,
                          void* out, size_t ld_out, void* hip_stream) {
  if (!known_dtype(out_dtype)) return fail(SARATHI_EUNSUPPORTED, "out_dtype %d", out_dtype);
  int rc = check_operand(format, rows, cols);
  if (!rc) rc = check_rows(out, ld_out, cols, esize(out_dtype), "out");
  if (!rc) rc = check_memory(format, rows, cols, operand, operand_bytes);
  if (rc) return rc;
  if (overlap(out, span(rows, ld_out, cols, esize(out_dtype)), operand, mx_bytes(format, rows, cols)))
    return fail(SARATHI_EINVAL, "operand overlaps out");
  const MxQuantArgs a{rows, cols, out, ld_out, static_cast<char*>(const_cast<void*>(operand))};
  const hipError_t e = launch_mx_dequantize(out_dtype, format, a, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? SARATHI_OK : hip_fail(e, "mx_dequantize");
}

int sarathi_mx_norm(int stream_dtype, int dtype, int format, int rows, int cols, float eps, const void* x, size_t ld_x,
                    const void* delta, size_t ld_delta, const void* gain, void* h_out, size_t ld_h, void* operand,
                    size_t operand_bytes, void* hip_stream) {
  if (!known_dtype(dtype) || !known_dtype(stream_dtype) || (stream_dtype == SARATHI_BF16 && dtype == SARATHI_F32))
    return fail(SARATHI_EUNSUPPORTED, "stream_dtype %d with dtype %d", stream_dtype, dtype);
  int rc = check_operand(format, rows, cols);
  if (rc) return rc;
  if (rows > MAX_NORM_ROWS) return fail(SARATHI_EUNSUPPORTED, "rows %d above %d", rows, MAX_NORM_ROWS);
  if (cols > MX_NORM_COLS) return fail(SARATHI_EUNSUPPORTED, "cols %d above %d", cols, MX_NORM_COLS);
  if (!(eps > 0.f) || !std::isfinite(eps)) return fail(SARATHI_EINVAL, "eps must be > 0");
  const size_t ss = esize(stream_dtype), es = esize(dtype);
  rc = check_rows(x, ld_x, cols, ss, "x");
  if (!rc && delta) rc = check_rows(delta, ld_delta, cols, es, "delta");
  if (!rc) rc = check_rows(gain, cols, cols, es, "gain");
  if (!rc && h_out) rc = check_rows(h_out, ld_h, cols, ss, "h_out");
  if (!rc) rc = check_memory(format, rows, cols, operand, operand_bytes);
  if (rc) return rc;
  const size_t nx = span(rows, ld_x, cols, ss), nd = span(rows, ld_delta, cols, es), nh = span(rows, ld_h, cols, ss);
  const size_t no = mx_bytes(format, rows, cols), ng = (size_t)cols * es;
  if (overlap(operand, no, x, nx) || (delta && overlap(operand, no, delta, nd)) || overlap(operand, no, gain, ng) ||
      (h_out && overlap(operand, no, h_out, nh)))
    return fail(SARATHI_EINVAL, "operand overlaps the rows or the gain");
  if (h_out) {
    if (h_out == x ? ld_h != ld_x : overlap(h_out, nh, x, nx))
      return fail(SARATHI_EINVAL, "h_out overlaps x (it may be x itself, with the same stride)");
    if ((delta && overlap(h_out, nh, delta, nd)) || overlap(h_out, nh, gain, ng))
      return fail(SARATHI_EINVAL, "h_out overlaps delta or the gain");
  }
  const MxNormArgs a{rows, cols, eps, x, delta, gain, h_out, ld_x, ld_delta, ld_h, static_cast<char*>(operand)};
  const hipError_t e = launch_mx_norm(stream_dtype, dtype, format, a, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? SARATHI_OK : hip_fail(e, "mx_norm");
}

size_t sarathi_mx_linear_scratch_bytes(int M, int N) {
  if (M < 1 || N < 1) return 0;
  return mx_linear_parts(M, N) * 4;
}

int sarathi_mx_linear_plan(int dtype, int kind, int a_format, int M, int N, int K, size_t scratch_bytes, int* bm,
                           int* bn, int* n_split) {
  if (!bm || !bn || !n_split) return fail(SARATHI_EINVAL, "NULL pointer");
  const int rc = check_linear(dtype, kind, a_format, M, N, K);
  if (rc) return rc;
  static float dummy;   // plan only: the scratch is never touched
  MxLinearArgs p{};
  p.kind = kind; p.dtype = dtype; p.M = M; p.N = N; p.quads = mx_quads(K);
  p.parts_cap = std::min(scratch_bytes / 4, mx_linear_parts(M, N));
  p.parts = p.parts_cap ? &dummy : nullptr;
  MxLinearPlan pl{};
  if (launch_mx_linear(a_format, p, nullptr, &pl) != hipSuccess) return fail(SARATHI_EINVAL, "no plan for this op");
  *bm = pl.bm; *bn = pl.bn; *n_split = pl.splits;
  return SARATHI_OK;
}

int sarathi_mx_linear(int dtype, int kind, int a_format, int M, int N, int K, const void* a, const void* w,
                      const void* resid, void* out, void* scratch, size_t scratch_bytes, void* hip_stream) {
  const int rc = check_linear(dtype, kind, a_format, M, N, K);
  if (rc) return rc;
  if (!a || !w || !out) return fail(SARATHI_EINVAL, "NULL pointer");
  const bool needs_resid = kind == SARATHI_LINEAR_RESID || kind == SARATHI_LINEAR_RESID_F32IN;
  if (needs_resid && !resid) return fail(SARATHI_EINVAL, "resid is NULL");
  if (!aligned16(a) || !aligned16(w)) return fail(SARATHI_EINVAL, "a and w must be 16-byte aligned");
  if (!aligned16(out) || (needs_resid && !aligned16(resid)))
    return fail(SARATHI_EINVAL, "out and resid must be 16-byte aligned");
  const size_t rs = dtype == SARATHI_F32 || kind == SARATHI_LINEAR_RESID_F32IN ? 4 : 2;
  const size_t os = dtype == SARATHI_F32 || kind == SARATHI_LINEAR_RESID ? 4 : 2;
  const size_t n = (size_t)M * N, nw = mx_bytes(SARATHI_MX_E2M1, N, K), na = mx_bytes(a_format, M, K);
  if (overlap(out, n * os, a, na) || overlap(out, n * os, w, kind == SARATHI_LINEAR_SWIGLU ? 2 * nw : nw))
    return fail(SARATHI_EINVAL, "out overlaps an operand");
  if (needs_resid && (resid == out ? rs != os : overlap(out, n * os, resid, n * rs)))
    return fail(SARATHI_EINVAL, "out overlaps resid (it may be resid where their types are the same)");
  const size_t parts = std::min(scratch_bytes / 4, mx_linear_parts(M, N));
  if (scratch && parts) {
    if (overlap(scratch, parts * 4, out, n * os) || overlap(scratch, parts * 4, a, na) ||
        overlap(scratch, parts * 4, w, kind == SARATHI_LINEAR_SWIGLU ? 2 * nw : nw) ||
        (needs_resid && overlap(scratch, parts * 4, resid, n * rs)))
      return fail(SARATHI_EINVAL, "scratch overlaps an operand, out or resid");
  }
  MxLinearArgs p{};
  p.kind = kind; p.dtype = dtype; p.M = M; p.N = N; p.quads = mx_quads(K);
  p.a = static_cast<const char*>(a);
  p.w = static_cast<const char*>(w);
  p.a_scale = reinterpret_cast<const uint32_t*>(p.a + mx_scale_offset(a_format, M, K));
  p.w_scale = reinterpret_cast<const uint32_t*>(p.w + mx_scale_offset(SARATHI_MX_E2M1, N, K));
  p.up = nw;
  p.resid = resid;
  p.out = out;
  if (scratch && parts && aligned16(scratch)) {
    p.parts = static_cast<float*>(scratch);
    p.parts_cap = parts;
  }
  const hipError_t e = launch_mx_linear(a_format, p, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? SARATHI_OK : hip_fail(e, "mx_linear");
}

}  // extern "C"
