// Device arguments and host launchers of the 8-bit KV cache's operators.
#pragma once

#include "kernels.h"

namespace sarathi {

constexpr float KV8_INT8_MAX = 127.f, KV8_E4M3_MAX = 448.f;
constexpr float KV8_TINY = 7.8886090522101181e-31f;   // 2^-100: smaller scales are zero

// One layer's codes (strides in bytes) and scales (strides in floats).
struct Kv8Layer {
  uint8_t* codes;
  float* scales;
  size_t slot, kv, head;        // position stride: head_dim
  size_t s_slot, s_kv, s_head;
  int log2_block;
};

// ---- a plan's rows: a span is up to KV8_SPAN rows of one slot that share their attention partials' layout,
// [slot, position, row, rows, first partial row, key splits, partial rows from split to split]; the kernel fills row
// r's slot and position, its combine entry (kernels.h) and its rotary table, (cos, sin) of pair i at
// tab[r * pairs + i].
constexpr int KV8_SPAN = 32;
constexpr int KV8_SPAN_INTS = 7;
constexpr int KV8_MAX_PAIRS = 64;
struct Kv8RowsArgs {
  const int* spans;
  int n_spans;
  int* row_slot;
  int* row_pos;
  int* comb;
  float2* tab;
  int pairs;
  float mscale;
  double theta[KV8_MAX_PAIRS];
};
hipError_t launch_kv8_rows(const Kv8RowsArgs& a, hipStream_t s);

// ---- append.  A unit is a touched block: [slot, block, row, (p0 << 16) | p1], the block's positions p0 .. p1 - 1
// being rows row .. of the batch (its positions before p0 hold earlier tokens).
struct Kv8AppendArgs {
  const void* qkv;
  size_t ld_qkv;
  void* q_out;
  size_t ld_q;
  const void* q_gain;           // null: no head norms
  const void* k_gain;
  float eps;
  int T, nh, nkv;
  const float2* tab;
  int rot, interleaved;         // leading dims rotated (0: none)
  const int* units;             // n_chunk units of several rows, then n_units - n_chunk of one
  int n_chunk, n_units;
  Kv8Layer kv;
};
hipError_t launch_kv8_append(int dtype, int format, int hd, int block, const Kv8AppendArgs& a, hipStream_t s);

// ---- read
struct Kv8ReadArgs {
  const int* row_slot;
  const int* row_pos;
  void* k_out;
  size_t ld_k;
  void* v_out;
  size_t ld_v;
  int T, nkv, hd;
  Kv8Layer kv;
};
hipError_t launch_kv8_read(int out_dtype, int format, const Kv8ReadArgs& a, hipStream_t s);

// ---- attention of decodes.  Item: a range of one decode's keys, [row, slot, first key, end key, partial row (-1: the
// row's only item)].  Rows of several items are joined: [row, items, first partial row].
constexpr int KV8_DEC_INTS = 5, KV8_JOIN_INTS = 3;
struct Kv8DecodeArgs {
  const void* q;
  size_t ld_q;
  void* out;
  size_t ld_out;
  const int* work;              // [n_work][KV8_DEC_INTS]
  const int* joins;             // [n_joins][KV8_JOIN_INTS]
  int n_joins;
  int n_work, nh, nkv;
  float* part;                  // partial rows (kernels.h)
  float scale_log2;             // softmax scale * log2 e
  Kv8Layer kv;
};
hipError_t launch_kv8_decode(int dtype, int format, int hd, const Kv8DecodeArgs& a, hipStream_t s);

// ---- attention of prompt chunks.  The query heads of a key/value head are packed with the chunk's rows: packed row
// p is chunk row p / group, head p % group; a block takes KV8_QB / group chunk rows.
constexpr int KV8_QB = 128;
constexpr int KV8_KT = 64;      // keys per tile
struct Kv8ChunkArgs {
  const void* q;
  size_t ld_q;
  void* out;
  size_t ld_out;
  const int* chunks;            // [n][slot, offset, len, first row]
  const int* work;              // [n_work][4]: chunk, first chunk row, partial base or -1, (tile begin << 16) | tile end
  int n_work, nh, nkv;
  int groups;                   // 4-wave groups per block: 1 or, of bf16, 2
  float* part;                  // partial row of the item's j-th chunk row: base + j
  float scale_log2;
  Kv8Layer kv;
};
hipError_t launch_kv8_chunk(int dtype, int format, int hd, const Kv8ChunkArgs& a, hipStream_t s);

}  // namespace sarathi
