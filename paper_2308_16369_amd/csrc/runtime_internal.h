// Host-side helpers shared between the sources of libsarathi's C-ABI.
#pragma once

#include <stddef.h>

#include <vector>

#include "sarathi.h"

namespace sarathi {

constexpr int PARTS_ROWS = 512;   // split-K partials are sized for batches up to this many rows (larger
                                  // batches fill the GPU without splitting; with less room fewer splits run)

// A batch of any number of prompt chunks plus decodes (the hybrid batch of
// the paper has at most one chunk).
struct ChunkDesc {
  int slot, offset, len;
};
struct BatchDesc {
  std::vector<ChunkDesc> chunks;
  int B = 0;
  const int* dslots = nullptr;
  const int* dctx = nullptr;
  int rows() const {
    int r = B;
    for (const ChunkDesc& c : chunks) r += c.len;
    return r;
  }
};

// The checks of the public calls (SARATHI_* code, message set): a batch's
// arrays, a batch against a cache of n_slots x S positions, a model cfg and a
// layer's weights.
int from_mixed(const sarathi_mixed_batch* b, BatchDesc* out);
int check_batch(const BatchDesc& b, int n_slots, int S);
int check_cfg(const sarathi_model_cfg* c);
int check_weights(const sarathi_model_cfg* cfg, const sarathi_layer_weights* w, int layer);

// Every host-side check of sarathi_hybrid_layer_forward that does not
// involve the workspace (SARATHI_* error code, message set); on success
// *need = the workspace bytes the batch needs for this KV's max_seq_len
// (sarathi_workspace_layout(...).total).
int hybrid_check_noalloc(const sarathi_model_cfg* cfg, const sarathi_layer_weights* w, const sarathi_kv* kv,
                         int layer, const sarathi_hybrid_batch* batch, const void* x_in, const void* x_out,
                         size_t* need);

}  // namespace sarathi
