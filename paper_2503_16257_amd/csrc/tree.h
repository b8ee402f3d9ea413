// Arguments of the kernels for trees of drafted tokens, and their launches (tree.hip, cache8_tree.hip, cache8_append.hip).
#pragma once

#include "cache8.h"

namespace vidkv {

struct TreeMasks {
  const int32_t* parent;       // [B][n], or nullptr: a chain
  const int32_t* count;        // or nullptr
  const int32_t* base;
  uint64_t* mask;              // [B][n][ceil(n / 64)]
  int32_t* pos;                // [n_axes][B][n], or nullptr
  int n, n_axes;
};

// Rows of probabilities as a kernel takes them, strides in bytes.
struct Probs {
  const char* data;
  long long sb, st;
};

struct TreeVerify {
  Probs target, draft;         // [B][n][vocab]; draft.data may be nullptr
  const int32_t* token;        // [B][n]
  const int32_t* parent;       // [B][n], or nullptr: a chain
  const int32_t* count;        // or nullptr
  const float* uniform;        // [B][n]
  int32_t* path;               // [B][n]
  int32_t* accepted;
  int32_t* next;
  int n, vocab, distinct;
};

hipError_t launch_tree_masks(const TreeMasks& a, int batch, hipStream_t st);
size_t tree_verify_ws_bytes(int batch, int n, int vocab);
hipError_t launch_tree_verify(const TreeVerify& a, int dtype, int batch, void* ws, hipStream_t st);
vidkv_status launch_c8_tree(const C8Geom& g, int layer, int n, float scale, const vidkv_view* q, const vidkv_view* K, const vidkv_view* V,
                            const uint64_t* mask, const uint8_t* cache, const int32_t* length, const int32_t* count,
                            const vidkv_view* out, void* ws, size_t ws_bytes, hipStream_t st);      // (ENOSPACE: fewer bytes than its plan's)
bool c8_append_fits(const C8Geom& g);
hipError_t launch_c8_append(const C8Geom& g, int n, const vidkv_view* K, long long k_layer, const vidkv_view* V, long long v_layer,
                            const int32_t* path, const int32_t* count, const int32_t* start, uint8_t* cache, hipStream_t st);

}  // namespace vidkv
