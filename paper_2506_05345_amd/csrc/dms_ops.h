// Internal declarations of the operators around the cache: rotary positions,
// windowed attention with sinks, sequence forks and pool compaction, trees of
// drafted tokens and token sampling.
#pragma once

#include <hip/hip_runtime.h>

#include "dms_common.h"

namespace dms {

constexpr int kMaxRotary = 512;      // rotated elements of a head
constexpr int kRopeAxes = 4;
constexpr int kPageLayers = 64;      // layers whose pool addresses travel in one launch

// Where a call's queries and keys (or their gradients) are read and written;
// strides in elements from a token to the next.
struct RopeTensors {
  const void* q;
  const void* k;
  void* q_out;
  void* k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
};
hipError_t launch_rope(const dms_rope_config& c, int tokens, const RopeTensors& t, const int32_t* positions,
                       const double* inv_freq, bool back, float* logits_out, uint8_t* decisions_out,
                       const float* dlogits, hipStream_t st);

size_t window_workspace_bytes(const dms_window_config& c);
bool window_grids_fit(const dms_window_config& c);   // of a configuration that is otherwise valid
hipError_t launch_window_fwd(const dms_window_config& c, const int32_t* cu, const void* q, const void* k,
                             const void* v, void* out, float* lse, void* ws, hipStream_t st);
hipError_t launch_window_bwd(const dms_window_config& c, const int32_t* cu, const void* q, const void* k,
                             const void* v, const float* lse, const void* dout, void* dq,
                             void* dk, void* dv, void* ws, hipStream_t st);

// Forks' and compactions' part of a context's workspace, its last bytes.
struct PagesLayout {
  size_t fk_base, fk_tiles, fk_block;   // per layer: page and tile prefix sums per (pair, head), the call's block of pages
  size_t cp_lists;                      // per layer: free ids below the live count and which pages move
  size_t cp_list_stride;                // int32 entries of one layer
  size_t bytes;                         // of this part
};
PagesLayout pages_layout(const dms_config& c, size_t max_heads, size_t at);

// layer -1: every layer.  pools: one pointer per layer of the context.
hipError_t launch_seq_fork(const dms_config& c, const Layout& lo, void* meta, void* ws, void* const* pools,
                           int layer, int n, const int32_t* src, const int32_t* dst, hipStream_t st);
hipError_t launch_compact(const dms_config& c, const Layout& lo, void* meta, void* ws, void* const* pools,
                          int layer, int32_t* used_out, hipStream_t st);

// Trees of drafted tokens.
constexpr int kTreeMaxNodes = 256;     // nodes of a tree: a thread each in its preparation
constexpr int kTreeWords = kTreeMaxNodes / 32;
constexpr int kTreeWorkgroups = 512;   // attention workgroups at most (a workspace holds their partial results)
size_t tree_workspace_bytes(const dms_config& c, int n, int total, int max_nodes);
// flags null: decisions from q, written to decisions_out where that is given.
hipError_t launch_tree_attention(const dms_config& c, const Layout& lo, void* meta, void* pool, int layer, int n,
                                 const int32_t* seq_ids, const int32_t* cu, int total, int max_nodes,
                                 const int32_t* parents, const void* q, const void* k, const void* v,
                                 const uint8_t* flags, uint8_t* decisions_out, void* out, void* ws, hipStream_t st);
hipError_t launch_tree_accept(int n, const int32_t* cu, int total, int max_nodes, const int32_t* parents,
                              const int32_t* tokens, const int32_t* targets, const int32_t* first, int32_t* path,
                              int32_t* path_len, int32_t* next, hipStream_t st);
hipError_t launch_tree_commit(const dms_config& c, const Layout& lo, void* meta, void* pool, int layer, int n,
                              const int32_t* seq_ids, const int32_t* cu, int total, int max_nodes, const int32_t* path,
                              const int32_t* path_len, const void* k, const void* v, const uint8_t* flags, void* ws,
                              hipStream_t st);

// Token sampling.
constexpr int kSampleMaxVocab = 1 << 20;
size_t sample_workspace_bytes(const dms_sample_config& c, int rows);
hipError_t launch_sample(const dms_sample_config& c, int rows, const void* logits, int64_t stride, const float* temperature,
                         const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* tokens,
                         float* logprobs, void* ws, hipStream_t st);

}  // namespace dms
