// Internal declarations of the operators around the cache: rotary positions,
// windowed attention with sinks, sequence forks and pool compaction.
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

}  // namespace dms
