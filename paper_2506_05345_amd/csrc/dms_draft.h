// Internal declarations of trees of drafted tokens over the cache and of token
// sampling.
#pragma once

#include <hip/hip_runtime.h>

#include "dms_common.h"

namespace dms {

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
