// C-ABI entry points of libdms: configuration checks, buffer layout, the host
// context and the per-call argument validation that runs before any HIP call.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <initializer_list>
#include <mutex>
#include <vector>

#include "dms_common.h"
#include "dms_draft.h"
#include "dms_fp8.h"
#include "dms_ops.h"
#include "dms_train.h"

namespace dms {

int validate_config(const dms_config& c) {
  if (c.num_layers < 1 || c.max_seqs < 1 || c.max_seqs > kMaxSeqs) return DMS_ERR_INVALID;
  if (c.num_kv_heads < 1 || c.group_size < 1 || c.window < 1) return DMS_ERR_INVALID;
  if (c.group_size > (c.kv_format == DMS_KV_MLA ? kMlaMaxGroup : kMaxGroup)) return DMS_ERR_UNSUPPORTED;
  if (c.head_dim < 1) return DMS_ERR_INVALID;
  if (c.kv_format == DMS_KV_MLA) {
    // latent rows: one KV head, caller decisions, no page retrieval
    if (c.head_dim != kMlaDim) return DMS_ERR_UNSUPPORTED;
    if (c.num_kv_heads != 1 || c.decision_source != DMS_DECIDE_CALLER || c.quest_page_budget != 0)
      return DMS_ERR_UNSUPPORTED;
  } else if (c.head_dim != 64 && c.head_dim != 128) {
    return DMS_ERR_UNSUPPORTED;
  }
  // Split-K partial accumulators (one g x row-width float32 block per
  // partial, kMaxWaves + max_seqs * Hkv partials, kMaxMlaUnits + max_seqs for
  // latent rows) are addressed through a buffer resource with 32-bit byte
  // offsets, so their area must stay below 2 GiB for every page format.
  {
    const bool mla_rows = c.kv_format == DMS_KV_MLA;
    const int64_t row = mla_rows ? kMlaLatent : c.head_dim;
    const int64_t partials = (mla_rows ? kMaxMlaUnits : kMaxWaves) +
                             static_cast<int64_t>(c.max_seqs) * c.num_kv_heads;
    if (partials * c.group_size * row * 4 >= (int64_t(1) << 31)) return DMS_ERR_UNSUPPORTED;
  }
  if (c.page_size != 32 && c.page_size != 64 && c.page_size != 128 && c.page_size != 256)
    return DMS_ERR_INVALID;
  if (c.num_pages < 1 || c.max_pages_per_head < 1 || c.max_chunk_tokens < 0) return DMS_ERR_INVALID;
  if (!(c.softmax_scale <= 0.0f || isfinite(c.softmax_scale))) return DMS_ERR_INVALID;
  if (isnan(c.softmax_scale)) return DMS_ERR_INVALID;
  if (c.eviction != DMS_EVICT_DELAYED && c.eviction != DMS_EVICT_IMMEDIATE) return DMS_ERR_INVALID;
  if (c.decision_source != DMS_DECIDE_CALLER && c.decision_source != DMS_DECIDE_QUERY)
    return DMS_ERR_INVALID;
  if (c.decision_source == DMS_DECIDE_QUERY && !isfinite(c.decision_bias)) return DMS_ERR_INVALID;
  if (c.kv_format != DMS_KV_BF16 && c.kv_format != DMS_KV_FP8 && c.kv_format != DMS_KV_MLA)
    return DMS_ERR_INVALID;
  if (c.quest_page_budget < 0 || c.quest_page_budget > c.max_pages_per_head) return DMS_ERR_INVALID;
  if (c.quest_page_budget > 0 && c.max_pages_per_head > 4096) return DMS_ERR_UNSUPPORTED;
  // slot and page indices are int32 on the device
  if (static_cast<int64_t>(c.max_pages_per_head) * c.page_size >= (int64_t(1) << 31)) return DMS_ERR_INVALID;
  if (static_cast<int64_t>(c.max_seqs) * c.num_kv_heads > (int64_t(1) << 22)) return DMS_ERR_INVALID;
  if (static_cast<int64_t>(c.max_chunk_tokens) * c.num_kv_heads >= (int64_t(1) << 31)) return DMS_ERR_INVALID;
  return DMS_OK;
}

Layout make_layout(const dms_config& c) {
  Layout lo{};
  const size_t S = c.max_seqs, H = c.num_kv_heads, w = c.window;
  const size_t maxp = c.max_pages_per_head, P = c.page_size, D = c.head_dim;
  lo.max_slots = static_cast<int>(maxp * P);
  lo.max_heads = static_cast<int>(S * H);
  const bool mla_rows = c.kv_format == DMS_KV_MLA;
  lo.max_partials = (mla_rows ? kMaxMlaUnits : kMaxWaves) + lo.max_heads;
  lo.ml_stride = mla_rows ? (c.group_size + kMaxGroup - 1) / kMaxGroup * kMaxGroup : kMaxGroup;
  lo.head_groups = mla_rows ? (c.group_size + kMaxGroup - 1) / kMaxGroup : 1;
  // meta
  lo.status = 0;
  lo.layer0 = kAlign;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, kAlign); return o; };
  lo.pos = take(S * 4);
  lo.len = take(S * H * 4);
  lo.ring = take(S * H * w * 4);
  lo.page_table = take(S * H * maxp * 4);
  lo.slot_meta = take(S * H * maxp * P * 4);
  lo.stack = take(static_cast<size_t>(c.num_pages) * 4);
  lo.top = take(4);
  lo.page_bounds = c.quest_page_budget > 0 ? take(static_cast<size_t>(c.num_pages) * 2 * D * 2) : 0;
  lo.layer_stride = off;
  lo.meta_bytes = lo.layer0 + lo.layer_stride * c.num_layers;
  // pool
  lo.page_bytes = c.kv_format == DMS_KV_FP8   ? P / 32 * fp8_tile_bytes(static_cast<int>(D))
                  : c.kv_format == DMS_KV_MLA ? P / 32 * mla_tile_bytes(static_cast<int>(D))
                                              : 2 * P * D * 2;
  lo.pool_bytes = lo.page_bytes * static_cast<size_t>(c.num_pages);
  // workspace
  off = 0;
  const size_t NH = lo.max_heads, NP = lo.max_partials;
  lo.ws_head_desc = take(NH * sizeof(HeadDesc));
  lo.ws_cum_tiles = take((NH + 1) * 4);
  lo.ws_part_ml = take(NP * lo.ml_stride * 8);
  const size_t Dout = c.kv_format == DMS_KV_MLA ? kMlaLatent : D;   // output row width
  lo.ws_part_acc = take(NP * c.group_size * Dout * 4);
  lo.ws_wave_bounds = take((kMaxWaves + 1) * 4);
  lo.ws_wave_desc = take(kMaxWaves * 2 * sizeof(int4));   // per decode wave: first segment
  lo.ws_head_waves = take(NH * sizeof(int4));              // per head: waves holding its tiles
  lo.ws_head_cnt = take(NH * lo.head_groups * 4);
  lo.ws_plan_ctr = take(16);
  lo.ws_ck_need = take(NH * 4);
  lo.ws_ck_fresh = take(NH * 4);
  lo.ws_ck_base = take(NH * 4);
  lo.ws_ck_pos0 = take(S * 4);
  lo.ws_ck_top = take(16);
  lo.ws_ck_slot = take(static_cast<size_t>(c.max_chunk_tokens) * H * 4);
  lo.ws_pf_cum = take((NH + 1) * 4);
  lo.ws_pf_meta = take(static_cast<size_t>(c.max_chunk_tokens) * H * 4);
  // prefill: chunk keys / values (latent rows) and the compacted kept ones,
  // in the pool's tile layout; sequence i of a call starts at tile
  // cu[i] / 32 + i
  lo.pf_tiles_per_head = static_cast<int>((static_cast<size_t>(c.max_chunk_tokens) + 31) / 32 + S + 1);
  lo.ws_pf_tiles = take(2 * H * static_cast<size_t>(lo.pf_tiles_per_head) * D *
                        (c.kv_format == DMS_KV_MLA ? 64 : 128));
  lo.ws_pf_tmeta = take(2 * H * static_cast<size_t>(lo.pf_tiles_per_head) * 32 * 4);   // their key rows
  lo.ws_pf_zeros = take(D * 64);   // zero values of a tile that does not exist
  lo.ws_pf_flags = take(static_cast<size_t>(c.max_chunk_tokens) * H);  // decisions from q
  // kept chunk tokens before every 32-aligned chunk position, per KV head
  // (same indexing as the tiles of one region)
  lo.ws_pf_kb = take(H * static_cast<size_t>(lo.pf_tiles_per_head) * 4);
  lo.ws_pf_order = take(NH * 36 + 4);   // attention rows, heaviest head first, and their first work items
  lo.ws_q_sel = take(NH * static_cast<size_t>(c.quest_page_budget) * 4);
  lo.ws_q_page = take(NH * static_cast<size_t>(c.quest_page_budget) * 4);
  lo.ws_q_len = take(NH * 4);
  lo.workspace_bytes = off + pages_layout(c, NH, off).bytes;
  return lo;
}

struct Ctx {
  dms_config cfg;
  Layout lo;
  void* meta;
  std::vector<void*> pools;
  void* ws;
  int decode_waves;  // resident decode waves, found on first decode
  // kernel timing session: event pairs and the kind of kernel each timed
  std::vector<hipEvent_t> ev;
  std::vector<int> ev_kind;
  int ev_used = 0;
  bool profiling = false;
};

}  // namespace dms

using dms::Ctx;

struct dms_ctx {
  Ctx c;
};

// Scratch of dms_decode_step_static (see static_scratch below): one copy per
// GPU, held until the process ends.
constexpr size_t kStaticScratchBytes = size_t(32) << 20;
static __device__ __align__(256) char scratch[kStaticScratchBytes];

namespace {

inline hipStream_t as_stream(void* s) { return static_cast<hipStream_t>(s); }

inline int hip_rc(hipError_t e) { return e == hipSuccess ? DMS_OK : DMS_ERR_HIP; }

// Latent-attention cache: keys only (the values are part of the key row).
inline bool mla(const dms_ctx* ctx) { return ctx->c.cfg.kv_format == DMS_KV_MLA; }

// Event pair for the next timed launch of a session (or nulls).
void next_events(Ctx& c, int kind, hipEvent_t* a, hipEvent_t* b) {
  *a = nullptr;
  *b = nullptr;
  if (!c.profiling || c.ev_used + 2 > static_cast<int>(c.ev.size())) return;
  *a = c.ev[c.ev_used];
  *b = c.ev[c.ev_used + 1];
  c.ev_kind[c.ev_used / 2] = kind;
  c.ev_used += 2;
}

int check_call(const dms_ctx* ctx, int layer, int n, const void* seq_ids) {
  if (!ctx) return DMS_ERR_INVALID;
  if (layer < 0 || layer >= ctx->c.cfg.num_layers) return DMS_ERR_INVALID;
  if (n < 1 || n > ctx->c.cfg.max_seqs) return DMS_ERR_INVALID;
  if (!seq_ids) return DMS_ERR_INVALID;
  return DMS_OK;
}

int check_chunk(const dms_ctx* ctx, const int32_t* cu, int total, int max_len) {
  if (!cu) return DMS_ERR_INVALID;
  if (total < 0 || total > ctx->c.cfg.max_chunk_tokens) return DMS_ERR_INVALID;
  if (max_len < 0 || max_len > total) return DMS_ERR_INVALID;
  if (total > 0 && max_len == 0) return DMS_ERR_INVALID;
  return DMS_OK;
}

// Page retrieval buffers in the workspace.
const int32_t* quest_lengths(const Ctx& c) {
  return reinterpret_cast<const int32_t*>(static_cast<char*>(c.ws) + c.lo.ws_q_len);
}
const int32_t* quest_pages(const Ctx& c) {
  return reinterpret_cast<const int32_t*>(static_cast<char*>(c.ws) + c.lo.ws_q_sel);
}
const int32_t* quest_phys_pages(const Ctx& c) {
  return reinterpret_cast<const int32_t*>(static_cast<char*>(c.ws) + c.lo.ws_q_page);
}

// ---------------------------------------------------------------------------
// Static scratch of dms_decode_step_static
// ---------------------------------------------------------------------------

// Device memory that dms_decode_step_static works in instead of the caller's
// workspace: planner output (head descriptors, tile prefix sums, per-wave
// ranges, per-head wave spans), split-K partials and arrival counters.  Every
// GPU the library runs on holds its own copy until the process ends.  In host
// code the name is only a stand-in for the symbol; kernels get the device
// address that hipGetSymbolAddress returns for the current device.
constexpr int kMaxScratchDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_dev[kMaxScratchDevices] = {};

// Device address of the current device's scratch, resolved once per device.
int static_scratch(void** out) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxScratchDevices) return DMS_ERR_HIP;
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (g_scratch_dev[dev] == nullptr) {
    void* p = nullptr;
    if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || p == nullptr) return DMS_ERR_HIP;
    g_scratch_dev[dev] = p;
  }
  *out = g_scratch_dev[dev];
  return DMS_OK;
}

// Offsets of the decode buffers for a call of `n` sequences over `waves`
// decode waves, packed from offset 0 of the scratch (the meta and pool
// offsets of `lo` are kept).  Returns the bytes used.
size_t static_layout(const dms_config& c, int n, int waves, dms::Layout* lo) {
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = dms::align_up(off + bytes, dms::kAlign); return o; };
  const size_t NH = static_cast<size_t>(n) * c.num_kv_heads, W = static_cast<size_t>(waves);
  lo->ws_head_desc = take(NH * sizeof(dms::HeadDesc));
  lo->ws_cum_tiles = take((NH + 1) * 4);
  // (the entry point takes standard-row formats only: one head group)
  lo->ml_stride = dms::kMaxGroup;
  lo->head_groups = 1;
  lo->ws_part_ml = take((W + NH) * lo->ml_stride * 8);
  lo->ws_part_acc = take((W + NH) * c.group_size * c.head_dim * 4);
  lo->ws_wave_bounds = take((W + 1) * 4);
  lo->ws_wave_desc = take(W * 2 * sizeof(int4));
  lo->ws_head_waves = take(NH * sizeof(int4));
  lo->ws_head_cnt = take(NH * lo->head_groups * 4);
  lo->max_partials = static_cast<int>(W + NH);   // partial index = wave + call head
  return off;
}

int ensure_waves(dms_ctx* ctx) {
  if (ctx->c.decode_waves > 0) return DMS_OK;
  int w = dms::decode_resident_waves(ctx->c.cfg);
  if (w <= 0) return DMS_ERR_HIP;
  ctx->c.decode_waves = w < dms::kMaxWaves ? w : dms::kMaxWaves;
  return DMS_OK;
}

}  // namespace

extern "C" {

int dms_layout(const dms_config* cfg, size_t* meta_bytes, size_t* pool_bytes,
               size_t* workspace_bytes, size_t* page_bytes) {
  if (!cfg) return DMS_ERR_INVALID;
  int rc = dms::validate_config(*cfg);
  if (rc) return rc;
  dms::Layout lo = dms::make_layout(*cfg);
  if (meta_bytes) *meta_bytes = lo.meta_bytes;
  if (pool_bytes) *pool_bytes = lo.pool_bytes;
  if (workspace_bytes) *workspace_bytes = lo.workspace_bytes;
  if (page_bytes) *page_bytes = lo.page_bytes;
  return DMS_OK;
}

int dms_state_layout(const dms_config* cfg, dms_state_offsets* out) {
  if (!cfg || !out) return DMS_ERR_INVALID;
  int rc = dms::validate_config(*cfg);
  if (rc) return rc;
  dms::Layout lo = dms::make_layout(*cfg);
  out->status = lo.status;
  out->layer0 = lo.layer0;
  out->layer_stride = lo.layer_stride;
  out->pos = lo.pos;
  out->len = lo.len;
  out->ring = lo.ring;
  out->page_table = lo.page_table;
  out->slot_meta = lo.slot_meta;
  out->stack = lo.stack;
  out->top = lo.top;
  out->page_bounds = lo.page_bounds;
  return DMS_OK;
}

int dms_create(const dms_config* cfg, void* meta_dev, void* const* pools_dev_host,
               void* workspace_dev, dms_ctx** out) {
  if (!cfg || !meta_dev || !pools_dev_host || !workspace_dev || !out) return DMS_ERR_INVALID;
  int rc = dms::validate_config(*cfg);
  if (rc) return rc;
  for (int l = 0; l < cfg->num_layers; ++l)
    if (!pools_dev_host[l]) return DMS_ERR_INVALID;
  dms_ctx* ctx = new (std::nothrow) dms_ctx;
  if (!ctx) return DMS_ERR_INVALID;
  ctx->c.cfg = *cfg;
  if (!(ctx->c.cfg.softmax_scale > 0.0f))
    ctx->c.cfg.softmax_scale = 1.0f / sqrtf(static_cast<float>(cfg->head_dim));
  ctx->c.lo = dms::make_layout(*cfg);
  ctx->c.meta = meta_dev;
  ctx->c.pools.assign(pools_dev_host, pools_dev_host + cfg->num_layers);
  ctx->c.ws = workspace_dev;
  ctx->c.decode_waves = 0;
  *out = ctx;
  return DMS_OK;
}

int dms_destroy(dms_ctx* ctx) {
  if (!ctx) return DMS_ERR_INVALID;
  for (auto& e : ctx->c.ev) (void)hipEventDestroy(e);
  delete ctx;
  return DMS_OK;
}

int dms_init_state(dms_ctx* ctx, void* stream) {
  if (!ctx) return DMS_ERR_INVALID;
  // set-up of the current device's static scratch (dms_decode_step_static)
  void* sp = nullptr;
  if (int rc = static_scratch(&sp)) return rc;
  return hip_rc(dms::launch_init_state(ctx->c.cfg, ctx->c.lo, ctx->c.meta, ctx->c.ws,
                                       as_stream(stream)));
}

int dms_seq_reset(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev, void* stream) {
  if (!ctx) return DMS_ERR_INVALID;
  if (layer < -1 || layer >= ctx->c.cfg.num_layers) return DMS_ERR_INVALID;
  if (n < 1 || n > ctx->c.cfg.max_seqs || !seq_ids_dev) return DMS_ERR_INVALID;
  return hip_rc(dms::launch_seq_reset(ctx->c.cfg, ctx->c.lo, ctx->c.meta, layer, n, seq_ids_dev,
                                      as_stream(stream)));
}

int dms_seq_fork(dms_ctx* ctx, int layer, int n, const int32_t* src_ids_dev, const int32_t* dst_ids_dev,
                 void* stream) {
  if (!ctx) return DMS_ERR_INVALID;
  if (layer < -1 || layer >= ctx->c.cfg.num_layers) return DMS_ERR_INVALID;
  if (n < 1 || n > ctx->c.cfg.max_seqs || !src_ids_dev || !dst_ids_dev) return DMS_ERR_INVALID;
  const Ctx& c = ctx->c;
  return hip_rc(dms::launch_seq_fork(c.cfg, c.lo, c.meta, c.ws, c.pools.data(), layer, n, src_ids_dev,
                                     dst_ids_dev, as_stream(stream)));
}

int dms_compact(dms_ctx* ctx, int layer, int32_t* pages_used_out_dev, void* stream) {
  if (!ctx) return DMS_ERR_INVALID;
  if (layer < -1 || layer >= ctx->c.cfg.num_layers) return DMS_ERR_INVALID;
  const Ctx& c = ctx->c;
  return hip_rc(dms::launch_compact(c.cfg, c.lo, c.meta, c.ws, c.pools.data(), layer, pages_used_out_dev,
                                    as_stream(stream)));
}

int dms_append(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev, const void* k_dev,
               const void* v_dev, const uint8_t* flags_dev, void* stream) {
  int rc = check_call(ctx, layer, n, seq_ids_dev);
  if (rc) return rc;
  if (!k_dev || !(v_dev || mla(ctx)) || !flags_dev) return DMS_ERR_INVALID;
  const Ctx& c = ctx->c;
  hipStream_t st = as_stream(stream);
  hipError_t e = dms::launch_plan(c.cfg, c.lo, c.meta, c.ws, layer, n, seq_ids_dev, flags_dev,
                                  nullptr, nullptr, true, 0, nullptr, st);
  if (e == hipSuccess) {
    // with page retrieval the written pages' bounds are recomputed in the
    // same launch as the K / V writes
    e = c.cfg.quest_page_budget > 0
            ? dms::launch_quest_append(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n, k_dev, v_dev, st)
            : dms::launch_scatter(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n, k_dev, v_dev, st);
  }
  return hip_rc(e);
}

int dms_decode(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev, const void* q_dev,
               float* out_dev, void* stream) {
  int rc = check_call(ctx, layer, n, seq_ids_dev);
  if (rc) return rc;
  if (!q_dev || !out_dev) return DMS_ERR_INVALID;
  if ((rc = ensure_waves(ctx))) return rc;
  const Ctx& c = ctx->c;
  hipStream_t st = as_stream(stream);
  const bool quest = c.cfg.quest_page_budget > 0;
  hipError_t e = hipSuccess;
  if (quest) e = dms::launch_quest_select(c.cfg, c.lo, c.meta, c.ws, layer, n, seq_ids_dev, q_dev, st);
  if (e == hipSuccess)
    e = dms::launch_plan(c.cfg, c.lo, c.meta, c.ws, layer, n, seq_ids_dev, nullptr, nullptr, nullptr,
                         false, c.decode_waves, out_dev, st, quest ? quest_lengths(c) : nullptr);
  hipEvent_t e0, e1;
  next_events(ctx->c, DMS_PROFILE_DECODE, &e0, &e1);
  if (e == hipSuccess)
    e = dms::launch_decode(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n, q_dev, nullptr,
                           nullptr, out_dev, c.decode_waves, st, e0, e1, quest ? quest_phys_pages(c) : nullptr);
  return hip_rc(e);
}

namespace {

// Append + decode of one layer; decisions from flags_dev (caller) or from
// q_dev (decisions_out_dev receives them, may be null).
int decode_step(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev, const void* q_dev,
                const void* k_dev, const void* v_dev, const uint8_t* flags_dev,
                uint8_t* decisions_out_dev, float* out_dev, void* stream) {
  const bool from_q = ctx->c.cfg.decision_source == DMS_DECIDE_QUERY;
  const Ctx& c = ctx->c;
  hipStream_t st = as_stream(stream);
  if (c.cfg.quest_page_budget > 0) {
    // page retrieval: plan the append; write K / V, recompute the written
    // pages' bounds and select every head's pages (one launch); then decode
    // over the selection, planning its tiles inside the decode launch (up to
    // 1024 heads) or with the planner
    hipError_t e = dms::launch_plan(c.cfg, c.lo, c.meta, c.ws, layer, n, seq_ids_dev,
                                    from_q ? nullptr : flags_dev, from_q ? q_dev : nullptr,
                                    decisions_out_dev, true, 0, nullptr, st);
    if (e == hipSuccess)
      e = dms::launch_quest_append_select(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n, q_dev, k_dev,
                                          v_dev, st);
    const bool in_launch = n * c.cfg.num_kv_heads <= dms::decode_attended_max_heads();
    if (e == hipSuccess && !in_launch)
      e = dms::launch_plan(c.cfg, c.lo, c.meta, c.ws, layer, n, seq_ids_dev, nullptr, nullptr, nullptr,
                           false, c.decode_waves, out_dev, st, quest_lengths(c));
    hipEvent_t e0, e1;
    next_events(ctx->c, DMS_PROFILE_DECODE, &e0, &e1);
    if (e == hipSuccess)
      e = in_launch ? dms::launch_decode_attended(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n, q_dev,
                                                  out_dev, c.decode_waves, st, e0, e1, quest_phys_pages(c),
                                                  quest_lengths(c))
                    : dms::launch_decode(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n, q_dev, nullptr,
                                         nullptr, out_dev, c.decode_waves, st, e0, e1, quest_phys_pages(c));
    return hip_rc(e);
  }
  if (dms::decode_step_fusable(c.cfg, n)) {
    // one launch: every workgroup plans the append in LDS, the last one to
    // read the state writes it, and the waves decode (writing the new K / V
    // into their slots and merging split heads)
    hipEvent_t e0, e1;
    next_events(ctx->c, DMS_PROFILE_DECODE, &e0, &e1);
    return hip_rc(dms::launch_decode_step(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n,
                                          seq_ids_dev, flags_dev, q_dev, k_dev, v_dev,
                                          decisions_out_dev, out_dev, c.decode_waves, st, e0, e1));
  }
  // planner (slot choice, page pops, state, wave ranges) -> decode, which
  // also writes the new K / V into their slots and merges split heads
  hipError_t e = dms::launch_plan(c.cfg, c.lo, c.meta, c.ws, layer, n, seq_ids_dev,
                                  from_q ? nullptr : flags_dev, from_q ? q_dev : nullptr,
                                  decisions_out_dev, true, c.decode_waves, out_dev, st);
  hipEvent_t e0, e1;
  next_events(ctx->c, DMS_PROFILE_DECODE, &e0, &e1);
  if (e == hipSuccess)
    e = dms::launch_decode(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n, q_dev, k_dev,
                           v_dev, out_dev, c.decode_waves, st, e0, e1);
  return hip_rc(e);
}

// Masked chunk attention then commit; decisions from flags_dev or from q_dev
// (written to decisions_out_dev, or to the workspace when that is null).
int prefill_chunk(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev,
                  const int32_t* cu_seqlens_dev, int total_tokens, int max_seqlen,
                  const void* q_dev, const void* k_dev, const void* v_dev,
                  const uint8_t* flags_dev, uint8_t* decisions_out_dev, float* out_dev,
                  void* stream) {
  const Ctx& c = ctx->c;
  hipStream_t st = as_stream(stream);
  hipError_t e = hipSuccess;
  const uint8_t* flags = flags_dev;
  if (c.cfg.decision_source == DMS_DECIDE_QUERY) {
    uint8_t* buf = decisions_out_dev != nullptr
                       ? decisions_out_dev
                       : reinterpret_cast<uint8_t*>(static_cast<char*>(c.ws) + c.lo.ws_pf_flags);
    e = dms::launch_prefill_decide(c.cfg, q_dev, total_tokens, buf, st);
    flags = buf;
  }
  hipEvent_t e0, e1;
  next_events(ctx->c, DMS_PROFILE_PREFILL, &e0, &e1);
  if (e == hipSuccess)
    e = dms::launch_prefill_attention(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n,
                                      seq_ids_dev, cu_seqlens_dev, total_tokens, max_seqlen, q_dev,
                                      k_dev, v_dev, flags, out_dev, st, e0, e1);
  if (e == hipSuccess)
    e = dms::launch_chunk_commit(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n, seq_ids_dev,
                                 cu_seqlens_dev, total_tokens, max_seqlen, k_dev, v_dev, flags, st);
  if (e == hipSuccess && c.cfg.quest_page_budget > 0)
    e = dms::launch_quest_bounds(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n, true,
                                 seq_ids_dev, st);
  return hip_rc(e);
}

}  // namespace

int dms_decode_step(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev, const void* q_dev,
                    const void* k_dev, const void* v_dev, const uint8_t* flags_dev,
                    float* out_dev, void* stream) {
  int rc = check_call(ctx, layer, n, seq_ids_dev);
  if (rc) return rc;
  if (ctx->c.cfg.decision_source != DMS_DECIDE_CALLER) return DMS_ERR_INVALID;
  if (!q_dev || !k_dev || !(v_dev || mla(ctx)) || !flags_dev || !out_dev) return DMS_ERR_INVALID;
  if ((rc = ensure_waves(ctx))) return rc;
  return decode_step(ctx, layer, n, seq_ids_dev, q_dev, k_dev, v_dev, flags_dev, nullptr, out_dev,
                     stream);
}

int dms_decode_step_static(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev,
                           const void* q_dev, const void* k_dev, const void* v_dev,
                           const uint8_t* flags_dev, float* out_dev, void* stream) {
  int rc = check_call(ctx, layer, n, seq_ids_dev);
  if (rc) return rc;
  const dms_config& cfg = ctx->c.cfg;
  if (cfg.decision_source != DMS_DECIDE_CALLER) return DMS_ERR_INVALID;
  if (cfg.kv_format == DMS_KV_MLA || cfg.quest_page_budget > 0) return DMS_ERR_UNSUPPORTED;
  if (!q_dev || !k_dev || !v_dev || !flags_dev || !out_dev) return DMS_ERR_INVALID;
  if ((rc = ensure_waves(ctx))) return rc;
  const Ctx& c = ctx->c;
  dms::Layout slo = c.lo;
  if (static_layout(cfg, n, c.decode_waves, &slo) > kStaticScratchBytes) return DMS_ERR_SCRATCH;
  void* sp = nullptr;
  if ((rc = static_scratch(&sp))) return rc;
  hipStream_t st = as_stream(stream);
  // the same planner and decode kernels as dms_decode_step; the planner also
  // clears the arrival counters of the call's heads, which an earlier call
  // (of any context) may have left in the scratch
  hipError_t e = dms::launch_plan(cfg, slo, c.meta, sp, layer, n, seq_ids_dev, flags_dev, nullptr,
                                  nullptr, true, c.decode_waves, out_dev, st, nullptr, true);
  hipEvent_t e0, e1;
  next_events(ctx->c, DMS_PROFILE_DECODE, &e0, &e1);
  if (e == hipSuccess)
    e = dms::launch_decode(cfg, slo, c.meta, sp, c.pools[layer], layer, n, q_dev, k_dev, v_dev,
                           out_dev, c.decode_waves, st, e0, e1);
  return hip_rc(e);
}

int dms_decode_step_q(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev,
                      const void* q_dev, const void* k_dev, const void* v_dev,
                      uint8_t* decisions_out_dev, float* out_dev, void* stream) {
  int rc = check_call(ctx, layer, n, seq_ids_dev);
  if (rc) return rc;
  if (ctx->c.cfg.decision_source != DMS_DECIDE_QUERY) return DMS_ERR_INVALID;
  if (!q_dev || !k_dev || !v_dev || !out_dev) return DMS_ERR_INVALID;
  if ((rc = ensure_waves(ctx))) return rc;
  return decode_step(ctx, layer, n, seq_ids_dev, q_dev, k_dev, v_dev, nullptr, decisions_out_dev,
                     out_dev, stream);
}

int dms_append_chunk(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev,
                     const int32_t* cu_seqlens_dev, int total_tokens, int max_seqlen,
                     const void* k_dev, const void* v_dev, const uint8_t* flags_dev,
                     void* stream) {
  int rc = check_call(ctx, layer, n, seq_ids_dev);
  if (rc) return rc;
  if ((rc = check_chunk(ctx, cu_seqlens_dev, total_tokens, max_seqlen))) return rc;
  if (total_tokens == 0) return DMS_OK;
  if (!k_dev || !(v_dev || mla(ctx)) || !flags_dev) return DMS_ERR_INVALID;
  const Ctx& c = ctx->c;
  hipStream_t st = as_stream(stream);
  hipError_t e = dms::launch_chunk_scan(c.cfg, c.lo, c.meta, c.ws, layer, n, seq_ids_dev, cu_seqlens_dev,
                                        total_tokens, max_seqlen, flags_dev, false, as_stream(stream));
  if (e == hipSuccess)
    e = dms::launch_chunk_commit(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n,
                                          seq_ids_dev, cu_seqlens_dev, total_tokens, max_seqlen,
                                          k_dev, v_dev, flags_dev, st);
  // page retrieval: a chunk may write into any page of a head (reused slots)
  if (e == hipSuccess && c.cfg.quest_page_budget > 0)
    e = dms::launch_quest_bounds(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n, true,
                                 seq_ids_dev, st);
  return hip_rc(e);
}

int dms_quest_selection(dms_ctx* ctx, int n, int32_t* pages_out_dev, int32_t* count_out_dev,
                        void* stream) {
  if (!ctx || ctx->c.cfg.quest_page_budget <= 0) return DMS_ERR_INVALID;
  if (n < 1 || n > ctx->c.cfg.max_seqs || !pages_out_dev || !count_out_dev) return DMS_ERR_INVALID;
  const Ctx& c = ctx->c;
  return hip_rc(dms::launch_quest_export(c.cfg, c.lo, c.ws, n, pages_out_dev, count_out_dev,
                                         as_stream(stream)));
}

int dms_prefill_chunk(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev,
                      const int32_t* cu_seqlens_dev, int total_tokens, int max_seqlen,
                      const void* q_dev, const void* k_dev, const void* v_dev,
                      const uint8_t* flags_dev, float* out_dev, void* stream) {
  int rc = check_call(ctx, layer, n, seq_ids_dev);
  if (rc) return rc;
  if (ctx->c.cfg.decision_source != DMS_DECIDE_CALLER) return DMS_ERR_INVALID;
  if ((rc = check_chunk(ctx, cu_seqlens_dev, total_tokens, max_seqlen))) return rc;
  if (total_tokens == 0) return DMS_OK;
  if (!q_dev || !k_dev || !(v_dev || mla(ctx)) || !flags_dev || !out_dev) return DMS_ERR_INVALID;
  return prefill_chunk(ctx, layer, n, seq_ids_dev, cu_seqlens_dev, total_tokens, max_seqlen, q_dev,
                       k_dev, v_dev, flags_dev, nullptr, out_dev, stream);
}

int dms_prefill_chunk_q(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev,
                        const int32_t* cu_seqlens_dev, int total_tokens, int max_seqlen,
                        const void* q_dev, const void* k_dev, const void* v_dev,
                        uint8_t* decisions_out_dev, float* out_dev, void* stream) {
  int rc = check_call(ctx, layer, n, seq_ids_dev);
  if (rc) return rc;
  if (mla(ctx)) return DMS_ERR_UNSUPPORTED;
  if (ctx->c.cfg.decision_source != DMS_DECIDE_QUERY) return DMS_ERR_INVALID;
  if ((rc = check_chunk(ctx, cu_seqlens_dev, total_tokens, max_seqlen))) return rc;
  if (total_tokens == 0) return DMS_OK;
  if (!q_dev || !k_dev || !v_dev || !out_dev) return DMS_ERR_INVALID;
  return prefill_chunk(ctx, layer, n, seq_ids_dev, cu_seqlens_dev, total_tokens, max_seqlen, q_dev,
                       k_dev, v_dev, nullptr, decisions_out_dev, out_dev, stream);
}

int dms_retained_lengths(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev,
                         int32_t* out_dev, void* stream) {
  int rc = check_call(ctx, layer, n, seq_ids_dev);
  if (rc) return rc;
  if (!out_dev) return DMS_ERR_INVALID;
  return hip_rc(dms::launch_retained(ctx->c.cfg, ctx->c.lo, ctx->c.meta, layer, n, seq_ids_dev,
                                     out_dev, as_stream(stream)));
}

int dms_export_state(dms_ctx* ctx, int layer, void* dst_host, size_t bytes, void* stream) {
  if (!ctx || !dst_host) return DMS_ERR_INVALID;
  if (layer < 0 || layer >= ctx->c.cfg.num_layers) return DMS_ERR_INVALID;
  if (bytes < ctx->c.lo.layer_stride) return DMS_ERR_INVALID;
  hipStream_t st = as_stream(stream);
  const char* src = static_cast<const char*>(ctx->c.meta) + ctx->c.lo.layer0 +
                    static_cast<size_t>(layer) * ctx->c.lo.layer_stride;
  hipError_t e = hipStreamSynchronize(st);
  if (e == hipSuccess) e = hipMemcpy(dst_host, src, ctx->c.lo.layer_stride, hipMemcpyDeviceToHost);
  return hip_rc(e);
}

int dms_status(dms_ctx* ctx, void* stream) {
  if (!ctx) return DMS_ERR_INVALID;
  int32_t v = 0;
  hipError_t e = hipStreamSynchronize(as_stream(stream));
  if (e == hipSuccess)
    e = hipMemcpy(&v, static_cast<char*>(ctx->c.meta) + ctx->c.lo.status, sizeof(v),
                  hipMemcpyDeviceToHost);
  if (e != hipSuccess) return DMS_ERR_HIP;
  return v;
}

int dms_clear_status(dms_ctx* ctx, void* stream) {
  if (!ctx) return DMS_ERR_INVALID;
  int32_t* status = reinterpret_cast<int32_t*>(static_cast<char*>(ctx->c.meta) + ctx->c.lo.status);
  return hip_rc(dms::launch_set_status(status, 0, as_stream(stream)));
}

int dms_profile_start(dms_ctx* ctx, int max_launches) {
  if (!ctx || max_launches < 1 || ctx->c.profiling) return DMS_ERR_INVALID;
  Ctx& c = ctx->c;
  c.ev.assign(2 * static_cast<size_t>(max_launches), nullptr);
  c.ev_kind.assign(static_cast<size_t>(max_launches), 0);
  for (auto& e : c.ev) {
    if (hipEventCreate(&e) != hipSuccess) {
      for (auto& x : c.ev)
        if (x) (void)hipEventDestroy(x);
      c.ev.clear();
      return DMS_ERR_HIP;
    }
  }
  c.ev_used = 0;
  c.profiling = true;
  return DMS_OK;
}

int dms_profile_stop(dms_ctx* ctx, float* ms_out, int* launches_out) {
  if (!ctx || !ctx->c.profiling) return DMS_ERR_INVALID;
  Ctx& c = ctx->c;
  float sum[2] = {0.0f, 0.0f};
  int cnt[2] = {0, 0};
  int rc = DMS_OK;
  for (int i = 0; i + 1 < c.ev_used; i += 2) {
    float ms = 0.0f;
    if (hipEventSynchronize(c.ev[i + 1]) != hipSuccess ||
        hipEventElapsedTime(&ms, c.ev[i], c.ev[i + 1]) != hipSuccess) {
      rc = DMS_ERR_HIP;
      break;
    }
    const int k = c.ev_kind[i / 2];
    sum[k] += ms;
    cnt[k] += 1;
  }
  for (int k = 0; k < 2; ++k) {
    if (ms_out) ms_out[k] = sum[k];
    if (launches_out) launches_out[k] = cnt[k];
  }
  for (auto& e : c.ev) (void)hipEventDestroy(e);
  c.ev.clear();
  c.ev_kind.clear();
  c.ev_used = 0;
  c.profiling = false;
  return rc;
}

const char* dms_strerror(int code) {
  switch (code) {
    case DMS_OK: return "ok";
    case DMS_ERR_INVALID: return "invalid configuration or argument";
    case DMS_ERR_UNSUPPORTED: return "unsupported configuration";
    case DMS_ERR_HIP: return "HIP runtime error";
    case DMS_ERR_OUT_OF_PAGES: return "KV page pool exhausted";
    case DMS_ERR_CAPACITY: return "a head exceeds max_pages_per_head";
    case DMS_ERR_BAD_SEQ: return "sequence id out of range or repeated in one call";
    case DMS_ERR_SCRATCH: return "call too large for the library's static scratch";
    default: return "unknown error code";
  }
}

// ---------------------------------------------------------------------------
// Training-time attention
// ---------------------------------------------------------------------------

static int validate_train_config(const dms_train_config* c) {
  if (!c) return DMS_ERR_INVALID;
  if (c->batch < 1 || c->seq_len < 1 || c->num_kv_heads < 1 || c->group_size < 1 || c->window < 1)
    return DMS_ERR_INVALID;
  if (c->group_size > dms::kMaxGroup) return DMS_ERR_UNSUPPORTED;
  if (c->head_dim != dms::kTrainHeadDim) return DMS_ERR_UNSUPPORTED;
  if (isnan(c->softmax_scale) || (c->softmax_scale > 0.0f && !isfinite(c->softmax_scale)))
    return DMS_ERR_INVALID;
  // element offsets of the largest tensors stay below 2^31 rows of head_dim
  const int64_t rows = static_cast<int64_t>(c->batch) * c->seq_len * c->num_kv_heads * c->group_size;
  if (rows >= (int64_t(1) << 31) / 8) return DMS_ERR_INVALID;
  // one grid row per (sequence, KV head)
  if (static_cast<int64_t>(c->batch) * c->num_kv_heads > 65535) return DMS_ERR_INVALID;
  return DMS_OK;
}

int dms_train_workspace(const dms_train_config* cfg, size_t* workspace_bytes) {
  const int rc = validate_train_config(cfg);
  if (rc) return rc;
  if (workspace_bytes) *workspace_bytes = dms::train_workspace_bytes(*cfg);
  return DMS_OK;
}

int dms_train_attention_fwd(const dms_train_config* cfg, const void* q_dev, const void* k_dev,
                            const void* v_dev, const float* alpha_dev, float* out_dev,
                            float* lse_dev, void* workspace_dev, void* stream) {
  const int rc = validate_train_config(cfg);
  if (rc) return rc;
  if (!q_dev || !k_dev || !v_dev || !alpha_dev || !out_dev || !lse_dev || !workspace_dev)
    return DMS_ERR_INVALID;
  return hip_rc(dms::launch_train_fwd(*cfg, q_dev, k_dev, v_dev, alpha_dev, out_dev, lse_dev,
                                      workspace_dev, as_stream(stream)));
}

int dms_train_attention_bwd(const dms_train_config* cfg, const void* q_dev, const void* k_dev,
                            const void* v_dev, const float* alpha_dev, const float* out_dev,
                            const float* lse_dev, const void* dout_dev, float* dq_dev,
                            float* dk_dev, float* dv_dev, float* dalpha_dev,
                            void* workspace_dev, void* stream) {
  const int rc = validate_train_config(cfg);
  if (rc) return rc;
  if (!q_dev || !k_dev || !v_dev || !alpha_dev || !out_dev || !lse_dev || !dout_dev || !dq_dev ||
      !dk_dev || !dv_dev || !dalpha_dev || !workspace_dev)
    return DMS_ERR_INVALID;
  return hip_rc(dms::launch_train_bwd(*cfg, q_dev, k_dev, v_dev, alpha_dev, out_dev, lse_dev,
                                      dout_dev, dq_dev, dk_dev, dv_dev, dalpha_dev, workspace_dev,
                                      as_stream(stream)));
}

int dms_gumbel_sigmoid_fwd(int n, const float* logits_dev, const float* u_dev, float tau,
                           float* alpha_dev, void* stream) {
  if (n < 0 || !(tau > 0.f) || !isfinite(tau)) return DMS_ERR_INVALID;
  if (n == 0) return DMS_OK;
  if (!logits_dev || !u_dev || !alpha_dev) return DMS_ERR_INVALID;
  return hip_rc(dms::launch_gumbel_fwd(n, logits_dev, u_dev, tau, alpha_dev, as_stream(stream)));
}

int dms_gumbel_sigmoid_bwd(int n, const float* alpha_dev, const float* dalpha_dev, float tau,
                           float* dlogits_dev, void* stream) {
  if (n < 0 || !(tau > 0.f) || !isfinite(tau)) return DMS_ERR_INVALID;
  if (n == 0) return DMS_OK;
  if (!alpha_dev || !dalpha_dev || !dlogits_dev) return DMS_ERR_INVALID;
  return hip_rc(dms::launch_gumbel_bwd(n, alpha_dev, dalpha_dev, tau, dlogits_dev, as_stream(stream)));
}

// ---------------------------------------------------------------------------
// Rotary positions
// ---------------------------------------------------------------------------

static int validate_rope_config(const dms_rope_config* c) {
  if (!c) return DMS_ERR_INVALID;
  if (c->num_kv_heads < 1 || c->group_size < 1 || c->head_dim < 2) return DMS_ERR_INVALID;
  // products of two int32 fit an int64; of three of them only once two are known to be small
  const int64_t heads = static_cast<int64_t>(c->num_kv_heads) * c->group_size;
  if (heads > (int64_t(1) << 20) || heads * c->head_dim > (int64_t(1) << 20)) return DMS_ERR_UNSUPPORTED;
  if (c->rotary_dim < 2 || c->rotary_dim % 2 || c->rotary_offset < 0) return DMS_ERR_INVALID;
  if (c->rotary_dim > c->head_dim || c->rotary_offset > c->head_dim - c->rotary_dim) return DMS_ERR_INVALID;
  if (c->rotary_dim > dms::kMaxRotary) return DMS_ERR_UNSUPPORTED;
  if (c->num_axes < 1 || c->num_axes > dms::kRopeAxes) return DMS_ERR_INVALID;
  if (c->axis_order != DMS_ROPE_SECTIONS && c->axis_order != DMS_ROPE_INTERLEAVED) return DMS_ERR_INVALID;
  if (c->pairing != DMS_ROPE_HALVES && c->pairing != DMS_ROPE_ADJACENT) return DMS_ERR_INVALID;
  int64_t pairs = 0;
  for (int x = 0; x < c->num_axes; ++x) {
    if (c->sections[x] < 0) return DMS_ERR_INVALID;
    if (c->axis_order == DMS_ROPE_INTERLEAVED && c->sections[x] > c->sections[0]) return DMS_ERR_INVALID;
    pairs += c->sections[x];
  }
  if (pairs != c->rotary_dim / 2) return DMS_ERR_INVALID;
  if (c->in_type != DMS_TYPE_BF16 && c->in_type != DMS_TYPE_F32) return DMS_ERR_INVALID;
  if (c->out_type != DMS_TYPE_BF16 && c->out_type != DMS_TYPE_F32) return DMS_ERR_INVALID;
  if (c->borrow != 0 && c->borrow != 1) return DMS_ERR_INVALID;
  if (c->borrow && !isfinite(c->decision_bias)) return DMS_ERR_INVALID;
  if (isnan(c->factor) || isinf(c->factor)) return DMS_ERR_INVALID;
  return DMS_OK;
}

// Tensors of one call: q and k each present with their output or both absent,
// strides no shorter than a row.
static int check_rope_call(const dms_rope_config* c, int tokens, const dms::RopeTensors& t, const void* positions,
                           const void* inv_freq) {
  if (tokens < 0) return DMS_ERR_INVALID;
  const int64_t kv = static_cast<int64_t>(c->num_kv_heads) * c->head_dim, qr = kv * c->group_size;
  if (t.q_stride < qr || t.k_stride < kv || t.q_out_stride < qr || t.k_out_stride < kv) return DMS_ERR_INVALID;
  // a wave per token, four to a workgroup, and a grid of fewer than 2^32 threads
  if (tokens > (1 << 26) - 4 || tokens * (qr + kv) >= int64_t(1) << 38) return DMS_ERR_UNSUPPORTED;
  if (tokens == 0) return DMS_OK;
  if (!t.q != !t.q_out || !t.k != !t.k_out || (!t.q && !t.k) || !positions || !inv_freq) return DMS_ERR_INVALID;
  return DMS_OK;
}

int dms_rope_fwd(const dms_rope_config* cfg, int tokens, const void* q_dev, int64_t q_stride, const void* k_dev,
                 int64_t k_stride, const int32_t* positions_dev, const double* inv_freq_dev, void* q_out_dev,
                 void* k_out_dev, float* logits_out_dev, uint8_t* decisions_out_dev, void* stream) {
  int rc = validate_rope_config(cfg);
  if (rc) return rc;
  const int64_t kv = static_cast<int64_t>(cfg->num_kv_heads) * cfg->head_dim, qr = kv * cfg->group_size;
  const dms::RopeTensors t{q_dev, k_dev, q_out_dev, k_out_dev, q_dev ? q_stride : qr, k_dev ? k_stride : kv, qr, kv};
  if ((rc = check_rope_call(cfg, tokens, t, positions_dev, inv_freq_dev))) return rc;
  if ((logits_out_dev || decisions_out_dev) && !(cfg->borrow && (q_dev || tokens == 0))) return DMS_ERR_INVALID;
  if (tokens == 0) return DMS_OK;
  return hip_rc(dms::launch_rope(*cfg, tokens, t, positions_dev, inv_freq_dev, false, logits_out_dev,
                                 decisions_out_dev, nullptr, as_stream(stream)));
}

int dms_rope_bwd(const dms_rope_config* cfg, int tokens, const void* dq_dev, const void* dk_dev,
                 const int32_t* positions_dev, const double* inv_freq_dev, const float* dlogits_dev,
                 void* dq_out_dev, int64_t dq_stride, void* dk_out_dev, int64_t dk_stride, void* stream) {
  int rc = validate_rope_config(cfg);
  if (rc) return rc;
  const int64_t kv = static_cast<int64_t>(cfg->num_kv_heads) * cfg->head_dim, qr = kv * cfg->group_size;
  const dms::RopeTensors t{dq_dev, dk_dev, dq_out_dev, dk_out_dev, qr, kv, dq_dev ? dq_stride : qr,
                           dk_dev ? dk_stride : kv};
  if ((rc = check_rope_call(cfg, tokens, t, positions_dev, inv_freq_dev))) return rc;
  if (dlogits_dev && !(cfg->borrow && (dq_dev || tokens == 0))) return DMS_ERR_INVALID;
  if (tokens == 0) return DMS_OK;
  return hip_rc(dms::launch_rope(*cfg, tokens, t, positions_dev, inv_freq_dev, true, nullptr, nullptr, dlogits_dev,
                                 as_stream(stream)));
}

// ---------------------------------------------------------------------------
// Attention with a sliding window and sinks
// ---------------------------------------------------------------------------

static int validate_window_config(const dms_window_config* c) {
  if (!c) return DMS_ERR_INVALID;
  if (c->num_seqs < 1 || c->num_seqs > 65535 || c->total_tokens < 0) return DMS_ERR_INVALID;
  if (c->max_seqlen < 0 || c->max_seqlen > c->total_tokens) return DMS_ERR_INVALID;
  if (c->total_tokens > 0 && c->max_seqlen == 0) return DMS_ERR_INVALID;
  if (c->num_kv_heads < 1 || c->group_size < 1 || c->window < 1 || c->sinks < 0) return DMS_ERR_INVALID;
  if (c->group_size > dms::kMaxGroup) return DMS_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return DMS_ERR_UNSUPPORTED;
  if (isnan(c->softmax_scale) || (c->softmax_scale > 0.0f && !isfinite(c->softmax_scale))) return DMS_ERR_INVALID;
  // -lse / scale of a row stays inside float32
  if (c->softmax_scale > 0.0f && c->softmax_scale < 0x1p-100f) return DMS_ERR_INVALID;
  // rows of the query tensors; a grid row per KV head; a token's bytes in 32 bits
  const int64_t heads = static_cast<int64_t>(c->num_kv_heads) * c->group_size;
  if (c->num_kv_heads > 4096 || heads * c->total_tokens >= int64_t(1) << 31) return DMS_ERR_UNSUPPORTED;
  if (!dms::window_grids_fit(*c)) return DMS_ERR_UNSUPPORTED;
  // positions and window ends in int32
  if (static_cast<int64_t>(c->max_seqlen) + std::min(c->window, c->max_seqlen) >= (int64_t(1) << 31) - 1024)
    return DMS_ERR_UNSUPPORTED;
  return DMS_OK;
}

int dms_window_workspace(const dms_window_config* cfg, size_t* workspace_bytes) {
  const int rc = validate_window_config(cfg);
  if (rc) return rc;
  if (workspace_bytes) *workspace_bytes = dms::window_workspace_bytes(*cfg);
  return DMS_OK;
}

// Every tensor present and aligned for 16-byte accesses.
static int check_aligned(std::initializer_list<const void*> tensors) {
  for (const void* p : tensors)
    if (!p || reinterpret_cast<uintptr_t>(p) % 16) return DMS_ERR_INVALID;
  return DMS_OK;
}

int dms_window_attention_fwd(const dms_window_config* cfg, const int32_t* cu_seqlens_dev, const void* q_dev,
                             const void* k_dev, const void* v_dev, void* out_dev, float* lse_dev,
                             void* workspace_dev, void* stream) {
  int rc = validate_window_config(cfg);
  if (rc) return rc;
  if (cfg->total_tokens == 0) return DMS_OK;
  if (!cu_seqlens_dev || !lse_dev || !workspace_dev || reinterpret_cast<uintptr_t>(workspace_dev) % dms::kAlign)
    return DMS_ERR_INVALID;
  if ((rc = check_aligned({q_dev, k_dev, v_dev, out_dev}))) return rc;
  return hip_rc(dms::launch_window_fwd(*cfg, cu_seqlens_dev, q_dev, k_dev, v_dev, out_dev, lse_dev, workspace_dev,
                                       as_stream(stream)));
}

int dms_window_attention_bwd(const dms_window_config* cfg, const int32_t* cu_seqlens_dev, const void* q_dev,
                             const void* k_dev, const void* v_dev, const void* out_dev, const float* lse_dev,
                             const void* dout_dev, void* dq_dev, void* dk_dev, void* dv_dev, void* workspace_dev,
                             void* stream) {
  int rc = validate_window_config(cfg);
  if (rc) return rc;
  if (cfg->total_tokens == 0) return DMS_OK;
  if (!cu_seqlens_dev || !lse_dev || !workspace_dev || reinterpret_cast<uintptr_t>(workspace_dev) % dms::kAlign)
    return DMS_ERR_INVALID;
  if ((rc = check_aligned({q_dev, k_dev, v_dev, out_dev, dout_dev, dq_dev, dk_dev, dv_dev}))) return rc;
  return hip_rc(dms::launch_window_bwd(*cfg, cu_seqlens_dev, q_dev, k_dev, v_dev, lse_dev, dout_dev, dq_dev, dk_dev,
                                       dv_dev, workspace_dev, as_stream(stream)));
}

// ---------------------------------------------------------------------------
// Trees of drafted tokens
// ---------------------------------------------------------------------------

// Sizes of a tree call, host values.
static int check_tree_sizes(const dms_config& c, int n, int total, int max_nodes) {
  if (n < 1 || n > c.max_seqs || total < 0 || max_nodes < 0 || max_nodes > total) return DMS_ERR_INVALID;
  if (total > 0 && max_nodes == 0) return DMS_ERR_INVALID;
  if (max_nodes > dms::kTreeMaxNodes) return DMS_ERR_UNSUPPORTED;
  if (total > static_cast<int64_t>(n) * max_nodes) return DMS_ERR_INVALID;
  // rows of the query tensor in int32; grids of fewer than 2^32 threads: a
  // workgroup of 256 per (head, 32 nodes), and per sequence
  const int64_t heads = static_cast<int64_t>(n) * c.num_kv_heads, words = (max_nodes + 31) / 32;
  if (static_cast<int64_t>(c.num_kv_heads) * c.group_size * total >= int64_t(1) << 31) return DMS_ERR_UNSUPPORTED;
  if (1 + n + heads * std::max<int64_t>(words, 1) >= int64_t(1) << 24) return DMS_ERR_UNSUPPORTED;
  return DMS_OK;
}

int dms_tree_workspace(const dms_config* cfg, int n, int total_nodes, int max_nodes, size_t* workspace_bytes) {
  if (!cfg) return DMS_ERR_INVALID;
  int rc = dms::validate_config(*cfg);
  if (rc) return rc;
  if ((rc = check_tree_sizes(*cfg, n, total_nodes, max_nodes))) return rc;
  if (workspace_bytes) *workspace_bytes = dms::tree_workspace_bytes(*cfg, n, total_nodes, max_nodes);
  return DMS_OK;
}

static int check_tree_call(const dms_ctx* ctx, int layer, int n, const void* seq_ids, const void* cu, int total,
                           int max_nodes) {
  int rc = check_call(ctx, layer, n, seq_ids);
  if (rc) return rc;
  if (!cu) return DMS_ERR_INVALID;
  return check_tree_sizes(ctx->c.cfg, n, total, max_nodes);
}

static bool off_workspace(const void* ws) { return !ws || reinterpret_cast<uintptr_t>(ws) % dms::kAlign; }

static int tree_attention(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev, const int32_t* cu_nodes_dev,
                          int total_nodes, int max_nodes, const int32_t* parents_dev, const void* q_dev,
                          const void* k_dev, const void* v_dev, const uint8_t* flags_dev, uint8_t* decisions_out_dev,
                          bool from_q, void* out_dev, void* workspace_dev, void* stream) {
  int rc = check_tree_call(ctx, layer, n, seq_ids_dev, cu_nodes_dev, total_nodes, max_nodes);
  if (rc) return rc;
  const dms::Ctx& c = ctx->c;
  if (mla(ctx) || c.cfg.eviction != DMS_EVICT_DELAYED) return DMS_ERR_UNSUPPORTED;
  if ((c.cfg.decision_source == DMS_DECIDE_QUERY) != from_q) return DMS_ERR_INVALID;
  if (total_nodes == 0) return DMS_OK;
  if (!parents_dev || (!from_q && !flags_dev) || off_workspace(workspace_dev)) return DMS_ERR_INVALID;
  if ((rc = check_aligned({q_dev, k_dev, v_dev, out_dev}))) return rc;
  return hip_rc(dms::launch_tree_attention(c.cfg, c.lo, c.meta, c.pools[layer], layer, n, seq_ids_dev, cu_nodes_dev,
                                           total_nodes, max_nodes, parents_dev, q_dev, k_dev, v_dev, flags_dev,
                                           decisions_out_dev, out_dev, workspace_dev, as_stream(stream)));
}

int dms_tree_attention(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev, const int32_t* cu_nodes_dev,
                       int total_nodes, int max_nodes, const int32_t* parents_dev, const void* q_dev,
                       const void* k_dev, const void* v_dev, const uint8_t* flags_dev, void* out_dev,
                       void* workspace_dev, void* stream) {
  return tree_attention(ctx, layer, n, seq_ids_dev, cu_nodes_dev, total_nodes, max_nodes, parents_dev, q_dev, k_dev,
                        v_dev, flags_dev, nullptr, false, out_dev, workspace_dev, stream);
}

int dms_tree_attention_q(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev, const int32_t* cu_nodes_dev,
                         int total_nodes, int max_nodes, const int32_t* parents_dev, const void* q_dev,
                         const void* k_dev, const void* v_dev, uint8_t* decisions_out_dev, void* out_dev,
                         void* workspace_dev, void* stream) {
  return tree_attention(ctx, layer, n, seq_ids_dev, cu_nodes_dev, total_nodes, max_nodes, parents_dev, q_dev, k_dev,
                        v_dev, nullptr, decisions_out_dev, true, out_dev, workspace_dev, stream);
}

int dms_tree_accept(int n, const int32_t* cu_nodes_dev, int total_nodes, int max_nodes, const int32_t* parents_dev,
                    const int32_t* tokens_dev, const int32_t* targets_dev, const int32_t* first_dev,
                    int32_t* path_out_dev, int32_t* path_len_out_dev, int32_t* next_out_dev, void* stream) {
  if (n < 1 || n > dms::kMaxSeqs || total_nodes < 0 || max_nodes < 0 || max_nodes > total_nodes) return DMS_ERR_INVALID;
  if (total_nodes > 0 && max_nodes == 0) return DMS_ERR_INVALID;
  if (max_nodes > dms::kTreeMaxNodes) return DMS_ERR_UNSUPPORTED;
  if (total_nodes > static_cast<int64_t>(n) * max_nodes) return DMS_ERR_INVALID;
  if (!cu_nodes_dev || !path_len_out_dev || !next_out_dev) return DMS_ERR_INVALID;
  if (total_nodes > 0 && (!parents_dev || !tokens_dev || !targets_dev || !path_out_dev)) return DMS_ERR_INVALID;
  return hip_rc(dms::launch_tree_accept(n, cu_nodes_dev, total_nodes, max_nodes, parents_dev, tokens_dev, targets_dev,
                                        first_dev, path_out_dev, path_len_out_dev, next_out_dev, as_stream(stream)));
}

int dms_tree_commit(dms_ctx* ctx, int layer, int n, const int32_t* seq_ids_dev, const int32_t* cu_nodes_dev,
                    int total_nodes, int max_nodes, const int32_t* path_dev, const int32_t* path_len_dev,
                    const void* k_dev, const void* v_dev, const uint8_t* flags_dev, void* workspace_dev, void* stream) {
  int rc = check_tree_call(ctx, layer, n, seq_ids_dev, cu_nodes_dev, total_nodes, max_nodes);
  if (rc) return rc;
  if (total_nodes == 0) return DMS_OK;
  if (!path_dev || !path_len_dev || !flags_dev || off_workspace(workspace_dev)) return DMS_ERR_INVALID;
  const dms::Ctx& c = ctx->c;
  if ((rc = check_aligned({k_dev, mla(ctx) ? k_dev : v_dev}))) return rc;
  hipError_t e = dms::launch_tree_commit(c.cfg, c.lo, c.meta, c.pools[layer], layer, n, seq_ids_dev, cu_nodes_dev,
                                         total_nodes, max_nodes, path_dev, path_len_dev, k_dev, v_dev, flags_dev,
                                         workspace_dev, as_stream(stream));
  // page retrieval: a path may write into any page of a head (reused slots)
  if (e == hipSuccess && c.cfg.quest_page_budget > 0)
    e = dms::launch_quest_bounds(c.cfg, c.lo, c.meta, c.ws, c.pools[layer], layer, n, true, seq_ids_dev,
                                 as_stream(stream));
  return hip_rc(e);
}

// ---------------------------------------------------------------------------
// Sampling
// ---------------------------------------------------------------------------

static int validate_sample_config(const dms_sample_config* c, int rows) {
  if (!c || c->vocab < 1 || rows < 0) return DMS_ERR_INVALID;
  if (c->logits_type != DMS_TYPE_BF16 && c->logits_type != DMS_TYPE_F32) return DMS_ERR_INVALID;
  if (c->vocab > dms::kSampleMaxVocab) return DMS_ERR_UNSUPPORTED;
  // grids of fewer than 2^32 threads
  if (rows >= 1 << 20) return DMS_ERR_UNSUPPORTED;
  return DMS_OK;
}

int dms_sample_workspace(const dms_sample_config* cfg, int rows, size_t* workspace_bytes) {
  const int rc = validate_sample_config(cfg, rows);
  if (rc) return rc;
  if (workspace_bytes) *workspace_bytes = dms::sample_workspace_bytes(*cfg, rows);
  return DMS_OK;
}

int dms_sample(const dms_sample_config* cfg, int rows, const void* logits_dev, int64_t row_stride,
               const float* temperature_dev, const int32_t* top_k_dev, const float* top_p_dev, const float* min_p_dev,
               const float* u_dev, int32_t* tokens_out_dev, float* logprobs_out_dev, void* workspace_dev,
               void* stream) {
  const int rc = validate_sample_config(cfg, rows);
  if (rc) return rc;
  // (offsets in bytes stay inside int64)
  if (row_stride < cfg->vocab || row_stride >= int64_t(1) << 40) return DMS_ERR_INVALID;
  if (rows == 0) return DMS_OK;
  if (!logits_dev || !u_dev || !tokens_out_dev || off_workspace(workspace_dev)) return DMS_ERR_INVALID;
  if (reinterpret_cast<uintptr_t>(logits_dev) % (cfg->logits_type == DMS_TYPE_BF16 ? 2 : 4)) return DMS_ERR_INVALID;
  return hip_rc(dms::launch_sample(*cfg, rows, logits_dev, row_stride, temperature_dev, top_k_dev, top_p_dev, min_p_dev,
                                   u_dev, tokens_out_dev, logprobs_out_dev, workspace_dev, as_stream(stream)));
}

}  // extern "C"
