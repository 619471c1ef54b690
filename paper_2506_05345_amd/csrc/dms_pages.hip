// Copies of whole sequences (forks) and compaction of a layer's page pool.
//
// Both move pages between places of one pool and are bound by HBM: a fork reads
// the live tiles of a source and writes them once per copy, a compaction reads
// and writes the live pages past the live count.  The host does not know the
// retained lengths, so a one-workgroup plan per layer leaves prefix sums in the
// workspace and the copy kernel's workgroups take equal shares of them.
#include <algorithm>

#include "dms_ops.h"

namespace dms {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int kPlanThreads = 1024;
constexpr int kCopyThreads = 256;
constexpr int kShare = 4;          // adjacent copies of one source that share its reads
constexpr int kIdChunk = 1 << 18;  // page ids marked at a time in LDS

__device__ inline int load_status(const int32_t* status) { return __atomic_load_n(status, __ATOMIC_RELAXED); }

__device__ inline int64_t wave_inclusive_scan64(int64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t u = __shfl_up(v, off, 64);
    if (lane >= off) v += u;
  }
  return v;
}

// Exclusive prefix sum of 64-bit counts across kPlanThreads threads (copies of
// one large sequence can add to more pages than an int32 holds before the call
// is refused); `lds` holds 17 values.
__device__ inline int64_t plan_scan(int64_t v, int64_t* lds, int64_t* total) {
  const int lane = threadIdx.x & 63, wid = threadIdx.x >> 6;
  const int64_t inc = wave_inclusive_scan64(v);
  if (lane == 63) lds[wid] = inc;
  __syncthreads();
  if (threadIdx.x == 0) {
    int64_t run = 0;
    for (int i = 0; i < kPlanThreads / 64; ++i) {
      const int64_t t = lds[i];
      lds[i] = run;
      run += t;
    }
    lds[16] = run;
  }
  __syncthreads();
  const int64_t ex = lds[wid] + inc - v;
  *total = lds[16];
  __syncthreads();
  return ex;
}

struct PagesArgs {
  char* meta;
  size_t layer0, layer_stride;
  size_t pos, len, ring, page_table, slot_meta, stack, top, page_bounds;
  int32_t* status;
  int H, w, P, maxp, max_slots, max_seqs, num_pages;
  int layer;               // first layer of the launch (state regions)
  int bounds_bytes;        // page bounds of one page, 0 when off
  size_t page_bytes;
  int tile_bytes;
  char* pools[kPageLayers];   // of the launch's layers
};

struct LayerPtrs {
  int32_t *pos, *len, *ring, *pt, *slot_meta, *stack, *top;
  char* bounds;
};

__device__ inline LayerPtrs layer_ptrs(const PagesArgs& a, int y) {
  char* b = a.meta + a.layer0 + static_cast<size_t>(a.layer + y) * a.layer_stride;
  return LayerPtrs{reinterpret_cast<int32_t*>(b + a.pos),        reinterpret_cast<int32_t*>(b + a.len),
                   reinterpret_cast<int32_t*>(b + a.ring),       reinterpret_cast<int32_t*>(b + a.page_table),
                   reinterpret_cast<int32_t*>(b + a.slot_meta),  reinterpret_cast<int32_t*>(b + a.stack),
                   reinterpret_cast<int32_t*>(b + a.top),        b + a.page_bounds};
}

// ---------------------------------------------------------------------------
// Fork
// ---------------------------------------------------------------------------

struct ForkArgs {
  PagesArgs p;
  const int32_t* src;
  const int32_t* dst;
  int n;
  size_t nh_max;
  // per layer of the context (index: layer * nh_max or nh_max + 1)
  int32_t* base;           // first page of each (pair, head) inside the call's block
  int32_t* tiles;          // tiles before each (pair, head) of the copy kernel's list, then the total
  int32_t* block;          // [2 * layer]: block's first stack entry, block's pages
};

// Pairs i .. i + kShare - 1 of an aligned group read their source together where
// it is the same as the pair's before: the first of them carries the row.
__device__ inline bool leads(const ForkArgs& a, int i) { return i % kShare == 0 || a.src[i] != a.src[i - 1]; }

// Checks of the whole call and, for one layer per workgroup, the pages and tiles
// before every (pair, head).  Nothing of the state changes here: the copy kernel
// runs only if no layer's workgroup found an error.
__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(ForkArgs a) {
  __shared__ uint32_t seen[kMaxSeqs / 32];
  __shared__ int64_t lds[17];
  const PagesArgs& p = a.p;
  const LayerPtrs s = layer_ptrs(p, blockIdx.x);
  const int layer = p.layer + blockIdx.x;
  const int top0 = *s.top;
  if (__syncthreads_or(load_status(p.status) != 0)) return;
  for (int i = threadIdx.x; i < (p.max_seqs + 31) / 32; i += blockDim.x) seen[i] = 0;
  __syncthreads();
  int bad = 0;
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    const int d = a.dst[i], o = a.src[i];
    if (d < 0 || d >= p.max_seqs || o < 0 || o >= p.max_seqs) {
      bad = 1;
      continue;
    }
    const uint32_t bit = 1u << (d & 31);
    if (atomicOr(&seen[d >> 5], bit) & bit) bad = 1;
    if (s.pos[d] != 0) bad = 1;
  }
  bad = __syncthreads_or(bad);
  if (!bad) {
    for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
      const int o = a.src[i];
      if (seen[o >> 5] >> (o & 31) & 1) bad = 1;
    }
    bad = __syncthreads_or(bad);
  }
  if (bad) {
    if (threadIdx.x == 0) set_status(p.status, DMS_ERR_BAD_SEQ);
    return;
  }
  const int64_t NH = static_cast<int64_t>(a.n) * p.H;
  int32_t* base = a.base + layer * a.nh_max;
  int32_t* tiles = a.tiles + layer * (a.nh_max + 1);
  int64_t pages = 0, run = 0;
  for (int64_t b = 0; b < NH; b += blockDim.x) {
    const int64_t hh = b + threadIdx.x;
    int np = 0, nt = 0;
    if (hh < NH) {
      const int i = static_cast<int>(hh / p.H);
      const int L = s.len[static_cast<size_t>(a.src[i]) * p.H + hh % p.H];
      np = (L + p.P - 1) / p.P;
      nt = leads(a, i) ? (L + kTile - 1) / kTile : 0;
    }
    int64_t tot, tot_t;
    const int64_t ex = plan_scan(np, lds, &tot), ext = plan_scan(nt, lds, &tot_t);
    if (hh < NH) {
      base[hh] = static_cast<int32_t>(pages + ex);
      tiles[hh] = static_cast<int32_t>(run + ext);
    }
    pages += tot;
    run += tot_t;
    if (pages > top0) break;   // uniform; the sums stay below 2^31 up to here
  }
  if (pages > top0) {
    if (threadIdx.x == 0) set_status(p.status, DMS_ERR_OUT_OF_PAGES);
    return;
  }
  if (threadIdx.x == 0) {
    tiles[NH] = static_cast<int32_t>(run);
    a.block[2 * layer] = top0 - static_cast<int>(pages);
    a.block[2 * layer + 1] = static_cast<int>(pages);
  }
}

// Workgroup x of a layer copies an equal share of the layer's list of tiles:
// each tile is read once and written to the copies that share the row.
__global__ __launch_bounds__(kCopyThreads) void fork_copy_kernel(ForkArgs a) {
  const PagesArgs& p = a.p;
  if (load_status(p.status) != 0) return;
  const LayerPtrs s = layer_ptrs(p, blockIdx.y);
  const int layer = p.layer + blockIdx.y;
  char* pool = p.pools[blockIdx.y];
  const int tid = threadIdx.x;
  const int NH = a.n * p.H;
  const int32_t* base = a.base + layer * a.nh_max;
  const int32_t* tiles = a.tiles + layer * (a.nh_max + 1);
  const int first = a.block[2 * layer];
  if (blockIdx.x == 0 && tid == 0) *s.top = first;
  const int64_t total = tiles[NH];
  const int t0 = static_cast<int>(blockIdx.x * total / gridDim.x), t1 = static_cast<int>((blockIdx.x + 1) * total / gridDim.x);
  if (t0 >= t1) return;
  int hh = 0, hi = NH - 1;   // last row that starts at or before t0: it holds tile t0
  while (hh < hi) {
    const int mid = (hh + hi + 1) >> 1;
    if (tiles[mid] <= t0) hh = mid; else hi = mid - 1;
  }
  const int tpp = p.P / kTile;
  int t = t0;
  while (t < t1) {
    const int c0 = tiles[hh], c1 = tiles[hh + 1];
    if (t >= c1) {           // rows without tiles of their own
      ++hh;
      continue;
    }
    const int i = hh / p.H, h = hh - i * p.H;
    int copies = 1;
    while ((i + copies) % kShare != 0 && i + copies < a.n && a.src[i + copies] == a.src[i]) ++copies;
    const size_t so = static_cast<size_t>(a.src[i]) * p.H + h;
    const int L = s.len[so];
    for (; t < min(t1, c1); ++t) {
      const int k = t - c0;   // tile of the head
      const char* from = pool + static_cast<size_t>(s.pt[so * p.maxp + k / tpp]) * p.page_bytes +
                         static_cast<size_t>(k % tpp) * p.tile_bytes;
      char* to[kShare];
      for (int c = 0; c < copies; ++c) {
        const int page = s.stack[first + base[static_cast<size_t>(i + c) * p.H + h] + k / tpp];
        to[c] = pool + static_cast<size_t>(page) * p.page_bytes + static_cast<size_t>(k % tpp) * p.tile_bytes;
        const size_t sd = static_cast<size_t>(a.dst[i + c]) * p.H + h;
        if (k % tpp == 0) {
          if (tid == 0) s.pt[sd * p.maxp + k / tpp] = page;
          if (p.bounds_bytes) {
            const char* bf = s.bounds + static_cast<size_t>(s.pt[so * p.maxp + k / tpp]) * p.bounds_bytes;
            char* bt = s.bounds + static_cast<size_t>(page) * p.bounds_bytes;
            if (16 * tid < p.bounds_bytes) *reinterpret_cast<u32x4*>(bt + 16 * tid) = *reinterpret_cast<const u32x4*>(bf + 16 * tid);
          }
        }
        if (tid < kTile && kTile * k + tid < L)
          s.slot_meta[sd * p.max_slots + kTile * k + tid] = s.slot_meta[so * p.max_slots + kTile * k + tid];
        if (k == 0) {
          for (int e = tid; e < p.w; e += kCopyThreads) s.ring[sd * p.w + e] = s.ring[so * p.w + e];
          if (tid == 0) {
            s.len[sd] = L;
            if (h == 0) s.pos[a.dst[i + c]] = s.pos[a.src[i]];
          }
        }
      }
      for (int e = 16 * tid; e < p.tile_bytes; e += 16 * kCopyThreads) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(from + e);
        for (int c = 0; c < copies; ++c) *reinterpret_cast<u32x4*>(to[c] + e) = x;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Compaction
// ---------------------------------------------------------------------------

struct CompactArgs {
  PagesArgs p;
  int32_t* map;            // [layers of the context][num_pages]
  int32_t* used_out;       // nullable, one entry per layer of the call
  int out0;                // entry of the launch's first layer
};

// map[id] = where live page id >= U goes, -1 for free ids >= U (U live pages).
// Below U the map holds the free ids in ascending order meanwhile: there are as
// many of them as live ids past U.
__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(CompactArgs a) {
  __shared__ uint32_t freed[kIdChunk / 32];
  __shared__ int lds[34];
  const PagesArgs& p = a.p;
  if (__syncthreads_or(load_status(p.status) != 0)) return;
  const LayerPtrs s = layer_ptrs(p, blockIdx.x);
  int32_t* map = a.map + static_cast<size_t>(p.layer + blockIdx.x) * p.num_pages;
  const int top = *s.top, U = p.num_pages - top;
  if (threadIdx.x == 0 && a.used_out) a.used_out[a.out0 + blockIdx.x] = U;
  int holes = 0, moved = 0;
  for (int64_t c0 = 0; c0 < p.num_pages; c0 += kIdChunk) {
    const int ids = static_cast<int>(min<int64_t>(kIdChunk, p.num_pages - c0));
    for (int i = threadIdx.x; i < (ids + 31) / 32; i += blockDim.x) freed[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < top; i += blockDim.x) {
      const int64_t id = s.stack[i] - c0;
      if (id >= 0 && id < ids) atomicOr(&freed[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    // 1024 words at a time, a word per thread
    for (int w0 = 0; 32 * w0 < ids; w0 += kPlanThreads) {
      const int wi = w0 + threadIdx.x;
      const int64_t id0 = c0 + 32 * static_cast<int64_t>(wi);
      uint32_t hole = 0, live = 0;
      if (32 * wi < ids) {
        const uint32_t in = ids - 32 * wi >= 32 ? ~0u : (1u << (ids - 32 * wi)) - 1;
        const uint32_t low = U - id0 >= 32 ? ~0u : U - id0 <= 0 ? 0u : (1u << (U - id0)) - 1;   // ids below U
        hole = freed[wi] & in & low;
        live = ~freed[wi] & in & ~low;
        for (uint32_t f = freed[wi] & in & ~low; f; f &= f - 1) map[id0 + __builtin_ctz(f)] = -1;
      }
      int2 tot;
      const int2 ex = block_exclusive_scan2(make_int2(__builtin_popcount(hole), __builtin_popcount(live)), lds, &tot);
      int r = holes + ex.x;
      for (; hole; hole &= hole - 1) map[r++] = static_cast<int32_t>(id0 + __builtin_ctz(hole));
      r = moved + ex.y;
      for (; live; live &= live - 1) map[id0 + __builtin_ctz(live)] = r++;
      holes += tot.x;
      moved += tot.y;
    }
    __syncthreads();
  }
  __threadfence_block();
  __syncthreads();
  for (int64_t id = U + static_cast<int64_t>(threadIdx.x); id < p.num_pages; id += blockDim.x) {
    const int r = map[id];
    if (r >= 0) map[id] = map[r];
  }
}

__global__ __launch_bounds__(kCopyThreads) void compact_move_kernel(CompactArgs a) {
  const PagesArgs& p = a.p;
  if (load_status(p.status) != 0) return;
  const LayerPtrs s = layer_ptrs(p, blockIdx.y);
  const int32_t* map = a.map + static_cast<size_t>(p.layer + blockIdx.y) * p.num_pages;
  char* pool = p.pools[blockIdx.y];
  const int top = *s.top, U = p.num_pages - top;
  const int tid = threadIdx.x, lane = tid & 63;
  const int64_t g0 = static_cast<int64_t>(blockIdx.x) * kCopyThreads + tid, gs = static_cast<int64_t>(gridDim.x) * kCopyThreads;
  for (int64_t i = g0; i < top; i += gs) s.stack[i] = p.num_pages - 1 - static_cast<int>(i);
  // page tables, a wave per head
  const int64_t heads = static_cast<int64_t>(p.max_seqs) * p.H;
  for (int64_t hh = blockIdx.x * (kCopyThreads / 64) + (tid >> 6); hh < heads; hh += gridDim.x * (kCopyThreads / 64)) {
    const int np = (s.len[hh] + p.P - 1) / p.P;
    for (int k = lane; k < np; k += 64) {
      const int id = s.pt[hh * p.maxp + k];
      if (id >= U) s.pt[hh * p.maxp + k] = map[id];
    }
  }
  // pages, a workgroup each
  for (int64_t id = U + static_cast<int64_t>(blockIdx.x); id < p.num_pages; id += gridDim.x) {
    const int to = map[id];
    if (to < 0) continue;
    const char* from = pool + static_cast<size_t>(id) * p.page_bytes;
    char* dst = pool + static_cast<size_t>(to) * p.page_bytes;
    for (size_t e = 16 * tid; e < p.page_bytes; e += 16 * kCopyThreads)
      *reinterpret_cast<u32x4*>(dst + e) = *reinterpret_cast<const u32x4*>(from + e);
    if (16 * tid < p.bounds_bytes)
      *reinterpret_cast<u32x4*>(s.bounds + static_cast<size_t>(to) * p.bounds_bytes + 16 * tid) =
          *reinterpret_cast<const u32x4*>(s.bounds + static_cast<size_t>(id) * p.bounds_bytes + 16 * tid);
  }
}

PagesArgs pages_args(const dms_config& c, const Layout& lo, void* meta) {
  PagesArgs p{};
  p.meta = static_cast<char*>(meta);
  p.layer0 = lo.layer0;
  p.layer_stride = lo.layer_stride;
  p.pos = lo.pos;
  p.len = lo.len;
  p.ring = lo.ring;
  p.page_table = lo.page_table;
  p.slot_meta = lo.slot_meta;
  p.stack = lo.stack;
  p.top = lo.top;
  p.page_bounds = lo.page_bounds;
  p.status = reinterpret_cast<int32_t*>(p.meta + lo.status);
  p.H = c.num_kv_heads;
  p.w = c.window;
  p.P = c.page_size;
  p.maxp = c.max_pages_per_head;
  p.max_slots = lo.max_slots;
  p.max_seqs = c.max_seqs;
  p.num_pages = c.num_pages;
  p.bounds_bytes = lo.page_bounds ? 4 * c.head_dim : 0;
  p.page_bytes = lo.page_bytes;
  p.tile_bytes = static_cast<int>(lo.page_bytes / (c.page_size / kTile));
  return p;
}

// Runs `launch(first layer, layers)` over the call's layers, kPageLayers at a time.
template <typename F>
hipError_t over_layers(const dms_config& c, PagesArgs& p, void* const* pools, int layer, F launch) {
  const int end = layer < 0 ? c.num_layers : layer + 1;
  for (int y = std::max(layer, 0); y < end; y += kPageLayers) {
    const int count = std::min(kPageLayers, end - y);
    p.layer = y;
    for (int i = 0; i < count; ++i) p.pools[i] = static_cast<char*>(pools[y + i]);
    launch(y, count);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_seq_fork(const dms_config& c, const Layout& lo, void* meta, void* ws, void* const* pools,
                           int layer, int n, const int32_t* src, const int32_t* dst, hipStream_t st) {
  ForkArgs a{};
  char* w = static_cast<char*>(ws);
  a.p = pages_args(c, lo, meta);
  a.src = src;
  a.dst = dst;
  a.n = n;
  a.nh_max = static_cast<size_t>(lo.max_heads);
  a.base = reinterpret_cast<int32_t*>(w + lo.ws_fk_base);
  a.tiles = reinterpret_cast<int32_t*>(w + lo.ws_fk_tiles);
  a.block = reinterpret_cast<int32_t*>(w + lo.ws_fk_block);
  hipError_t e = over_layers(c, a.p, pools, layer, [&](int, int layers) {
    hipLaunchKernelGGL(fork_plan_kernel, dim3(layers), dim3(kPlanThreads), 0, st, a);
  });
  if (e != hipSuccess) return e;
  return over_layers(c, a.p, pools, layer, [&](int, int layers) {
    hipLaunchKernelGGL(fork_copy_kernel, dim3(std::max(1, 2048 / layers), layers), dim3(kCopyThreads), 0, st, a);
  });
}

hipError_t launch_compact(const dms_config& c, const Layout& lo, void* meta, void* ws, void* const* pools,
                          int layer, int32_t* used_out, hipStream_t st) {
  CompactArgs a{};
  a.p = pages_args(c, lo, meta);
  a.map = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + lo.ws_cp_map);
  a.used_out = used_out;
  return over_layers(c, a.p, pools, layer, [&](int y, int layers) {
    a.out0 = y - std::max(layer, 0);
    hipLaunchKernelGGL(compact_plan_kernel, dim3(layers), dim3(kPlanThreads), 0, st, a);
    hipLaunchKernelGGL(compact_move_kernel, dim3(std::max(1, 2048 / layers), layers), dim3(kCopyThreads), 0, st, a);
  });
}

}  // namespace dms
