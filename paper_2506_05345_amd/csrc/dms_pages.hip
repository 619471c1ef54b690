// Copies of whole sequences (forks) and compaction of a layer's page pool.
//
// Both move pages between places of one pool and are bound by HBM: a fork reads
// the live tiles of a source and writes them once per copy, a compaction reads
// and writes the live pages past the live count.  The host does not know the
// retained lengths, so a one-workgroup plan per layer leaves prefix sums in the
// workspace and the copy kernel's workgroups take equal shares of them.
//
// Measured, one layer of 8 heads, d = 128, two pools in turn: 8 prompts of 32K
// tokens into 120 chains (2.0 GB), 8192 workgroups writing past the caches 396 us
// (5.1 TB/s; 357 at the shortest, 385 on one pool); 2048 of them 446, 16384 412,
// 8 copies to a read 405, cached writes 461.  85 live of 128 chains compacted
// (1.5 GB): 293 us with 24K workgroups, 311 with 8192, 329 with 2048.  A plain
// copy of 2 GiB reaches 5.1 TB/s, a fill 6.8.
#include <algorithm>

#include "dms_ops.h"

namespace dms {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int kPlanThreads = 1024;
constexpr int kCopyThreads = 256;
constexpr int kShare = 4;          // adjacent copies of one source that share its reads
constexpr int kPieces = 4;         // 16-byte pieces a thread has in flight
constexpr int kForkGroups = 8192;     // workgroups of a fork's copies, of a compaction's
constexpr int kCompactGroups = 32768;
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

// Copies are not read again by the call: written past the caches.
__device__ inline void store_past(char* p, u32x4 x) { __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(p)); }

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
    const size_t so = static_cast<size_t>(a.src[i]) * p.H + h;
    const int L = s.len[so];
    // the copies of this row: their heads and first pages in the call's block
    size_t sd[kShare];
    const int32_t* pages[kShare];
    bool on[kShare];
#pragma unroll
    for (int c = 0; c < kShare; ++c) {
      on[c] = c == 0 || (on[c - 1] && (i + c) % kShare != 0 && i + c < a.n && a.src[i + c] == a.src[i]);
      const int ic = on[c] ? i + c : i;
      sd[c] = static_cast<size_t>(a.dst[ic]) * p.H + h;
      pages[c] = s.stack + first + base[static_cast<size_t>(ic) * p.H + h];
    }
    for (; t < min(t1, c1); ++t) {
      const int k = t - c0;   // tile of the head
      const int pg = k / tpp;
      const size_t in_page = static_cast<size_t>(k - pg * tpp) * p.tile_bytes;
      const int from_page = s.pt[so * p.maxp + pg];
      const char* from = pool + static_cast<size_t>(from_page) * p.page_bytes + in_page;
      char* to[kShare];
#pragma unroll
      for (int c = 0; c < kShare; ++c)
        to[c] = on[c] ? pool + static_cast<size_t>(pages[c][pg]) * p.page_bytes + in_page : nullptr;
      for (int e0 = 0; e0 < p.tile_bytes; e0 += kPieces * 16 * kCopyThreads) {
        u32x4 x[kPieces];
#pragma unroll
        for (int n = 0; n < kPieces; ++n) {
          const int e = e0 + 16 * (n * kCopyThreads + tid);
          if (e < p.tile_bytes) x[n] = *reinterpret_cast<const u32x4*>(from + e);
        }
#pragma unroll
        for (int c = 0; c < kShare; ++c)
          if (on[c])
#pragma unroll
            for (int n = 0; n < kPieces; ++n) {
              const int e = e0 + 16 * (n * kCopyThreads + tid);
              if (e < p.tile_bytes) store_past(to[c] + e, x[n]);
            }
      }
#pragma unroll
      for (int c = 0; c < kShare; ++c) {
        if (!on[c]) continue;
        if (tid < kTile && kTile * k + tid < L)
          s.slot_meta[sd[c] * p.max_slots + kTile * k + tid] = s.slot_meta[so * p.max_slots + kTile * k + tid];
        if (in_page == 0) {
          const int page = pages[c][pg];
          if (tid == 0) s.pt[sd[c] * p.maxp + pg] = page;
          if (16 * tid < p.bounds_bytes)
            *reinterpret_cast<u32x4*>(s.bounds + static_cast<size_t>(page) * p.bounds_bytes + 16 * tid) =
                *reinterpret_cast<const u32x4*>(s.bounds + static_cast<size_t>(from_page) * p.bounds_bytes + 16 * tid);
        }
        if (k == 0) {
          for (int e = tid; e < p.w; e += kCopyThreads) s.ring[sd[c] * p.w + e] = s.ring[so * p.w + e];
          if (tid == 0) {
            s.len[sd[c]] = L;
            if (h == 0) s.pos[sd[c] / p.H] = s.pos[a.src[i]];
          }
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Compaction
// ---------------------------------------------------------------------------

struct CompactArgs {
  PagesArgs p;
  int32_t* lists;          // [layers of the context][list_stride]: see CompactLists
  size_t list_stride;
  int32_t* used_out;       // nullable, one entry per layer of the call
  int out0;                // entry of the launch's first layer
};

// A layer's part of the workspace, U live pages: the free ids below U in
// ascending order, of every 32 ids which are live and at least U, and how many
// such ids come before them.  There are as many live ids past U as free ones
// below it, and the r-th of these takes the r-th of those.
struct CompactLists {
  int32_t* holes;
  uint32_t* live;
  int32_t* before;
};
__device__ inline CompactLists lists_of(const CompactArgs& a, int y) {
  int32_t* b = a.lists + static_cast<size_t>(a.p.layer + y) * a.list_stride;
  const int words = (a.p.num_pages + 31) / 32;
  return CompactLists{b, reinterpret_cast<uint32_t*>(b + a.p.num_pages / 2 + 1), b + a.p.num_pages / 2 + 1 + words};
}
__device__ inline int moved_to(const CompactLists& l, int id) {   // of a live id >= U
  const uint32_t below = l.live[id >> 5] & ((1u << (id & 31)) - 1);
  return l.holes[l.before[id >> 5] + __builtin_popcount(below)];
}

__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(CompactArgs a) {
  __shared__ uint32_t freed[kIdChunk / 32];
  __shared__ int lds[34];
  const PagesArgs& p = a.p;
  if (__syncthreads_or(load_status(p.status) != 0)) return;
  const LayerPtrs s = layer_ptrs(p, blockIdx.x);
  const CompactLists l = lists_of(a, blockIdx.x);
  const int top = *s.top, U = p.num_pages - top;
  if (threadIdx.x == 0 && a.used_out) a.used_out[a.out0 + blockIdx.x] = U;
  int holes = 0, moved = 0;
  for (int64_t c0 = 0; c0 < p.num_pages; c0 += kIdChunk) {
    const int ids = static_cast<int>(min<int64_t>(kIdChunk, p.num_pages - c0));
    for (int i = threadIdx.x; i < (ids + 31) / 32; i += kPlanThreads) freed[i] = 0;
    __syncthreads();
    for (int i0 = threadIdx.x; i0 < top; i0 += 8 * kPlanThreads) {
      int id[8];
#pragma unroll
      for (int n = 0; n < 8; ++n) id[n] = s.stack[min(i0 + n * kPlanThreads, top - 1)];   // past the end: the last one again
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        const int64_t x = id[n] - c0;
        if (x >= 0 && x < ids) atomicOr(&freed[x >> 5], 1u << (x & 31));
      }
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
      }
      int2 tot;
      const int2 ex = block_exclusive_scan2(make_int2(__builtin_popcount(hole), __builtin_popcount(live)), lds, &tot);
      if (32 * wi < ids) {
        l.live[id0 >> 5] = live;
        l.before[id0 >> 5] = moved + ex.y;
      }
      for (int r = holes + ex.x; hole; hole &= hole - 1) l.holes[r++] = static_cast<int32_t>(id0 + __builtin_ctz(hole));
      holes += tot.x;
      moved += tot.y;
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(kCopyThreads) void compact_move_kernel(CompactArgs a) {
  const PagesArgs& p = a.p;
  if (load_status(p.status) != 0) return;
  const LayerPtrs s = layer_ptrs(p, blockIdx.y);
  const CompactLists l = lists_of(a, blockIdx.y);
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
      if (id >= U) s.pt[hh * p.maxp + k] = moved_to(l, id);
    }
  }
  // pages, a workgroup each
  for (int64_t id = U + static_cast<int64_t>(blockIdx.x); id < p.num_pages; id += gridDim.x) {
    if (!(l.live[id >> 5] >> (id & 31) & 1)) continue;
    const int to = moved_to(l, static_cast<int>(id));
    const char* from = pool + static_cast<size_t>(id) * p.page_bytes;
    char* dst = pool + static_cast<size_t>(to) * p.page_bytes;
    for (size_t e0 = 0; e0 < p.page_bytes; e0 += kPieces * 16 * kCopyThreads) {
      u32x4 x[kPieces];
#pragma unroll
      for (int n = 0; n < kPieces; ++n) {
        const size_t e = e0 + 16 * (n * kCopyThreads + tid);
        if (e < p.page_bytes) x[n] = *reinterpret_cast<const u32x4*>(from + e);
      }
#pragma unroll
      for (int n = 0; n < kPieces; ++n) {
        const size_t e = e0 + 16 * (n * kCopyThreads + tid);
        if (e < p.page_bytes) store_past(dst + e, x[n]);
      }
    }
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

PagesLayout layout_of(const dms_config& c, const Layout& lo) {
  const size_t heads = lo.max_heads;
  return pages_layout(c, heads, lo.workspace_bytes - pages_layout(c, heads, 0).bytes);
}

}  // namespace

PagesLayout pages_layout(const dms_config& c, size_t max_heads, size_t at) {
  PagesLayout l{};
  const size_t layers = c.num_layers, words = (static_cast<size_t>(c.num_pages) + 31) / 32;
  size_t off = at;
  auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, kAlign); return o; };
  l.fk_base = take(layers * max_heads * 4);
  l.fk_tiles = take(layers * (max_heads + 1) * 4);
  l.fk_block = take(layers * 8);
  l.cp_list_stride = static_cast<size_t>(c.num_pages) / 2 + 1 + 2 * words;
  l.cp_lists = take(layers * l.cp_list_stride * 4);
  l.bytes = off - at;
  return l;
}

hipError_t launch_seq_fork(const dms_config& c, const Layout& lo, void* meta, void* ws, void* const* pools,
                           int layer, int n, const int32_t* src, const int32_t* dst, hipStream_t st) {
  ForkArgs a{};
  char* w = static_cast<char*>(ws);
  a.p = pages_args(c, lo, meta);
  a.src = src;
  a.dst = dst;
  a.n = n;
  a.nh_max = static_cast<size_t>(lo.max_heads);
  const PagesLayout l = layout_of(c, lo);
  a.base = reinterpret_cast<int32_t*>(w + l.fk_base);
  a.tiles = reinterpret_cast<int32_t*>(w + l.fk_tiles);
  a.block = reinterpret_cast<int32_t*>(w + l.fk_block);
  hipError_t e = over_layers(c, a.p, pools, layer, [&](int, int layers) {
    hipLaunchKernelGGL(fork_plan_kernel, dim3(layers), dim3(kPlanThreads), 0, st, a);
  });
  if (e != hipSuccess) return e;
  // at most a workgroup for every tile that the rows can hold where kShare copies share each of them.  Distinct
  // sources get a fourth of one per tile: 4 prompts of 400 tokens, 2 heads, then take 21 us instead of 17, but 28
  // layers of one such prompt copied 4 times 25 instead of 26.5, and 16 prompts of 2000 tokens, 8 heads, 28 instead
  // of 32 (evicting heads hold an eighth of the tiles that their page tables could).
  const int64_t rows = (static_cast<int64_t>(n) + kShare - 1) / kShare * c.num_kv_heads;
  const int64_t most = rows * c.max_pages_per_head * (c.page_size / kTile);
  return over_layers(c, a.p, pools, layer, [&](int, int layers) {
    const int64_t x = std::min<int64_t>(most, std::max(1, kForkGroups / layers));
    hipLaunchKernelGGL(fork_copy_kernel, dim3(static_cast<unsigned>(x), layers), dim3(kCopyThreads), 0, st, a);
  });
}

hipError_t launch_compact(const dms_config& c, const Layout& lo, void* meta, void* ws, void* const* pools,
                          int layer, int32_t* used_out, hipStream_t st) {
  CompactArgs a{};
  a.p = pages_args(c, lo, meta);
  const PagesLayout l = layout_of(c, lo);
  a.lists = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + l.cp_lists);
  a.list_stride = l.cp_list_stride;
  a.used_out = used_out;
  return over_layers(c, a.p, pools, layer, [&](int y, int layers) {
    a.out0 = y - std::max(layer, 0);
    hipLaunchKernelGGL(compact_plan_kernel, dim3(layers), dim3(kPlanThreads), 0, st, a);
    const int x = std::min(std::max(c.num_pages / 4, 64), std::max(1, kCompactGroups / layers));
    hipLaunchKernelGGL(compact_move_kernel, dim3(x, layers), dim3(kCopyThreads), 0, st, a);
  });
}

}  // namespace dms
