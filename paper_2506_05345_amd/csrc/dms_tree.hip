// Trees of drafted tokens over the cache, gfx950: attention of every node over
// the retained slots and its own ancestors, the accepted path of a tree, and
// the append of that path.
//
// Node x of a sequence at position pos (tokens appended so far) stands at
// t = pos + depth(x), and sees
//   a live slot of its KV head iff its token is not flagged or younger than w:
//     flag = 0 or p > t - w (the delayed eviction that the tokens between would
//     have done);
//   the nodes on the path from the root to itself, by the same rule with their
//   own flags.
// Nothing is appended: a commit later appends the rows of one path.
//
// Attention is a split-K flash decode whose columns are the (node, query head)
// pairs of a KV head.  Every launch of a call is small and fixed by the host;
// what only the device knows (lengths) goes through the flat list of tiles:
//   tree_prep_kernel    ancestors of every node as bits, depths, the drafted
//                       rows as tiles in the pool's layout (8-bit pages: in
//                       their stored form), prefix sums of the heads' tiles;
//   tree_attn_kernel    U workgroups, of 128 columns at most, take a part of the list;
//   tree_merge_kernel   joins the heads that several parts attended.
// Times below are of kernels on one MI355X; the sizes: "deep" 48 sequences of 8 KV heads
// at 32768 tokens (8 times fewer kept) with trees of 12 nodes, 60 columns a head; "wide" 8
// of those with 64 nodes, 320 columns.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "dms_common.h"
#include "dms_draft.h"
#include "dms_fp8.h"
#include "dms_tiles.h"

namespace dms {
namespace {

#define DMS_CONST __attribute__((address_space(4)))

constexpr float kRescale = 8.0f;       // lazy rescale threshold, log2 units
constexpr float kMInit = -1.0e30f;     // running max before the first visible key
constexpr int kPrepThreads = 256;

__device__ inline int load_status(const int32_t* status) { return __atomic_load_n(status, __ATOMIC_RELAXED); }

// One (sequence, KV head) of a call.
struct __attribute__((aligned(32))) TreeRow {
  int sh, L, tok0, m, p0, tile0, seq, pad;   // state head, live slots, first node, nodes, position, first tile of the tree
};

// One equal part of a call's tiles: the first head's row beside it, so that a
// workgroup starts with one load.
struct __attribute__((aligned(64))) TreePart {
  int tb, te, hh, c0;      // flat tiles [tb, te), the head that holds tb, its first flat tile
  TreeRow r;
};

struct TreeArgs {
  int32_t* status;
  const int32_t* seq_ids;
  const int32_t* cu;
  const int32_t* parents;
  const uint16_t* q;       // [total, Hq, D]
  const uint16_t* k;       // [total, H, D]
  const uint16_t* v;
  const uint8_t* flags;    // [total, H]; with decisions from q: written by the preparation
  uint8_t* flags_out;      // the same, or null
  const char* pool;
  const int32_t* page_table;
  const int32_t* slot_meta;
  const int32_t* len;
  const int32_t* pos;
  uint16_t* out;           // [total, Hq, D] bf16
  TreeRow* rows;           // [n * H]
  int32_t* cum;            // [n * H + 1] flat tiles before each head
  TreePart* part;          // [cells] (te = tb: no such part)
  int2* head_parts;        // [n * H] first and last part of each head
  uint32_t* anc;           // [total][words] ancestors and itself, bit a: node a of its tree
  int32_t* depth;          // [total]
  int32_t* deepest;        // [n]
  char* tiles;             // [H][tph] tiles of the drafted rows
  uint32_t* tmeta;         // [H][tph][32] their rows (position | flag << 31), as the pool's slot owners
  float* part_o;           // [2 cells U][UC][D]: the sums of a part's first and last head
  float2* part_ml;         // [2 cells U][UC] their maxima and denominators
  size_t page_bytes;
  int n, H, g, w, P, log2P, maxp, max_slots, max_seqs, total, max_nodes, words, tph;
  int cells, U, UC, min_tiles;   // parts at most, units (workgroups) to a part, columns of a unit, least tiles of a part
  int zero_neuron;
  int once;                // every tile is read by one workgroup
  float bias, scale_log2;
};

__device__ inline int tiles_of(int L, int m) { return m ? ((L + 31) >> 5) + ((m + 31) >> 5) : 0; }
// Parts that share `total` flat tiles, and where part w begins.
__device__ inline int parts_of(int total, int min_tiles, int cells) { return max(1, min(cells, total / min_tiles)); }
__device__ inline int part_begin(int w, int total, int parts) {
  return static_cast<int>(static_cast<int64_t>(w) * total / parts);
}
__device__ inline int part_holding(int tile, int total, int parts) {
  return static_cast<int>((static_cast<int64_t>(tile + 1) * parts - 1) / total);
}

// ---------------------------------------------------------------------------
// Preparation
// ---------------------------------------------------------------------------

// Block 0: the call's ids and sizes are checked, the heads described, their tiles
// summed and cut into parts:
//   few tiles in all: every head into slices of its own, of min_tiles or so, so that a
//     workgroup starts and ends one head only (16 heads of 78 tiles: 18.7 us, cut
//     without regard to heads 26.5);
//   many: equal parts of the flat list whatever heads they meet, so that ragged heads
//     cannot unbalance the chip.
constexpr int kPlanHeads = 512;    // heads that the plan holds in LDS
__device__ inline TreeRow tree_row(const TreeArgs& a, int hh) {
  const int i = hh / a.H, s = a.seq_ids[i], c0 = a.cu[i];
  TreeRow r;
  r.sh = s * a.H + hh % a.H;
  r.L = a.len[r.sh];
  r.tok0 = c0;
  r.m = a.cu[i + 1] - c0;
  r.p0 = a.pos[s];
  r.tile0 = (hh % a.H) * a.tph + c0 / 32 + i;
  r.seq = i;
  r.pad = 0;
  return r;
}
__device__ void tree_plan(const TreeArgs& a) {
  __shared__ union {
    uint32_t seen[kMaxSeqs / 32];
    TreeRow rows[kPlanHeads];
  } u;
  __shared__ int cum[kPlanHeads], first[kPlanHeads], lds[17];
  for (int i = threadIdx.x; i < (a.max_seqs + 31) / 32; i += blockDim.x) u.seen[i] = 0;
  __syncthreads();
  int bad_id = 0, bad = 0;
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    const int s = a.seq_ids[i], c0 = a.cu[i], c1 = a.cu[i + 1];
    if (s < 0 || s >= a.max_seqs) bad_id = 1;
    else if (atomicOr(&u.seen[s >> 5], 1u << (s & 31)) & (1u << (s & 31))) bad_id = 1;
    bad |= c0 < 0 || c1 < c0 || c1 > a.total || c1 - c0 > a.max_nodes;
    bad |= (i == 0 && c0 != 0) || (i == a.n - 1 && c1 != a.total);
  }
  bad_id = __syncthreads_or(bad_id);
  bad = __syncthreads_or(bad);
  if (bad_id || bad) {
    if (threadIdx.x == 0) set_status(a.status, bad_id ? DMS_ERR_BAD_SEQ : DMS_ERR_INVALID);
    return;
  }
  const int NH = a.n * a.H;
  const bool held = NH <= kPlanHeads;     // rows and sums in LDS for what follows
  int total = 0;
  for (int base = 0; base < NH; base += blockDim.x) {
    const int hh = base + threadIdx.x;
    int tiles = 0;
    if (hh < NH) {
      const TreeRow r = tree_row(a, hh);
      a.rows[hh] = r;
      if (held) u.rows[hh] = r;
      tiles = tiles_of(r.L, r.m);
    }
    int tot;
    const int ex = block_exclusive_scan(tiles, lds, &tot);
    if (hh < NH) {
      a.cum[hh] = total + ex;
      if (held) cum[hh] = total + ex;
    }
    total += tot;
  }
  if (threadIdx.x == 0) a.cum[NH] = total;
  __syncthreads();
  if (held && total < 2 * a.min_tiles * a.cells && NH <= a.cells / 2) {
    // slices of ceil(total / (cells - NH)) tiles at most, min_tiles at least: no more than cells of them
    const int slice = max(a.min_tiles, (total + a.cells - NH - 1) / (a.cells - NH));
    int run = 0;
    for (int base = 0; base < NH; base += blockDim.x) {
      const int hh = base + threadIdx.x;
      const int ns = hh < NH ? (tiles_of(u.rows[hh].L, u.rows[hh].m) + slice - 1) / slice : 0;
      int tot;
      const int w0 = run + block_exclusive_scan(ns, lds, &tot);
      if (hh < NH) {
        first[hh] = w0;
        a.head_parts[hh] = make_int2(w0, w0 + ns - 1);
      }
      run += tot;
    }
    __syncthreads();
    for (int w = threadIdx.x; w < a.cells; w += blockDim.x) {
      int lo = 0, hi = NH - 1;      // the last head whose first part is not past w: one with tiles
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= w) lo = mid; else hi = mid - 1;
      }
      const TreeRow r = u.rows[lo];
      const int T = tiles_of(r.L, r.m), ns = (T + slice - 1) / slice, s = w - first[lo];
      TreePart* p = a.part + w;
      p->tb = w < run ? cum[lo] + part_begin(s, T, ns) : 0;
      p->te = w < run ? cum[lo] + part_begin(s + 1, T, ns) : 0;
      p->hh = lo;
      p->c0 = cum[lo];
      p->r = r;
    }
    return;
  }
  const int parts = parts_of(total, a.min_tiles, a.cells);
  for (int w = threadIdx.x; w < a.cells; w += blockDim.x) {
    const bool on = w < parts && total > 0;
    const int tb = on ? part_begin(w, total, parts) : 0, te = on ? part_begin(w + 1, total, parts) : 0;
    int lo = 0, hi = NH - 1;      // the last head whose first tile is not past tb
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if ((held ? cum[mid] : a.cum[mid]) <= tb) lo = mid; else hi = mid - 1;
    }
    TreePart* p = a.part + w;
    p->tb = tb;
    p->te = te;
    p->hh = lo;
    p->c0 = held ? cum[lo] : a.cum[lo];
    p->r = held ? u.rows[lo] : tree_row(a, lo);
  }
  for (int hh = threadIdx.x; hh < NH; hh += blockDim.x) {
    const int c0 = a.cum[hh], c1 = a.cum[hh + 1];
    a.head_parts[hh] = c1 > c0 ? make_int2(part_holding(c0, total, parts), part_holding(c1 - 1, total, parts)) : make_int2(0, 0);
  }
}

// The next n blocks: ancestors of a sequence's nodes.  Bits and jumps double
// until every node's jump has left the tree (at most 8 rounds of 256 nodes, where
// a walk up a chain would take as many dependent reads as nodes).
__device__ void tree_ancestors(const TreeArgs& a, int i) {
  __shared__ uint32_t bits[kTreeMaxNodes][kTreeWords + 1];   // (odd stride: rows spread over the banks)
  __shared__ int jump[kTreeMaxNodes];
  __shared__ int deepest;
  const int tok0 = max(0, min(a.cu[i], a.total)), end = max(tok0, min(a.cu[i + 1], a.total));
  const int m = min(end - tok0, a.max_nodes);
  const int x = threadIdx.x;
  if (x == 0) deepest = 0;
  int mine = -1;
  if (x < m) {
    mine = a.parents[tok0 + x];
    if (mine < -1 || mine >= x) {
      set_status(a.status, DMS_ERR_INVALID);
      mine = -1;
    }
    for (int u = 0; u < a.words; ++u) bits[x][u] = 0;
    bits[x][x >> 5] = 1u << (x & 31);
    jump[x] = mine;
  }
  __syncthreads();
  for (int span = 1; span < m; span *= 2) {
    uint32_t add[kTreeWords];
    int next = -1;
    const int j = x < m ? jump[x] : -1;
    if (j >= 0) {
      next = jump[j];
#pragma unroll
      for (int u = 0; u < kTreeWords; ++u) add[u] = u < a.words ? bits[j][u] : 0u;
    }
    __syncthreads();
    if (j >= 0) {
#pragma unroll
      for (int u = 0; u < kTreeWords; ++u)
        if (u < a.words) bits[x][u] |= add[u];
      jump[x] = next;
    }
    __syncthreads();
  }
  if (x < m) {
    int d = -1;
    for (int u = 0; u < a.words; ++u) {
      const uint32_t b = bits[x][u];
      d += __popc(b);
      a.anc[static_cast<size_t>(tok0 + x) * a.words + u] = b;
    }
    a.depth[tok0 + x] = d;
    atomicMax(&deepest, d);
  }
  __syncthreads();
  if (x == 0) a.deepest[i] = deepest;
}

// The other blocks: 32 drafted rows of one KV head as a tile; rows past the tree
// are 0.
template <int D, bool FP8>
__device__ void tree_tile(const TreeArgs& a, int hh, int k) {
  __shared__ uint16_t vrows[32][D + 2];
  __shared__ int up[kTreeMaxNodes];
  const int i = hh / a.H, h = hh % a.H, tid = threadIdx.x, s = a.seq_ids[i];
  const int tok0 = a.cu[i], m = a.cu[i + 1] - tok0;
  if (tok0 < 0 || m < 0 || m > a.max_nodes || m > a.total - tok0 || 32 * k >= m || s < 0 || s >= a.max_seqs) return;
  const int tile0 = h * a.tph + tok0 / 32 + i + k;
  for (int x = tid; x < 32 * k + 32 && x < m; x += kPrepThreads) up[x] = a.parents[tok0 + x];
  __syncthreads();
  if (tid < 32) {
    const int x = 32 * k + tid;
    uint32_t row = 0;
    if (x < m) {
      const size_t node = static_cast<size_t>(tok0) + x;
      bool flag;
      if (a.flags_out != nullptr) {
        const uint32_t bits = a.q[(node * a.H + h) * a.g * D];
        flag = (__uint_as_float(bits << 16) + a.bias) > 0.f;
        a.flags_out[node * a.H + h] = flag;
      } else {
        flag = a.flags[node * a.H + h] != 0;
      }
      int depth = 0;
      for (int y = up[x], last = x; y >= 0 && y < last; last = y, y = up[y]) ++depth;   // (parents that break the rules end it)
      row = static_cast<uint32_t>(a.pos[s] + depth) | (flag ? kFlagBit : 0u);
    }
    a.tmeta[static_cast<size_t>(tile0) * 32 + tid] = row;
  }
  constexpr int kPieces = 32 * D / 8;
  char* tile = a.tiles + static_cast<size_t>(tile0) * (FP8 ? fp8_tile_bytes(D) : tile_bytes(D));
  for (int pc = tid; pc < kPieces; pc += kPrepThreads) {
    const int j = pc / (D / 8), part = pc % (D / 8), e0 = 8 * part;
    uint4 kx = make_uint4(0u, 0u, 0u, 0u), vx = make_uint4(0u, 0u, 0u, 0u);
    if (32 * k + j < m) {
      const size_t row = ((static_cast<size_t>(tok0) + 32 * k + j) * a.H + h) * D + e0;
      kx = *reinterpret_cast<const uint4*>(a.k + row);
      vx = *reinterpret_cast<const uint4*>(a.v + row);
    }
    if constexpr (FP8) {
      fp8_store_token(tile, j, D, part, kx, vx);
    } else {
      *reinterpret_cast<uint4*>(tile + k_elem_off(j, e0)) = kx;
      const uint32_t vw[4] = {vx.x, vx.y, vx.z, vx.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) vrows[j][e0 + e] = static_cast<uint16_t>(vw[e >> 1] >> (16 * (e & 1)));
    }
  }
  if constexpr (!FP8) {
    __syncthreads();
    // value piece x: dim x / 4, rows 8 (x % 4) .. + 7
    for (int x = tid; x < kPieces; x += kPrepThreads) {
      const int e = x >> 2, j0 = 8 * (x & 3);
      u32x4 p;
#pragma unroll
      for (int t = 0; t < 4; ++t)
        p[t] = static_cast<uint32_t>(vrows[j0 + 2 * t][e]) | (static_cast<uint32_t>(vrows[j0 + 2 * t + 1][e]) << 16);
      *reinterpret_cast<u32x4*>(tile + v_elem_off(j0, e, D)) = p;
    }
  }
}

// One launch for all of it, bound by the plan's chain of dependent loads (ids, sizes,
// lengths, parts): 5.4 us with one sequence, 6.3 with 64 heads, 10 with 384.
template <int D, bool FP8>
__global__ __launch_bounds__(kPrepThreads) void tree_prep_kernel(TreeArgs a) {
  if (load_status(a.status) != 0) return;
  const unsigned b = blockIdx.x;
  if (b == 0) {
    tree_plan(a);
  } else if (b <= static_cast<unsigned>(a.n)) {
    tree_ancestors(a, b - 1);
  } else {
    const unsigned x = b - 1 - a.n;
    tree_tile<D, FP8>(a, x / a.words, x % a.words);
  }
}

// ---------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------

// How the four waves of a workgroup share a unit's columns (32 to a wave) and
// tiles: CW side by side over the columns, KW = 4 / CW over the tiles.  Tiles go
// through LDS by hardware copies, as they are stored: the products read their
// operands from there, so that the registers are left to queries and sums, and
// two workgroups fit a compute unit, each attending while the other waits.
//   CW = 1: every wave attends tiles of its own and never waits for another
//     before the end of a segment.  A tile's keys are copied as soon as the
//     products have read those of the tile R before, its values likewise.
//   CW = 2: stages of KW tiles in a ring of S, one barrier a stage.
//   CW = 4: a wave attends the two tiles of a stage together (TPS), their chains
//     of products and exponentials side by side.
// Deep calls are bound by memory: 165 us for 0.85 GB, 5.1 TB/s, what a large copy reaches;
// while tiles stream it is 7, the rest goes into a segment's start and its fold.  Wide ones
// are bound by the chain of a step (scores, maximum, exponentials, values) at two waves a
// SIMD: 82 us, 0.55 PFLOP/s, matrix units busy 28 % of it.  Two column blocks a wave, for
// half the LDS reads, leave one wave a SIMD: 159 us.  Three 2-wave workgroups a compute unit
// for CW = 2: 168 against 166.  Parts of 4 or 16 tiles at least: no faster than 8.
template <int D, bool FP8, int CW_>
struct Shape {
  static constexpr int CW = CW_, NW = 4, KW = NW / CW, UC = 32 * CW;
  static constexpr bool PRIVATE = CW == 1;
  static constexpr int kTile = FP8 ? D * 64 + 256 : D * 128;      // a stored tile
  static constexpr int kFold = 32 * D * 4;                        // a wave's block of float32 sums
  static constexpr int kSlots = FP8 ? 8 : 4;                      // tiles in LDS
  static constexpr int TPS = CW == 4 ? 2 : 1;
  static constexpr int R = kSlots / NW, S = kSlots / (KW * TPS);
  static constexpr int kWaveBytes = R * kTile > kFold ? R * kTile : kFold;
  static constexpr int kLds = NW * kWaveBytes;
  __device__ static constexpr int slot_at(int slot) { return PRIVATE ? slot / R * kWaveBytes + slot % R * kTile : slot * kTile; }
};

__device__ inline void copy16_once(const void* src, uint32_t m0) {   // a tile that this wave alone reads
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off nt" : : "s"(m0), "v"(src) : "memory", "m0", "vcc");
}
__device__ inline void copy4(const void* src, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, off" : : "s"(m0), "v"(src) : "memory", "m0", "vcc");
}
__device__ inline u32x4 lds16(uint32_t at) { return *reinterpret_cast<DMS_LDS const u32x4*>(at); }
__device__ inline u32x2 lds8(uint32_t at) { return *reinterpret_cast<DMS_LDS const u32x2*>(at); }

// 8 E4M3 codes to bf16 times a power of two (exact)
__device__ inline u32x4 f8_bf16x8(uint32_t w0, uint32_t w1, float scale) {
  u32x4 o;
  o[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false));
  o[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true));
  o[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false));
  o[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true));
  return o;
}

// Byte offsets of the lane's first key and value piece in a tile, and of its
// scales (8-bit pages).  The 32x32x16 products take
//   keys: lane l of k-step s dims 16 s + 8 (l / 32) .. + 7 of row row_token(l % 32);
//   values: lane l of (32-dim block b, half y) rows 16 y + 8 (l / 32) .. + 7 of
//     dim 32 b + l % 32.
struct LaneAt {
  uint32_t k, v, ks, vs;
};
template <int D, bool FP8>
__device__ inline LaneAt lane_at(int lane) {
  const int hf = lane >> 5, kt = row_token(lane & 31), h = (kt >> 2) & 1, r = 4 * (kt >> 3) + (kt & 3);
  LaneAt at;
  at.k = h * 1024 + hf * 256 + r * 16;
  if (FP8) {
    at.v = D * 32 + hf * 256 + (lane & 15) * 16 + 8 * ((lane >> 4) & 1);
    at.ks = D * 64 + (kt >> 3) * 64 + (kt & 7) * 4;
    at.vs = D * 64 + hf * 64 + 32;
  } else {
    at.v = D * 64 + ((lane >> 4) & 1) * 1024 + hf * 256 + (lane & 15) * 16;
    at.ks = at.vs = 0;
  }
  return at;
}

template <int D, bool FP8>
__device__ inline u32x4 value_operand(uint32_t tile, const LaneAt& at, int b, int y) {
  if constexpr (FP8) {
    const u32x2 c = lds8(tile + at.v + b * 1024 + y * 512);
    return f8_bf16x8(c[0], c[1], 1.0f);
  } else {
    return lds16(tile + at.v + b * 2048 + y * 512);
  }
}
// value (row j, dim e) of a tile in LDS; an 8-bit one without its scale
template <int D, bool FP8>
__device__ inline float stored_value(uint32_t tile, int j, int e) {
  if constexpr (FP8) {
    const int code = *reinterpret_cast<DMS_LDS const uint8_t*>(tile + static_cast<uint32_t>(fp8_v_off(j, e, D)));
    return __builtin_amdgcn_cvt_f32_fp8(code, 0);
  } else {
    return __uint_as_float(static_cast<uint32_t>(*reinterpret_cast<DMS_LDS const uint16_t*>(tile + static_cast<uint32_t>(v_elem_off(j, e, D)))) << 16);
  }
}

// A segment of a part: tiles t0 .. t1 - 1 of head hh.
struct Segment {
  int sh, L, tok0, m, p0, tile0;     // see TreeRow
  int hh, t0, t1, T, nc, deep;
};

// The state of a wave's 32 columns; lane l: column l % 32.
template <int D>
struct Columns {
  u32x4 q[D / 16];
  f32x16 o[D / 32];
  float m, l;
  int t;                 // position of the column's node
  const uint32_t* anc;   // its ancestors, one word per tile of the tree
};

// Rows of tile t that some column does not see, and what that takes.
struct TileMask {
  bool masked, tree;
  uint32_t alive, old, odd;   // rows there; flagged and old enough for the deepest node; values not finite
};

// The tile's rows whose values are not finite.
template <int D, bool FP8>
__device__ __forceinline__ uint32_t odd_rows(uint32_t tile, int lane) {
  const LaneAt at = lane_at<D, FP8>(fresh(lane));
  uint32_t mine = 0;
#pragma unroll 1
  for (int z = 0; z < D / 16; ++z) {
    const int b = z >> 1, y = z & 1;
    const u32x4 v = value_operand<D, FP8>(tile, at, b, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t x = (v[e >> 1] >> (16 * (e & 1))) & 0x7F80u;
      mine |= (x == 0x7F80u ? 1u : 0u) << (16 * y + e);
    }
  }
  mine <<= 8 * (lane >> 5);
#pragma unroll
  for (int off = 32; off; off >>= 1) mine |= __shfl_xor(mine, off, 64);
  return __builtin_amdgcn_readfirstlane(mine);
}

// CAREFUL: a hidden row takes part in the products with weight 0, and 0 times an
// infinity or NaN is NaN.  Sums that end finite met none.  Where they do not, the
// segment is attended again with the rows whose values are not finite found (odd),
// zeroed in the products, and added by hand to the columns that see them.  (Slots past
// the live length, whose values may be anything, are zeroed in LDS beforehand.)
template <int D, bool FP8, bool CAREFUL>
__device__ __forceinline__ TileMask tile_mask(const TreeArgs& a, const Segment& sg, uint32_t meta, uint32_t tile, int t, int lane) {
  TileMask k;
  k.tree = t >= sg.nc;
  const int rows = t >= sg.t1 ? 0 : k.tree ? sg.m - 32 * (t - sg.nc) : sg.L - 32 * t;
  k.alive = rows >= 32 ? ~0u : (1u << rows) - 1u;
  const bool soon = (meta & kFlagBit) != 0 && sg.deep - static_cast<int>(meta & ~kFlagBit) >= a.w;
  k.old = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(soon)) & k.alive;
  k.masked = k.tree || k.old != 0 || k.alive != ~0u;
  k.odd = 0;
  if (CAREFUL && k.masked) k.odd = odd_rows<D, FP8>(tile, lane) & k.alive;
  return k;
}

// Zeroes the values (8-bit pages: and their scales) of rows `valid` on of a tile in
// LDS; threads t, t + n, ..
template <int D, bool FP8>
__device__ inline void zero_values(uint32_t tile, int valid, int t, int n) {
  for (int P = t; P < D * (FP8 ? 2 : 4); P += n) {
    const int nv = valid - 8 * ((P >> 4) & 3);       // rows of this 16-byte piece that stay
    if (nv >= 8) continue;
    u32x4 keep;
    if (FP8) {       // two dims of eight codes
      const uint64_t k8 = nv <= 0 ? 0ull : ~0ull >> (8 * (8 - nv));
      keep = u32x4{static_cast<uint32_t>(k8), static_cast<uint32_t>(k8 >> 32), static_cast<uint32_t>(k8), static_cast<uint32_t>(k8 >> 32)};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) keep[e] = (2 * e < nv ? 0x0000FFFFu : 0u) | (2 * e + 1 < nv ? 0xFFFF0000u : 0u);
    }
    auto* x = reinterpret_cast<DMS_LDS u32x4*>(tile + D * (FP8 ? 32 : 64) + P * 16);
    *x = *x & keep;
  }
  if (FP8 && t >= valid && t < 32) *reinterpret_cast<DMS_LDS float*>(tile + static_cast<uint32_t>(fp8_vs_off(t, D))) = 0.f;
}

constexpr int kAhead = 4;   // products between an operand's LDS read and its use

// Scores of TPS tiles; their chains of products take turns.
template <int D, bool FP8, int TPS>
__device__ __forceinline__ void tile_scores(const Columns<D>& c, f32x16 (&s)[TPS], const uint32_t (&tile)[TPS], const LaneAt& at) {
  constexpr int KS = D / 16;
#pragma unroll
  for (int x = 0; x < TPS; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[x][i] = 0.f;
  if constexpr (FP8) {
    float ks[TPS];
#pragma unroll
    for (int x = 0; x < TPS; ++x) ks[x] = *reinterpret_cast<DMS_LDS const float*>(tile[x] + at.ks);
    // piece (p, y) of 16 codes holds k-steps 4 p + y and 4 p + 2 + y
    u32x4 op[2];
    auto read = [&](int e) { return lds16(tile[e % TPS] + at.k + (e / TPS >> 1) * 2048 + (e / TPS & 1) * 512); };
    op[0] = read(0);
    op[1] = read(1);
#pragma unroll
    for (int e = 0; e < TPS * KS / 2; ++e) {
      const u32x4 raw = op[e & 1];
      if (e + 2 < TPS * KS / 2) op[e & 1] = read(e + 2);
      const int x = e % TPS, p = e / TPS;
      s[x] = mfma(f8_bf16x8(raw[0], raw[1], ks[x]), c.q[4 * (p >> 1) + (p & 1)], s[x]);
      s[x] = mfma(f8_bf16x8(raw[2], raw[3], ks[x]), c.q[4 * (p >> 1) + 2 + (p & 1)], s[x]);
    }
  } else {
    u32x4 op[kAhead];
    auto read = [&](int e) { return lds16(tile[e % TPS] + at.k + (e / TPS >> 1) * 2048 + (e / TPS & 1) * 512); };
#pragma unroll
    for (int e = 0; e < kAhead; ++e) op[e] = read(e);
#pragma unroll
    for (int e = 0; e < TPS * KS; ++e) {
      __builtin_amdgcn_sched_barrier(0);
      s[e % TPS] = mfma(op[e % kAhead], c.q[e / TPS], s[e % TPS]);
      if (e + kAhead < TPS * KS) op[e % kAhead] = read(e + kAhead);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Rows whose values are not finite, added to the columns that see them.
template <int D, bool FP8>
__device__ __forceinline__ void odd_values(Columns<D>& c, const u32x4 (&pu)[2], uint32_t vis, uint32_t odd, uint32_t tile, int lane) {
  for (uint32_t left = odd; left; left &= left - 1) {
    const int j = __builtin_ctz(left), ln = fresh(lane);
    uint32_t pair = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i == (8 * (j >> 4) + (j & 7)) >> 1) pair = pu[i >> 2][i & 3];
    float pj = __uint_as_float(j & 1 ? pair & 0xFFFF0000u : pair << 16);
    pj = __shfl(pj, (ln & 31) + 32 * ((j >> 3) & 1), 64);
    const bool seen = (vis >> j) & 1;
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float val = stored_value<D, FP8>(tile, j, 32 * b + 8 * (i >> 2) + 4 * (ln >> 5) + (i & 3));
        c.o[b][i] = seen ? fmaf(pj, val, c.o[b][i]) : c.o[b][i];
        asm volatile("" ::: "memory");     // one value at a time: this is rare, its registers are not
      }
  }
}

// TPS tiles from the products' scores on: masks, running maximum and sum, weights
// and the products with the values.  keys_done() once nothing but the values (and,
// for 8-bit pages, the values' scales) is read any more, values_ready() before
// those are.
template <int D, bool FP8, int TPS, bool CAREFUL, class KeysDone, class ValuesReady>
__device__ __forceinline__ void attend_tiles(const TreeArgs& a, const Segment& sg, Columns<D>& c, const uint32_t (&tile)[TPS],
                                             const uint32_t (&meta)[TPS], int t, const LaneAt& at, int lane, KeysDone keys_done,
                                             ValuesReady values_ready) {
  constexpr int OB = D / 32;
  const int hf = lane >> 5;
  const float sl2 = a.scale_log2, thr = kRescale / sl2;
  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
  f32x16 s[TPS];
  tile_scores<D, FP8, TPS>(c, s, tile, at);
  keys_done();
  if (CAREFUL) values_ready();
  TileMask k[TPS];
  uint32_t vis[TPS];
#pragma unroll
  for (int x = 0; x < TPS; ++x) {
    k[x] = tile_mask<D, FP8, CAREFUL>(a, sg, meta[x], tile[x], t + x, lane);
    vis[x] = ~0u;
    if (k[x].masked) {
      vis[x] = k[x].alive;
      if (k[x].tree && k[x].alive) vis[x] &= c.anc[t + x - sg.nc];
      for (uint32_t left = k[x].old; left; left &= left - 1) {
        const int j = __builtin_ctz(left);
        const int kp = static_cast<int>(__builtin_amdgcn_readlane(static_cast<int>(meta[x]), j) & ~kFlagBit);
        if (c.t - kp >= a.w) vis[x] &= ~(1u << j);
      }
      const uint32_t mine = vis[x] >> (8 * hf);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[x][i] = (mine >> (16 * (i >> 3) + (i & 7))) & 1 ? s[x][i] : -INFINITY;
    }
  }
  float mx = s[0][0];
#pragma unroll
  for (int x = 0; x < TPS; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[x][i]);
  mx = col_max(mx);
  const bool raise = mx > c.m + thr;   // false while the column has seen no key
  if (__builtin_amdgcn_ballot_w64(raise)) {
    const float m_new = raise ? mx : c.m;
    const float alpha = __builtin_amdgcn_exp2f((c.m - m_new) * sl2);
    c.l *= alpha;
#pragma unroll
    for (int b = 0; b < OB; ++b) c.o[b] *= alpha;
    c.m = m_new;
  }
  // weights 2^((s - m) scale), rounded to bf16 for the products; the
  // denominator adds the rounded values, so that one dominant key returns its
  // value row exactly.  8-bit pages: the weight of the product carries the
  // value scale, a power of two, so that its rounding is the same
  const float mb = c.m * sl2;
  u32x4 pu[TPS][2];
  auto weight_pair = [&](int x, int j) {
    f32x2 pr = {__builtin_amdgcn_exp2f(fmaf(s[x][2 * j], sl2, -mb)), __builtin_amdgcn_exp2f(fmaf(s[x][2 * j + 1], sl2, -mb))};
    const bf16x2 pb = __builtin_convertvector(pr, bf16x2);
    c.l = __builtin_amdgcn_fdot2_f32_bf16(pb, ones, c.l, false);
    if constexpr (FP8) {
      const f32x2 vs = *reinterpret_cast<DMS_LDS const f32x2*>(tile[x] + at.vs + (j >> 2) * 128 + (j & 3) * 8);
      pr[0] *= vs[0];
      pr[1] *= vs[1];
      pu[x][j >> 2][j & 3] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, bf16x2));
    } else {
      pu[x][j >> 2][j & 3] = __builtin_bit_cast(uint32_t, pb);
    }
  };
#pragma unroll
  for (int j = 0; j < 8; ++j) weight_pair(0, j);
  if (!CAREFUL) values_ready();
  if constexpr (CAREFUL) {
#pragma unroll
    for (int x = 0; x < TPS; ++x) {
      if (x > 0)
#pragma unroll
        for (int j = 0; j < 8; ++j) weight_pair(x, j);
      const uint32_t mine = (k[x].alive & ~k[x].odd) >> (8 * hf);
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        u32x4 keep;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t bit = mine >> (16 * y + 2 * e);
          keep[e] = ((bit & 1) ? 0x0000FFFFu : 0u) | ((bit & 2) ? 0xFFFF0000u : 0u);
        }
#pragma unroll
        for (int b = 0; b < OB; ++b) c.o[b] = mfma(value_operand<D, FP8>(tile[x], at, b, y) & keep, pu[x][y], c.o[b]);
      }
      if (k[x].odd) odd_values<D, FP8>(c, pu[x], vis[x], k[x].odd, tile[x], lane);
    }
    return;
  }
  // product e: tile e / (2 OB), row half (e / OB) % 2, dim block e % OB; the second
  // tile's weights beside the first one's products
  u32x4 op[kAhead];
  auto read = [&](int e) { return value_operand<D, FP8>(tile[e / (2 * OB)], at, e % OB, e / OB % 2); };
#pragma unroll
  for (int e = 0; e < kAhead; ++e) op[e] = read(e);
#pragma unroll
  for (int e = 0; e < 2 * OB * TPS; ++e) {
    __builtin_amdgcn_sched_barrier(0);
    c.o[e % OB] = mfma(op[e % kAhead], pu[e / (2 * OB)][e / OB % 2], c.o[e % OB]);
    if (e + kAhead < 2 * OB * TPS) op[e % kAhead] = read(e + kAhead);
    if (TPS > 1 && e < 2 * OB) {
#pragma unroll
      for (int j = e * 8 / (2 * OB); j < (e + 1) * 8 / (2 * OB); ++j) weight_pair(TPS - 1, j);
    }
  }
  __builtin_amdgcn_sched_barrier(0);
}

// The workgroup's part of the flat list, segment by segment (a segment: what a part holds
// of one head).  U units of the same part lie side by side on one XCD and share its L2.
template <int D, bool FP8, int CW>
__global__ __launch_bounds__(256, 2) void tree_attn_kernel(TreeArgs a) {
  using Sh = Shape<D, FP8, CW>;
  constexpr int NW = Sh::NW, KW = Sh::KW, UC = Sh::UC, KS = D / 16, OB = D / 32, TB = Sh::kTile;
  __shared__ __attribute__((aligned(1024))) char tiles_lds[Sh::kLds];
  __shared__ __attribute__((aligned(16))) uint32_t meta_lds[Sh::kSlots][64];
  __shared__ float2 ml_lds[NW][32];
  __shared__ float factor_lds[KW][UC];
  __shared__ int row_lds[UC];
  if (load_status(a.status) != 0) return;
  const int tid = threadIdx.x, lane = tid & 63, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // waves of the same columns on different SIMDs: a unit with few columns leaves none idle
  const int cw = wave / KW, kw = wave % KW;
  const int Hq = a.H * a.g;
  // the U units of a part (their columns) read the same tiles: workgroups of one XCD
  // (the dispatcher deals them round-robin), dispatched next to each other
  const int x8 = blockIdx.x % kXcds, y8 = blockIdx.x / kXcds;
  const int unit = y8 % a.U, cell = kXcds * (y8 / a.U) + x8;
  if (cell >= a.cells) return;
  typedef int __attribute__((ext_vector_type(4))) i32x4;
  typedef int __attribute__((ext_vector_type(8))) i32x8;
  const i32x4 mine = *((const DMS_CONST i32x4*)(a.part + cell));
  i32x8 rd = *((const DMS_CONST i32x8*)(&a.part[cell].r));
  const int tb = mine[0], te = mine[1];
  int hh = mine[2], c0 = mine[3];
  const LaneAt at = lane_at<D, FP8>(lane);
  const uint32_t lds0 = lds_addr(tiles_lds), meta0 = lds_addr(meta_lds[0]);

  for (int f = tb; f < te;) {
    Segment sg;
    sg.sh = rd[0];
    sg.L = rd[1];
    sg.tok0 = rd[2];
    sg.m = rd[3];
    sg.p0 = rd[4];
    sg.tile0 = rd[5];
    sg.deep = rd[4] + ((const DMS_CONST int32_t*)a.deepest)[rd[6]];
    sg.hh = hh;
    sg.T = tiles_of(sg.L, sg.m);
    sg.t0 = f - c0;
    sg.t1 = min(sg.T, sg.t0 + te - f);
    sg.nc = (sg.L + 31) >> 5;
    f += sg.t1 - sg.t0;
    if (f < te) {          // the next head with nodes
      do c0 = ((const DMS_CONST int32_t*)a.cum)[++hh];
      while (((const DMS_CONST int32_t*)a.cum)[hh + 1] <= f);
      rd = *((const DMS_CONST i32x8*)(a.rows + hh));
    }
    if (unit * UC >= sg.m * a.g) continue;     // a smaller tree: no such columns
    const int h = sg.hh % a.H, cols = sg.m * a.g;
    const int nt = sg.t1 - sg.t0;

    // ---- tiles: sources and copies
    auto page_of = [&](int t) {
      return t < sg.nc ? ((const DMS_CONST int32_t*)(a.page_table + static_cast<size_t>(sg.sh) * a.maxp))[(32 * t) >> a.log2P] : 0;
    };
    auto source = [&](int t, int page) -> const char* {
      return t < sg.nc ? a.pool + static_cast<size_t>(page) * a.page_bytes + static_cast<size_t>(((32 * t) & (a.P - 1)) >> 5) * TB
                       : a.tiles + (static_cast<size_t>(sg.tile0) + (t - sg.nc)) * TB;
    };
    auto meta_of = [&](int t) -> const uint32_t* {
      return t < sg.nc ? reinterpret_cast<const uint32_t*>(a.slot_meta + static_cast<size_t>(sg.sh) * a.max_slots) + 32 * t
                       : a.tmeta + (static_cast<size_t>(sg.tile0) + (t - sg.nc)) * 32;
    };

    // ---- this wave's columns
    const int col0 = unit * UC + cw * 32;
    const bool busy = col0 < cols;
    Columns<D> c;
    auto load_columns = [&]() {
      const int ln = fresh(lane), col = col0 + (ln & 31);
      const bool ok = col < cols;
      const int node = ok ? col / a.g : 0, qh = ok ? col % a.g : 0;
      const size_t tok = static_cast<size_t>(sg.tok0) + node;
      const uint16_t* q = a.q + (tok * Hq + h * a.g + qh) * D + 8 * (ln >> 5);
#pragma unroll
      for (int s = 0; s < KS; ++s) c.q[s] = ok ? *reinterpret_cast<const u32x4*>(q + 16 * s) : u32x4{0u, 0u, 0u, 0u};
      // the borrowed decision neuron takes no part in attention (App. C)
      if (a.zero_neuron && qh == 0 && hf == 0) c.q[0][0] &= 0xFFFF0000u;
      c.t = sg.p0 + a.depth[tok];
      c.anc = a.anc + tok * a.words;
      c.m = kMInit;
      c.l = 0.f;
#pragma unroll
      for (int b = 0; b < OB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) c.o[b][i] = 0.f;
    };

    auto attend = [&](auto careful_c) {
      constexpr bool CAREFUL = decltype(careful_c)::value;
      if constexpr (Sh::PRIVATE) {
        constexpr int R = Sh::R, KC = (FP8 ? D / 32 + 1 : D / 16) + 1, VC = FP8 ? D / 32 : D / 16;
        // keys of own tile u (with the rows' owners; 8-bit pages: the scales too) and its values
        auto copy_keys = [&](int u, const char* tile) {
          const int slot = wave * R + u % R;
          const uint32_t dst = lds0 + Sh::slot_at(slot);
#pragma unroll
          for (int x = 0; x < D * (FP8 ? 32 : 64) / 1024; ++x) copy16_once(tile + 16 * lane + 1024 * x, dst + 1024 * x);
          if constexpr (FP8) copy4(tile + D * 64 + 4 * lane, dst + D * 64);
          copy4(meta_of(sg.t0 + kw + u * KW) + (lane & 31), meta0 + 256 * slot);
        };
        auto copy_values = [&](int u, const char* tile) {
          constexpr int V0 = D * (FP8 ? 32 : 64);
          const uint32_t dst = lds0 + Sh::slot_at(wave * R + u % R) + V0;
#pragma unroll
          for (int x = 0; x < V0 / 1024; ++x) copy16_once(tile + V0 + 16 * lane + 1024 * x, dst + 1024 * x);
        };
        const int n = max(0, (nt - kw + KW - 1) / KW);   // own tiles: t0 + kw, + KW, ..
#pragma unroll
        for (int u = 0; u < R; ++u)
          if (u < n) {
            const int t = sg.t0 + kw + u * KW;
            const char* src = source(t, page_of(t));
            copy_keys(u, src);
            copy_values(u, src);
          }
        load_columns();
        int page = R < n ? page_of(sg.t0 + kw + R * KW) : 0;
        for (int u = 0; u < n; ++u) {
          const int t = sg.t0 + kw + u * KW, slot = wave * R + u % R;
          const uint32_t tile[1] = {lds0 + static_cast<uint32_t>(Sh::slot_at(slot))};
          if (u + R - 1 < n) wait_copies_but<VC + (R - 1) * (KC + VC)>();
          else wait_copies();
          asm volatile("" ::: "memory");
          const uint32_t meta[1] = {meta_lds[slot][lane & 31]};
          const bool more = u + R < n;
          const char* next = source(sg.t0 + kw + (u + R) * KW, page);
          attend_tiles<D, FP8, 1, CAREFUL>(a, sg, c, tile, meta, t, at, lane,
              [&]() {
                // 8-bit pages: the scales lie in the keys' copies and are read for the weights
                if constexpr (!FP8) {
                  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                  if (more) copy_keys(u + R, next);
                }
              },
              [&]() {
                if (more) wait_copies_but<(R - 1) * (KC + VC) + (FP8 ? 0 : KC)>();
                else wait_copies();
                asm volatile("" ::: "memory");
                if (t == sg.nc - 1 && (sg.L & 31)) {
                  zero_values<D, FP8>(tile[0], sg.L & 31, fresh(lane), 64);
                  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                }
              });
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          if (more) {
            if constexpr (FP8) copy_keys(u + R, next);
            copy_values(u + R, next);
          }
          if (u + R + 1 < n) page = page_of(sg.t0 + kw + (u + R + 1) * KW);
        }
      } else {
        // a stage's copies: KW TPS tiles, the waves' shares of its pieces alike (past the
        // end: the last tile again, not attended)
        constexpr int S = Sh::S, TPS = Sh::TPS, kTiles = KW * TPS, kShare = NW / kTiles;
        constexpr int kPieces = TB / 1024 / kShare, PC = kPieces + 1 + FP8;
        const int ns = (nt + kTiles - 1) / kTiles;
        const int my = wave / kShare, share = wave % kShare;
        auto copy_stage = [&](int st, int page) {
          const int t = min(sg.t0 + st * kTiles + my, sg.t1 - 1), slot = st % S * kTiles + my;
          const char* tile = source(t, page) + 16 * lane;
          const uint32_t dst = lds0 + Sh::slot_at(slot);
#pragma unroll
          for (int x = 0; x < kPieces; ++x) {
            const int at1 = 1024 * (kPieces * share + x);
            if (CW < 4 && a.once) copy16_once(tile + at1, dst + at1);
            else lds_copy16(tile + at1, dst + at1);
          }
          if constexpr (FP8) copy4(tile + D * 64 - 12 * lane, dst + D * 64);
          copy4(meta_of(t) + (lane & 31), meta0 + 256 * slot);
        };
        auto stage_page = [&](int st) { return page_of(min(sg.t0 + st * kTiles + my, sg.t1 - 1)); };
#pragma unroll
        for (int st = 0; st < S - 1; ++st)
          if (st < ns) copy_stage(st, stage_page(st));
        load_columns();
        int page = stage_page(S - 1);
        for (int st = 0; st < ns; ++st) {
          // all but the stages after it have landed
          if (st + S - 2 < ns) wait_copies_but<(S - 2) * PC>();
          else wait_copies();
          __syncthreads();     // the stage is there, and no wave reads the one before it
          if (st + S - 1 < ns) copy_stage(st + S - 1, page);
          const int last = sg.nc - 1 - (sg.t0 + st * kTiles);
          if ((sg.L & 31) && last >= 0 && last < kTiles && sg.nc - 1 < sg.t1) {
            for (int x = last; x < kTiles; ++x)    // (past the end: the last tile again)
              if (x == last || sg.nc == sg.t1) zero_values<D, FP8>(lds0 + Sh::slot_at(st % S * kTiles + x), sg.L & 31, fresh(tid), 64 * NW);
            __syncthreads();
          }
          const int t = sg.t0 + st * kTiles + kw * TPS, slot = st % S * kTiles + kw * TPS;
          if (busy && t < sg.t1) {
            uint32_t tile[TPS], meta[TPS];
#pragma unroll
            for (int x = 0; x < TPS; ++x) {
              tile[x] = lds0 + Sh::slot_at(slot + x);
              meta[x] = meta_lds[slot + x][lane & 31];
            }
            attend_tiles<D, FP8, TPS, CAREFUL>(a, sg, c, tile, meta, t, at, lane, []() {}, []() {});
          }
          page = stage_page(st + S);
        }
      }
    };
    attend(std::false_type{});
    float z = 0.f;
#pragma unroll
    for (int b = 0; b < OB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) z = fmaf(c.o[b][i], 0.f, z);
    if (__syncthreads_or(z != 0.f)) attend(std::true_type{});    // (tiles are read)

    // ---- fold the waves of a column block and write it: the outputs of a whole
    // head, else a partial (slot 2 w: a head that began before this part; 2 w + 1:
    // one that ends after it).  A wave's sums lie in its own share of the tiles'
    // LDS, 16-byte pieces flipped by column to spread the banks.
    const bool whole = sg.t0 == 0 && sg.t1 == sg.T;
    const int part = 2 * (cell * a.U + unit) + (sg.t0 == 0);
    auto fold_at = [&](int w, int cc, int piece) {
      return reinterpret_cast<f32x4*>(tiles_lds + w * Sh::kWaveBytes + cc * (D * 4) + 16 * (piece ^ (cc & 7)));
    };
    const float l = col_sum(c.l);
    const int ln = fresh(lane), th = fresh(tid);     // (addresses formed here, not held ahead of the loops)
    __syncthreads();
    if (ln < 32) ml_lds[wave][ln] = make_float2(c.m, l);
#pragma unroll
    for (int b = 0; b < OB; ++b)
#pragma unroll
      for (int y = 0; y < 4; ++y)
        *fold_at(wave, ln & 31, 8 * b + 2 * y + (ln >> 5)) =
            f32x4{c.o[b][4 * y], c.o[b][4 * y + 1], c.o[b][4 * y + 2], c.o[b][4 * y + 3]};
    __syncthreads();
    if (th < UC) {     // a thread a column: what its waves' sums are multiplied by, and where it goes
      const int cx = th / 32, cc = th % 32, col = unit * UC + th;
      float M = kMInit, L = 0.f, f[KW];
#pragma unroll
      for (int y = 0; y < KW; ++y) M = fmaxf(M, ml_lds[cx * KW + y][cc].x);
#pragma unroll
      for (int y = 0; y < KW; ++y) {
        const float2 ml = ml_lds[cx * KW + y][cc];
        f[y] = __builtin_amdgcn_exp2f((ml.x - M) * a.scale_log2);
        L += ml.y * f[y];
      }
      const float inv = whole ? 1.0f / L : 1.0f;
#pragma unroll
      for (int y = 0; y < KW; ++y) factor_lds[y][th] = f[y] * inv;
      const int node = col / a.g;
      row_lds[th] = col >= cols ? -1 : whole ? (sg.tok0 + node) * Hq + h * a.g + (col - node * a.g) : part * UC + th;
      if (!whole && col < cols) a.part_ml[static_cast<size_t>(part) * UC + th] = make_float2(M, L);
    }
    __syncthreads();
    // UC columns, D / 4 pieces each
    for (int e = th; e < UC * (D / 4); e += 64 * NW) {
      const int piece = e % (D / 4), uc = e / (D / 4), row = row_lds[uc];
      if (row < 0) continue;
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int y = 0; y < KW; ++y) sum += *fold_at(uc / 32 * KW + y, uc % 32, piece) * factor_lds[y][uc];
      const size_t dst = static_cast<size_t>(row) * D + 4 * piece;
      if (whole) {
        const f32x2 lo = {sum[0], sum[1]}, hi = {sum[2], sum[3]};
        *reinterpret_cast<u32x2*>(a.out + dst) = u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
                                                       __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
      } else {
        *reinterpret_cast<f32x4*>(a.part_o + dst) = sum;
      }
    }
    __syncthreads();       // the next segment's copies go where the sums are
  }
}

// Joins the heads that several parts attended: D / 4 threads a column, a batch of
// its partials in flight at a time, a workgroup for 1024 / D columns of a head.  Two
// rounds of dependent loads: 2 us for one head, 6 for 16 heads of 10 parts, 11.5 deep and
// wide (14 and 19 MB of partials).  One wave to several columns, a column after the other,
// took 64 us.
template <int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a) {
  constexpr int kCols = 1024 / D, kBatch = 8;
  const int status = load_status(a.status);
  const int NH = a.n * a.H, per = (a.max_nodes * a.g + kCols - 1) / kCols;
  if (status != 0) return;
  const int piece = threadIdx.x % (D / 4);
  for (int64_t x = blockIdx.x; x < static_cast<int64_t>(NH) * per; x += gridDim.x) {
    const int hh = static_cast<int>(x / per), col = static_cast<int>(x % per) * kCols + threadIdx.x / (D / 4);
    const TreeRow r = a.rows[hh];
    const int2 span = a.head_parts[hh];
    const int w0 = __builtin_amdgcn_readfirstlane(span.x), w1 = __builtin_amdgcn_readfirstlane(span.y);
    if (w0 == w1 || col >= r.m * a.g) continue;    // one part wrote it
    const int unit = col / a.UC, uc = col - unit * a.UC;
    float M = kMInit, L = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int w = w0; w <= w1; w += kBatch) {
      f32x4 v[kBatch];
      float2 ml[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int y = w + u;
        ml[u] = make_float2(kMInit, 0.f);
        v[u] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (y > w1) continue;
        const size_t pc = (static_cast<size_t>(2) * (y * a.U + unit) + (y == w0)) * a.UC + uc;
        ml[u] = a.part_ml[pc];
        v[u] = *reinterpret_cast<const f32x4*>(a.part_o + pc * D + 4 * piece);
      }
      float m = M;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) m = fmaxf(m, ml[u].x);
      const float f0 = __builtin_amdgcn_exp2f((M - m) * a.scale_log2);
      acc *= f0;
      L *= f0;
      M = m;
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const float f = __builtin_amdgcn_exp2f((ml[u].x - M) * a.scale_log2);
        L += ml[u].y * f;
        acc += v[u] * f;
      }
    }
    acc *= 1.0f / L;
    const int h = hh % a.H, node = col / a.g;
    const f32x2 lo = {acc[0], acc[1]}, hi = {acc[2], acc[3]};
    *reinterpret_cast<u32x2*>(a.out + ((static_cast<size_t>(r.tok0) + node) * (a.H * a.g) + h * a.g + (col - node * a.g)) * D + 4 * piece) =
        u32x2{__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2)),
              __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2))};
  }
}

// ---------------------------------------------------------------------------
// Accepted paths
// ---------------------------------------------------------------------------

// A wave per sequence; lane l holds nodes l, l + 64, ..  Each step finds the
// lowest child of the present node whose token is the wanted one; a child's
// index is past its parent's, so the walk ends.  Latency: 1.8 us for one tree of 16
// nodes, 6.2 for 512 of up to 128.
__global__ __launch_bounds__(256) void tree_accept_kernel(const int32_t* cu, const int32_t* parents, const int32_t* tokens,
                                                          const int32_t* targets, const int32_t* first, int n, int total,
                                                          int max_nodes, int32_t* path, int32_t* path_len, int32_t* next) {
  constexpr int kPer = kTreeMaxNodes / 64;
  const int lane = threadIdx.x & 63;
  const int i = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= n) return;
  const int tok0 = max(0, min(cu[i], total)), m = min(max(tok0, min(cu[i + 1], total)) - tok0, max_nodes);
  int par[kPer], tok[kPer], tgt[kPer];
#pragma unroll
  for (int u = 0; u < kPer; ++u) {
    const int x = lane + 64 * u;
    par[u] = x < m ? parents[tok0 + x] : -2;
    tok[u] = x < m ? tokens[tok0 + x] : 0;
    tgt[u] = x < m ? targets[tok0 + x] : 0;
  }
  int at = -1, want = first != nullptr ? first[i] : -1, count = 0;
  bool any = first == nullptr;   // the root is accepted as it is
  while (count < m) {
    int found = -1;
#pragma unroll
    for (int u = kPer - 1; u >= 0; --u) {
      const int x = lane + 64 * u;
      const uint64_t hit = __builtin_amdgcn_ballot_w64(x > at && par[u] == at && (any || tok[u] == want));
      if (hit) found = 64 * u + __builtin_ctzll(hit);
    }
    if (found < 0) break;
    any = false;
#pragma unroll
    for (int u = 0; u < kPer; ++u)
      if (found >> 6 == u) want = __builtin_amdgcn_readlane(tgt[u], found & 63);
    if (lane == 0) path[tok0 + count] = found;
    ++count;
    at = found;
  }
  for (int x = count + lane; x < m; x += 64) path[tok0 + x] = -1;
  if (lane == 0) {
    path_len[i] = count;
    next[i] = want;
  }
}

// ---------------------------------------------------------------------------
// Commit of accepted paths: rule R1 for every token of a path, in order
// ---------------------------------------------------------------------------

struct CommitArgs {
  LayerState st;
  int32_t* status;
  const int32_t* seq_ids;
  const int32_t* cu;
  const int32_t* path;
  const int32_t* path_len;
  const uint8_t* flags;   // [total, H]
  const uint16_t* k;      // [total, H, D]
  const uint16_t* v;
  char* pool;
  size_t page_bytes;
  int32_t* need;          // [n H] pages to pop, or the error that refuses the call
  int32_t* fresh;         // [n H] tokens that take fresh slots
  int32_t* base;          // [n H] first pop of each head (calls of more than kScanHeads heads)
  int32_t* before;        // [n] positions, [n H] lengths, then stack height, ids' error, verdict, pops
  int n, H, w, P, log2P, D, maxp, max_slots, max_seqs, total, max_nodes;
  int immediate, fp8, mla;
};
constexpr int kScanHeads = 2048;   // up to here every workgroup sums the pops itself

__device__ inline int32_t* commit_pos(const CommitArgs& a) { return a.before; }
__device__ inline int32_t* commit_len(const CommitArgs& a) { return a.before + a.n; }
__device__ inline int32_t* commit_word(const CommitArgs& a, int x) { return a.before + a.n + static_cast<size_t>(a.n) * a.H + x; }

// Path of sequence i, or false if the call may not use it.
__device__ inline bool commit_path(const CommitArgs& a, int i, int& tok0, int& len) {
  tok0 = a.cu[i];
  const int end = a.cu[i + 1];
  len = a.path_len[i];
  return tok0 >= 0 && end >= tok0 && end <= a.total && end - tok0 <= a.max_nodes && len >= 0 && len <= end - tok0 &&
         (i > 0 || tok0 == 0) && (i < a.n - 1 || end == a.total);
}

// Whether path token c (at pos + c) takes the slot of the token w before it.
__device__ inline bool commit_reuse(const CommitArgs& a, const int* nodes, int sh, int h, int tok0, int pos, int c) {
  if (static_cast<int64_t>(pos) + c < a.w) return false;
  const int j = a.immediate ? c : c - a.w;
  if (j >= 0) return a.flags[(static_cast<size_t>(tok0) + nodes[j]) * a.H + h] != 0;
  return (static_cast<uint32_t>(a.st.ring[static_cast<size_t>(sh) * a.w + (pos + c) % a.w]) & kFlagBit) != 0;
}

// What one head's path takes, by a wave; its nodes are left in LDS.
struct CommitHead {
  int need, fresh, pos, len0;     // pages to pop, or the error that refuses the call
  int s, tok0, len;
};
__device__ inline CommitHead commit_scan_head(const CommitArgs& a, int hh, int* nodes) {
  const int lane = threadIdx.x & 63, i = hh / a.H, h = hh % a.H, s = a.seq_ids[i];
  int tok0, len, fresh = 0;
  CommitHead r{DMS_ERR_INVALID, 0, 0, 0, 0, 0, 0};
  if (s < 0 || s >= a.max_seqs || !commit_path(a, i, tok0, len)) return r;
  const int m = a.cu[i + 1] - tok0, sh = s * a.H + h;
  r.s = s;
  r.tok0 = tok0;
  r.len = len;
  r.pos = a.st.pos[s];
  r.len0 = a.st.len[sh];
  int off = 0;
  for (int c = lane; c < len; c += 64) {
    int x = a.path[tok0 + c];
    if (x < 0 || x >= m) {
      off = 1;
      x = 0;
    }
    nodes[c] = x;
  }
  const bool bad = __builtin_amdgcn_ballot_w64(off != 0) != 0;
  // (the wave's own LDS writes are visible to it)
  __builtin_amdgcn_wave_barrier();
  for (int c0 = 0; c0 < len; c0 += 64) {
    const int c = c0 + lane;
    const bool f = c < len && !commit_reuse(a, nodes, sh, h, tok0, r.pos, c);
    fresh += __builtin_popcountll(__builtin_amdgcn_ballot_w64(f));
  }
  r.fresh = fresh;
  const int64_t L1 = static_cast<int64_t>(r.len0) + fresh;
  if (!bad)
    r.need = L1 > a.max_slots ? DMS_ERR_CAPACITY
                              : static_cast<int>((L1 + a.P - 1) / a.P - (static_cast<int64_t>(r.len0) + a.P - 1) / a.P);
  return r;
}

// Whether an id is off or named twice, as a workgroup finds it.
__device__ inline bool commit_bad_ids(const CommitArgs& a, uint32_t* seen) {
  for (int x = threadIdx.x; x < (a.max_seqs + 31) / 32; x += blockDim.x) seen[x] = 0;
  __syncthreads();
  int bad = 0;
  for (int x = threadIdx.x; x < a.n; x += blockDim.x) {
    const int s = a.seq_ids[x];
    if (s < 0 || s >= a.max_seqs) bad = 1;
    else if (atomicOr(&seen[s >> 5], 1u << (s & 31)) & (1u << (s & 31))) bad = 1;
  }
  return __syncthreads_or(bad);
}

// Pass 1, a wave per head and one more for the ids: fresh tokens and pages of
// every head, and the state that pass 2 overwrites.  (Two launches, for no workgroup may
// write before all heads are known to fit.  64 sequences of 8 heads, up to 24 tokens a
// path: 4.3 + 7.9 us, dependent loads and scattered stores.)
__global__ __launch_bounds__(256) void commit_scan_kernel(CommitArgs a) {
  __shared__ uint32_t seen[kMaxSeqs / 32];
  __shared__ int nodes_lds[4][kTreeMaxNodes];
  if (load_status(a.status) != 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (blockIdx.x == 0) {
    const bool bad = commit_bad_ids(a, seen);
    if (threadIdx.x == 0) {
      *commit_word(a, 0) = *a.st.top;
      *commit_word(a, 1) = bad ? DMS_ERR_BAD_SEQ : DMS_OK;
    }
    return;
  }
  const int64_t hh64 = (static_cast<int64_t>(blockIdx.x) - 1) * 4 + wave;
  if (hh64 >= static_cast<int64_t>(a.n) * a.H) return;
  const int hh = static_cast<int>(hh64);
  const CommitHead r = commit_scan_head(a, hh, nodes_lds[wave]);
  if (lane == 0) {
    a.need[hh] = r.need;
    a.fresh[hh] = r.fresh;
    commit_len(a)[hh] = r.len0;
    if (hh % a.H == 0) commit_pos(a)[hh / a.H] = r.pos;
  }
}

// What the call's heads pop in all and whether one refuses it, as a workgroup
// sums it; before: pops of the heads ahead of hh.
__device__ inline int commit_verdict(const CommitArgs& a, int hh, int* lds, int& before, int& pops) {
  const int64_t NH = static_cast<int64_t>(a.n) * a.H;
  int all = 0, mine = 0, err = 0;
  for (int64_t x = threadIdx.x; x < NH; x += blockDim.x) {
    const int nd = a.need[x];
    err |= nd == DMS_ERR_INVALID ? 1 : nd == DMS_ERR_CAPACITY ? 2 : 0;
    all += max(nd, 0);
    if (x < hh) mine += max(nd, 0);
  }
  for (int off = 32; off; off >>= 1) {
    all += __shfl_xor(all, off, 64);
    mine += __shfl_xor(mine, off, 64);
    err |= __shfl_xor(err, off, 64);
  }
  const int wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    lds[3 * wave] = all;
    lds[3 * wave + 1] = mine;
    lds[3 * wave + 2] = err;
  }
  __syncthreads();
  all = mine = err = 0;
  for (int x = 0; x < nw; ++x) {
    all += lds[3 * x];
    mine += lds[3 * x + 1];
    err |= lds[3 * x + 2];
  }
  before = mine;
  pops = all;
  const int ids = *commit_word(a, 1), top = *commit_word(a, 0);
  return ids != DMS_OK ? ids : err & 1 ? DMS_ERR_INVALID : err & 2 ? DMS_ERR_CAPACITY : all > top ? DMS_ERR_OUT_OF_PAGES : DMS_OK;
}

// Calls of many heads: the pops summed once, by one workgroup.
__global__ __launch_bounds__(1024) void commit_pages_kernel(CommitArgs a) {
  __shared__ int lds[51];
  if (load_status(a.status) != 0) return;
  int before, pops;
  const int err = commit_verdict(a, 0, lds, before, pops);
  if (threadIdx.x == 0) {
    *commit_word(a, 2) = err;
    *commit_word(a, 3) = pops;
  }
  if (err != DMS_OK) return;
  const int64_t NH = static_cast<int64_t>(a.n) * a.H;
  int run = 0;
  for (int64_t b = 0; b < NH; b += blockDim.x) {
    const int64_t hh = b + threadIdx.x;
    int tot;
    __syncthreads();
    const int off = block_exclusive_scan(hh < NH ? a.need[hh] : 0, lds, &tot);
    if (hh < NH) a.base[hh] = run + off;
    run += tot;
  }
}

// Slots, ring, slot owners, pages and the rows of the tokens that keep their slot, of
// one head, by THREADS threads: a workgroup of kTreeMaxNodes or a wave.
template <int THREADS>
__device__ inline void commit_write_head(const CommitArgs& a, int hh, const CommitHead& r, int top0, int before, int* nodes,
                                         int* slots, int* keeps, int* lds) {
  static_assert(THREADS == 64 || THREADS == kTreeMaxNodes, "a token a thread, or a wave");
  const int tid = threadIdx.x % THREADS, h = hh % a.H;
  const int s = r.s, sh = s * a.H + h, tok0 = r.tok0, len = r.len, pos = r.pos, L0 = r.len0;
  auto sync = []() {
    if (THREADS > 64) __syncthreads();
    else {      // a wave's LDS accesses are in order
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };
  if (len == 0) return;
  if (tid == 0) {
    a.st.len[sh] = L0 + r.fresh;
    if (h == 0) a.st.pos[s] = pos + len;
  }
  const int32_t* popped = a.st.stack + top0 - 1 - before;     // k-th new page at -k
  const size_t pt = static_cast<size_t>(sh) * a.maxp;
  const int new0 = (L0 + a.P - 1) >> a.log2P;
  for (int x = tid; x < r.need; x += THREADS) a.st.page_table[pt + new0 + x] = popped[-x];
  if (THREADS > 64) {      // (a wave has them from its scan)
    for (int c = tid; c < len; c += THREADS) nodes[c] = a.path[tok0 + c];
    sync();
  }
  // slots: fresh tokens in order; a reusing one has that of the token w before
  // it, in the path or in the ring
  int ahead = 0;
  for (int c0 = 0; c0 < len; c0 += THREADS) {     // (a workgroup: once)
    const int c = c0 + tid;
    const bool on = c < len;
    const bool reuse = on && commit_reuse(a, nodes, sh, h, tok0, pos, c);
    const uint64_t bal = __builtin_amdgcn_ballot_w64(on && !reuse);
    int rank = ahead + __builtin_popcountll(bal & ((1ull << (tid & 63)) - 1ull));
    if (THREADS > 64) {
      if ((tid & 63) == 0) lds[tid >> 6] = __builtin_popcountll(bal);
      sync();
      for (int x = 0; x < (tid >> 6); ++x) rank += lds[x];
    }
    ahead += __builtin_popcountll(bal);
    if (on) {
      slots[c] = !reuse ? L0 + rank
                 : c < a.w ? static_cast<int>(static_cast<uint32_t>(a.st.ring[static_cast<size_t>(sh) * a.w + (pos + c) % a.w]) & ~kFlagBit)
                           : -1;
      // a token keeps its slot unless the token w later takes it
      keeps[c] = len - c <= a.w || !commit_reuse(a, nodes, sh, h, tok0, pos, c + a.w);
    }
  }
  sync();
  for (int c0 = a.w; c0 < len; c0 += a.w) {     // one window of the path at a time
    for (int x = c0 + tid; x < min(len, c0 + a.w); x += THREADS)
      if (slots[x] < 0) slots[x] = slots[x - a.w];
    sync();
  }
  for (int c = tid; c < len; c += THREADS) {
    const uint32_t fb = a.flags[(static_cast<size_t>(tok0) + nodes[c]) * a.H + h] ? kFlagBit : 0u;
    if (len - c <= a.w)
      a.st.ring[static_cast<size_t>(sh) * a.w + (pos + c) % a.w] = static_cast<int32_t>(static_cast<uint32_t>(slots[c]) | fb);
    if (keeps[c])
      a.st.slot_meta[static_cast<size_t>(sh) * a.max_slots + slots[c]] = static_cast<int32_t>(static_cast<uint32_t>(pos + c) | fb);
  }
  // rows: D / 8 consecutive lanes each (an aligned lane group for the 8-bit
  // quantizer: it takes every branch together)
  const int kq = a.D / 8;
  for (int x = tid; x < len * kq; x += THREADS) {
    const int y = x / kq, part = x - y * kq;
    if (!keeps[y]) continue;
    const int slot = slots[y], row = slot & (a.P - 1), j = row & 31, pi = slot >> a.log2P;
    const int page = pi >= new0 ? popped[new0 - pi] : a.st.page_table[pt + pi];
    const size_t src = ((static_cast<size_t>(tok0) + nodes[y]) * a.H + h) * a.D;
    const uint4 kx = reinterpret_cast<const uint4*>(a.k + src)[part];
    char* pg = a.pool + static_cast<size_t>(page) * a.page_bytes;
    if (a.mla) {
      *reinterpret_cast<uint4*>(pg + (row >> 5) * mla_tile_bytes(a.D) + k_elem_off(j, 8 * part)) = kx;
      continue;
    }
    const uint4 vx = reinterpret_cast<const uint4*>(a.v + src)[part];
    if (a.fp8) {
      fp8_store_token(pg + (row >> 5) * fp8_tile_bytes(a.D), j, a.D, part, kx, vx);
      continue;
    }
    char* tile = pg + (row >> 5) * tile_bytes(a.D);
    *reinterpret_cast<uint4*>(tile + k_elem_off(j, 8 * part)) = kx;
    const uint32_t vw[4] = {vx.x, vx.y, vx.z, vx.w};
#pragma unroll
    for (int d = 0; d < 8; ++d)
      *reinterpret_cast<uint16_t*>(tile + v_elem_off(j, part * 8 + d, a.D)) = static_cast<uint16_t>(vw[d >> 1] >> (16 * (d & 1)));
  }
}

// Pass 2, a workgroup per head.
template <bool SUMMED>
__global__ __launch_bounds__(kTreeMaxNodes) void commit_write_kernel(CommitArgs a) {
  __shared__ int lds[12];
  __shared__ int nodes[kTreeMaxNodes], slots[kTreeMaxNodes], keeps[kTreeMaxNodes];
  if (load_status(a.status) != 0) return;
  const int hh = blockIdx.x, tid = threadIdx.x;
  int before, pops, err;
  if (SUMMED) {
    err = *commit_word(a, 2);
    pops = *commit_word(a, 3);
    before = err == DMS_OK ? a.base[hh] : 0;
  } else {
    err = commit_verdict(a, hh, lds, before, pops);
  }
  const int64_t last = static_cast<int64_t>(a.n) * a.H - 1;
  if (err != DMS_OK) {
    // the other workgroups of this launch read no status past their first line
    if (hh == last && tid == 0) set_status(a.status, err);
    return;
  }
  const int top0 = *commit_word(a, 0);
  if (hh == last && tid == 0) *a.st.top = top0 - pops;
  const int i = hh / a.H;
  const CommitHead r{a.need[hh], a.fresh[hh], commit_pos(a)[i], commit_len(a)[hh], a.seq_ids[i], a.cu[i], a.path_len[i]};
  commit_write_head<kTreeMaxNodes>(a, hh, r, top0, before, nodes, slots, keeps, lds);
}

// Calls of up to kSmallHeads heads in one launch: a workgroup, a wave per head (one call
// of 16 heads: 10.7 us, in two launches 4.4 + 6.0 and the pause between them).
constexpr int kSmallHeads = 16;
__global__ __launch_bounds__(64 * kSmallHeads) void commit_small_kernel(CommitArgs a) {
  __shared__ uint32_t seen[kMaxSeqs / 32];
  __shared__ int nodes[kSmallHeads][kTreeMaxNodes], slots[kSmallHeads][kTreeMaxNodes], keeps[kSmallHeads][kTreeMaxNodes];
  __shared__ int needs[kSmallHeads];
  if (load_status(a.status) != 0) return;
  const int lane = threadIdx.x & 63, hh = threadIdx.x >> 6, NH = a.n * a.H;
  const int top0 = *a.st.top;
  CommitHead r{};
  if (hh < NH) r = commit_scan_head(a, hh, nodes[hh]);
  if (lane == 0) needs[hh] = r.need;
  const bool bad = commit_bad_ids(a, seen);      // (every wave has read the state that is written below)
  int before = 0, pops = 0, err = 0;
  for (int x = 0; x < kSmallHeads; ++x) {
    const int nd = needs[x];
    err |= nd == DMS_ERR_INVALID ? 1 : nd == DMS_ERR_CAPACITY ? 2 : 0;
    if (x < hh) before += max(nd, 0);
    pops += max(nd, 0);
  }
  const int rc = bad ? DMS_ERR_BAD_SEQ : err & 1 ? DMS_ERR_INVALID : err & 2 ? DMS_ERR_CAPACITY
                 : pops > top0 ? DMS_ERR_OUT_OF_PAGES : DMS_OK;
  if (threadIdx.x == 0) {
    if (rc != DMS_OK) set_status(a.status, rc);
    else *a.st.top = top0 - pops;
  }
  if (rc == DMS_OK && hh < NH) commit_write_head<64>(a, hh, r, top0, before, nodes[hh], slots[hh], keeps[hh], nullptr);
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------

// two workgroups a compute unit, at most what a workspace holds partials for
int tree_workgroups() {
  int dev = 0, v = 0;
  if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || v < 1)
    return kTreeWorkgroups;
  return std::min(2 * v, kTreeWorkgroups);
}

// Waves side by side over the columns, for the largest tree of a call.
int tree_waves(int cols) { return cols <= 32 ? 1 : cols <= 64 ? 2 : 4; }

struct TreeLayout {
  size_t rows, cum, part, head_parts, anc, depth, deepest, flags, tiles, tmeta, part_o, part_ml, need, fresh, base, before, bytes;
  int words, tph, UC;
};
TreeLayout tree_layout(const dms_config& c, int n, int total, int max_nodes) {
  TreeLayout lo{};
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = align_up(off + bytes, kAlign); return o; };
  const size_t H = c.num_kv_heads, NH = static_cast<size_t>(n) * H, T = total, D = c.head_dim;
  lo.need = take(NH * 4);
  lo.fresh = take(NH * 4);
  lo.base = take(NH * 4);
  lo.before = take((n + NH + 4) * 4);
  if (c.kv_format != DMS_KV_MLA) {
    lo.words = std::max(1, (max_nodes + 31) / 32);
    lo.tph = total / 32 + n + 1;
    lo.UC = 32 * tree_waves(max_nodes * c.group_size);
    lo.rows = take(NH * sizeof(TreeRow));
    lo.cum = take((NH + 1) * 4);
    lo.part = take(kTreeWorkgroups * sizeof(TreePart));
    lo.head_parts = take(NH * sizeof(int2));
    lo.anc = take(T * lo.words * 4);
    lo.depth = take(T * 4);
    lo.deepest = take(static_cast<size_t>(n) * 4);
    lo.flags = take(T * H);
    lo.tiles = take(H * static_cast<size_t>(lo.tph) * (c.kv_format == DMS_KV_FP8 ? fp8_tile_bytes(c.head_dim) : tile_bytes(c.head_dim)));
    lo.tmeta = take(H * static_cast<size_t>(lo.tph) * 32 * 4);
    lo.part_o = take(size_t(2) * kTreeWorkgroups * lo.UC * D * 4);
    lo.part_ml = take(size_t(2) * kTreeWorkgroups * lo.UC * 8);
  }
  lo.bytes = off;
  return lo;
}

template <int D, bool FP8>
hipError_t launch_attention(const TreeArgs& a, hipStream_t st) {
  const unsigned prep = 1u + a.n + static_cast<unsigned>(a.n) * a.H * a.words;
  hipLaunchKernelGGL((tree_prep_kernel<D, FP8>), dim3(prep), dim3(kPrepThreads), 0, st, a);
  if (a.UC == 32) hipLaunchKernelGGL((tree_attn_kernel<D, FP8, 1>), dim3(a.cells * a.U), dim3(256), 0, st, a);
  else if (a.UC == 64) hipLaunchKernelGGL((tree_attn_kernel<D, FP8, 2>), dim3(a.cells * a.U), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((tree_attn_kernel<D, FP8, 4>), dim3(a.cells * a.U), dim3(256), 0, st, a);
  const int64_t blocks = static_cast<int64_t>(a.n) * a.H * ((a.max_nodes * a.g + 1024 / D - 1) / (1024 / D));
  const unsigned merge = static_cast<unsigned>(std::min<int64_t>(blocks, 1 << 20));
  hipLaunchKernelGGL((tree_merge_kernel<D>), dim3(merge), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

size_t tree_workspace_bytes(const dms_config& c, int n, int total, int max_nodes) {
  return tree_layout(c, n, total, max_nodes).bytes;
}

hipError_t launch_tree_attention(const dms_config& c, const Layout& lo, void* meta, void* pool, int layer, int n,
                                 const int32_t* seq_ids, const int32_t* cu, int total, int max_nodes,
                                 const int32_t* parents, const void* q, const void* k, const void* v,
                                 const uint8_t* flags, uint8_t* decisions_out, void* out, void* ws, hipStream_t st) {
  const TreeLayout tl = tree_layout(c, n, total, max_nodes);
  char* w = static_cast<char*>(ws);
  const LayerState s = layer_state(lo, meta, layer);
  TreeArgs a{};
  a.status = reinterpret_cast<int32_t*>(static_cast<char*>(meta) + lo.status);
  a.seq_ids = seq_ids;
  a.cu = cu;
  a.parents = parents;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.flags = flags;
  if (flags == nullptr) {
    a.flags_out = decisions_out != nullptr ? decisions_out : reinterpret_cast<uint8_t*>(w + tl.flags);
    a.flags = a.flags_out;
  }
  a.pool = static_cast<const char*>(pool);
  a.page_table = s.page_table;
  a.slot_meta = s.slot_meta;
  a.len = s.len;
  a.pos = s.pos;
  a.out = static_cast<uint16_t*>(out);
  a.rows = reinterpret_cast<TreeRow*>(w + tl.rows);
  a.cum = reinterpret_cast<int32_t*>(w + tl.cum);
  a.part = reinterpret_cast<TreePart*>(w + tl.part);
  a.head_parts = reinterpret_cast<int2*>(w + tl.head_parts);
  a.anc = reinterpret_cast<uint32_t*>(w + tl.anc);
  a.depth = reinterpret_cast<int32_t*>(w + tl.depth);
  a.deepest = reinterpret_cast<int32_t*>(w + tl.deepest);
  a.tiles = w + tl.tiles;
  a.tmeta = reinterpret_cast<uint32_t*>(w + tl.tmeta);
  a.part_o = reinterpret_cast<float*>(w + tl.part_o);
  a.part_ml = reinterpret_cast<float2*>(w + tl.part_ml);
  a.page_bytes = lo.page_bytes;
  a.n = n;
  a.H = c.num_kv_heads;
  a.g = c.group_size;
  a.w = c.window;
  a.P = c.page_size;
  a.log2P = 31 - __builtin_clz(c.page_size);
  a.maxp = c.max_pages_per_head;
  a.max_slots = lo.max_slots;
  a.max_seqs = c.max_seqs;
  a.total = total;
  a.max_nodes = max_nodes;
  a.words = tl.words;
  a.tph = tl.tph;
  a.UC = tl.UC;
  // units and their columns by the largest tree of the call: beside it, the units of smaller
  // trees that have no such columns go past their parts, and the waves of one that has few
  // idle (48 sequences at 32768 tokens, 8 heads, one tree of 128 nodes and 47 of 4: 416 us;
  // 48 trees of 4 nodes 149, of 12 nodes 165)
  a.U = (max_nodes * c.group_size + tl.UC - 1) / tl.UC;
  a.cells = std::max(1, tree_workgroups() / kXcds / a.U) * kXcds;
  a.min_tiles = 8;
  a.once = a.U == 1;
  a.zero_neuron = c.decision_source == DMS_DECIDE_QUERY;
  a.bias = c.decision_bias;
  a.scale_log2 = c.softmax_scale * 1.4426950408889634f;
  const bool fp8 = c.kv_format == DMS_KV_FP8;
  if (c.head_dim == 64) return fp8 ? launch_attention<64, true>(a, st) : launch_attention<64, false>(a, st);
  return fp8 ? launch_attention<128, true>(a, st) : launch_attention<128, false>(a, st);
}

hipError_t launch_tree_accept(int n, const int32_t* cu, int total, int max_nodes, const int32_t* parents,
                              const int32_t* tokens, const int32_t* targets, const int32_t* first, int32_t* path,
                              int32_t* path_len, int32_t* next, hipStream_t st) {
  hipLaunchKernelGGL(tree_accept_kernel, dim3((n + 3) / 4), dim3(256), 0, st, cu, parents, tokens, targets, first, n, total,
                     max_nodes, path, path_len, next);
  return hipGetLastError();
}

hipError_t launch_tree_commit(const dms_config& c, const Layout& lo, void* meta, void* pool, int layer, int n,
                              const int32_t* seq_ids, const int32_t* cu, int total, int max_nodes, const int32_t* path,
                              const int32_t* path_len, const void* k, const void* v, const uint8_t* flags, void* ws,
                              hipStream_t st) {
  const TreeLayout tl = tree_layout(c, n, total, max_nodes);
  char* w = static_cast<char*>(ws);
  CommitArgs a{};
  a.st = layer_state(lo, meta, layer);
  a.status = reinterpret_cast<int32_t*>(static_cast<char*>(meta) + lo.status);
  a.seq_ids = seq_ids;
  a.cu = cu;
  a.path = path;
  a.path_len = path_len;
  a.flags = flags;
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.pool = static_cast<char*>(pool);
  a.page_bytes = lo.page_bytes;
  a.need = reinterpret_cast<int32_t*>(w + tl.need);
  a.fresh = reinterpret_cast<int32_t*>(w + tl.fresh);
  a.base = reinterpret_cast<int32_t*>(w + tl.base);
  a.before = reinterpret_cast<int32_t*>(w + tl.before);
  a.n = n;
  a.H = c.num_kv_heads;
  a.w = c.window;
  a.P = c.page_size;
  a.log2P = 31 - __builtin_clz(c.page_size);
  a.D = c.head_dim;
  a.maxp = c.max_pages_per_head;
  a.max_slots = lo.max_slots;
  a.max_seqs = c.max_seqs;
  a.total = total;
  a.max_nodes = max_nodes;
  a.immediate = c.eviction == DMS_EVICT_IMMEDIATE;
  a.fp8 = c.kv_format == DMS_KV_FP8;
  a.mla = c.kv_format == DMS_KV_MLA;
  const unsigned NH = static_cast<unsigned>(n) * c.num_kv_heads;
  if (NH <= kSmallHeads) {
    hipLaunchKernelGGL(commit_small_kernel, dim3(1), dim3(64 * kSmallHeads), 0, st, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(commit_scan_kernel, dim3(1 + (NH + 3) / 4), dim3(256), 0, st, a);
  if (NH > kScanHeads) {
    hipLaunchKernelGGL(commit_pages_kernel, dim3(1), dim3(1024), 0, st, a);
    hipLaunchKernelGGL(commit_write_kernel<true>, dim3(NH), dim3(kTreeMaxNodes), 0, st, a);
  } else {
    hipLaunchKernelGGL(commit_write_kernel<false>, dim3(NH), dim3(kTreeMaxNodes), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace dms
