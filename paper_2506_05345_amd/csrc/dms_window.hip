// Attention with a sliding window and sinks over packed sequences, gfx950.
//
// Key j is visible to query t iff j <= t and (j > t - w or j < sinks).
//   fwd: s = scale q.k, out = sum exp(s - m) v / l, lse = m + log l;
//   bwd: P = exp(s - lse), dP = dO V^T, D_t = dO.out, dS = P (dP - D),
//        dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO.
// D_t is formed as sum_j P_j dP_j / sum_j P_j: from the rounded `out` it would be
// off by up to 2^-8 of |dO||out|, which dS = P (dP - D) of a row with few keys or
// peaked weights does not forgive (where one key takes nearly all the weight
// dP - D is nearly 0).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "dms_ops.h"
#include "dms_tiles.h"

namespace dms {
namespace {

constexpr int kThreads = 256;
constexpr int kCols = 128;            // (position, query head) columns of a query block, 32 per wave
constexpr int kAhead = 4;              // operands are read this many MFMAs ahead, in pinned order
constexpr float kRescale = 8.0f;      // lazy rescale threshold, log2 units
constexpr float kMInit = -1.0e30f;    // running max before the first visible key
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct WindowArgs {
  const int32_t* cu;
  const __bf16 *q, *k, *v, *dout;
  const float* lse;
  __bf16 *out, *dq, *dk, *dv;
  float* lse_out;
  float* nlse;             // [Hq][Ts] -lse / scale (raw score units) of each query (workspace)
  float* nsum;             // [Hq][Ts] -D of each query (workspace)
  float* part;             // [splits][T][H][2 D]: sums of a key block's shares of steps (splits > 1; workspace)
  float* far_part;         // [T / far + 1][sink tiles][H][2][32][D]: (dk, dv) of sinks' far queries, and, without
                           // splits, as much again of the sinks from their key blocks (workspace)
  int64_t Ts;              // rows of a head in nlse, nsum: T + 128, whole copies are read past a sequence
  int n, T, H, g, w, sinks;
  int single;              // every row sees one key: P = 1 and dS = 0
  int PB;                  // positions of a query block: kCols / g
  uint32_t inv_pb;         // 2^32 / PB + 1
  uint32_t inv_g;          // 65536 / g + 1: col / g = col * inv_g >> 16 for columns below 128
  int far;                 // a sink's queries from this position on go to workgroups of `far` positions (a multiple of 128)
  uint32_t inv_far;
  int sink_tiles;          // 32-key tiles of sinks with such queries
  int splits;              // workgroups that share a key block's steps
  float scale_log2;
};

// Bounds of sequence i inside the packed tensors, whatever cu holds.
__device__ inline int2 bounds_of(const WindowArgs& a, int i) {
  const int lo = min(max(a.cu[i], 0), a.T);
  return make_int2(lo, min(max(a.cu[i + 1], lo), a.T));
}

__device__ inline float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

// x / d for 0 <= x < 2^31, inv = 2^32 / d + 1: the product is at most one too large.
__device__ inline int divide(int x, int d, uint32_t inv) {
  if (d == 1) return x;
  const int q = static_cast<int>(__umulhi(static_cast<uint32_t>(x), inv));
  return q * static_cast<int64_t>(d) > x ? q - 1 : q;
}
constexpr uint32_t inverse(int d) { return static_cast<uint32_t>((uint64_t(1) << 32) / d + 1); }

// Block b of a packed launch whose blocks hold PB tokens each (inv = 2^32 / PB + 1): sequence i owns blocks
// cu[i] / PB + i .. cu[i + 1] / PB + i, at least as many as it needs, so that a block finds its sequence
// by a search over cu (64 candidates a round) and the host needs no prefix sums.  With per_seq = 0 the
// blocks are cu[i] / PB + 0, 1, ... instead, which is unambiguous for sequences longer than PB.
struct Block {
  int s0, len, p0;   // first token and length of the sequence, first position of the block (>= len: no block)
};
__device__ inline Block block_of(const WindowArgs& a, int b, int PB, uint32_t inv, int per_seq = 1) {
  int lo = 0, cnt = a.n;
  while (cnt > 1) {
    const int lane = threadIdx.x & 63;
    const int step = (cnt + 63) >> 6;
    const int i = min(lo + lane * step, a.n);
    const bool le = lane * step < cnt && divide(min(max(a.cu[i], 0), a.T), PB, inv) + per_seq * i <= b;
    const int k = max(1, __builtin_popcountll(__builtin_amdgcn_ballot_w64(le)));
    lo += (k - 1) * step;
    cnt = min(step, cnt - (k - 1) * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  const int2 r = bounds_of(a, lo);
  return Block{r.x, r.y - r.x, max(b - (divide(r.x, PB, inv) + per_seq * lo), 0) * PB};
}

// Keys that queries [p0, p1) of a sequence see, listed without a gap: the sinks, then the window from its
// first key on (a window that reaches the sinks: the whole sequence up to p1).  Entry e of the list is key e
// among the sinks and key base + e past them; tiles are 32 entries.
struct KeyTiles {
  int base, nt;
};
__device__ inline KeyTiles key_tiles(const WindowArgs& a, int p0, int p1) {
  const int base = max(0, p0 - a.w + 1 - a.sinks);
  return KeyTiles{base, (p1 - base + 31) >> 5};
}

// Tiles of the list that the queries [q0, q1] (positions of one wave) see: some key of [some0, some1) and of
// those with sinks, every key of [all0, all1).
struct WaveTiles {
  int some0, some1, all0, all1, sinks;
};
__device__ inline WaveTiles wave_tiles(const WindowArgs& a, const KeyTiles& t, int q0, int q1) {
  WaveTiles w;
  w.some0 = max(0, (q0 - a.w + 1 - t.base) >> 5);
  w.some1 = q0 > q1 ? 0 : ((q1 - t.base) >> 5) + 1;
  w.all0 = max(0, (q1 - a.w + 32 - t.base) >> 5);
  w.all1 = (q0 + 1 - t.base) >> 5;
  w.sinks = (a.sinks + 31) >> 5;
  return w;
}
__device__ inline bool tile_seen(const WaveTiles& w, int i) {
  return i < w.some1 && (i >= w.some0 || i < w.sinks);
}
// Hides what position t does not see of tile i: register x of a lane is entry 32 i + 16 (x / 8) + 8 hf + x % 8.
// Most tiles at an edge have one edge only: a comparison and a select for each score.
__device__ inline void hide(f32x16& s, const WindowArgs& a, const KeyTiles& kt, const WaveTiles& wt, int i, int t,
                            int hf) {
  if (i >= wt.all0 && i < wt.all1) return;
  const int first = 32 * i + 8 * hf;
  const int hi = t - kt.base - first;        // last entry seen
  if (i < wt.all0) {
    const int lo = hi - a.w;                 // last one before the window
    if (i < wt.sinks) {
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int k = 16 * (x >> 3) + (x & 7);
        s[x] = k > lo || k < a.sinks - first ? s[x] : -INFINITY;
      }
    } else {
#pragma unroll
      for (int x = 0; x < 16; ++x) s[x] = 16 * (x >> 3) + (x & 7) > lo ? s[x] : -INFINITY;
    }
  }
  if (i >= wt.all1) {
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] = 16 * (x >> 3) + (x & 7) <= hi ? s[x] : -INFINITY;
  }
}

__device__ inline float max3(float a, float b, float c) {   // scores of visible NaN keys are ignored here
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}
__device__ inline bool not_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }
// 0 times an Inf or a NaN is a NaN, which every later sum keeps: one sum tells whether a row met any.
__device__ inline bool is_nan(float x) { return (__float_as_uint(x) & 0x7FFFFFFFu) > 0x7F800000u; }

// The exact walks: a result whose sums may have met an Inf or NaN of a hidden key or query (0 times it is a
// NaN) is formed again by one wave from what is visible alone.  A lane takes the weight of one of 64 keys or
// rows, then all lanes add the 64, a pair of the head's elements each.  Only elements that were stored as NaN
// are open; a walk ends, and leaves the stored ones, once all of these are NaN again, and it looks first at the
// one key that every query sees, its own.  16384 tokens of 8 x 5 heads, w = 256, 4 sinks, forward and backward:
// 139 and 595 us; all values NaN 264 and 732, all output gradients NaN 137 and 776, one token's values NaN 950
// and 8700 (one key or row at a time and to the end, 29 ms and 124 ms, 142 us and 124 ms, 4 and 90 ms).  What
// has to be walked to its end stays slow: all values +Inf 8 and 3 ms, all output gradients +Inf 0.1 and 47 ms.
__device__ inline float low(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ inline float high(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }
// This lane's pair of a row's D elements (D = 64: two lanes to a pair).
template <int D>
__device__ inline uint32_t pair_of(const __bf16* row) {
  return reinterpret_cast<const uint32_t*>(row)[threadIdx.x & (D / 2 - 1)];
}
template <int D>
__device__ inline void store_pair(__bf16* row, float x, float y) {
  const f32x2 pr = {x, y};
  reinterpret_cast<uint32_t*>(row)[threadIdx.x & (D / 2 - 1)] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, bf16x2));
}
// This lane's row times the row whose pairs lie over the lanes.
template <int D>
__device__ inline float row_dot(const __bf16* row, uint32_t pairs) {
  float s = 0.f;
#pragma unroll 2
  for (int c = 0; c < D / 8; ++c) {
    const u32x4 r = ld16(row + 8 * c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t two = r[i], other = __builtin_amdgcn_readlane(pairs, 4 * c + i);
      s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, other), s, false);
    }
  }
  return s;
}
__device__ inline float lane_value(float x, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane));
}
__device__ inline bool any_lane(bool x) { return __builtin_amdgcn_ballot_w64(x) != 0; }
constexpr int kAdd = 8;   // rows read together

// What the wave has stored lies before what it reads next (other lanes' elements, through another type).
__device__ inline void after_stores() { __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup"); }

// Entry e of the keys that position t sees, listed without a gap from `base` on (as in KeyTiles).
__device__ inline int seen_key(const WindowArgs& a, int base, int e) { return e < a.sinks ? e : base + e; }

// Row (position t of the sequence at s0, query head hq) of the output, whose scores hold no NaN.
template <int D>
__device__ inline void exact_row(const WindowArgs& a, int s0, int t, int hq) {
  const int lane = threadIdx.x & 63, Hq = a.H * a.g, h = hq / a.g;
  auto key_row = [&](int j) { return (static_cast<size_t>(s0 + j) * a.H + h) * D; };
  const size_t row = (static_cast<size_t>(s0 + t) * Hq + hq) * D;
  after_stores();
  const uint32_t was = pair_of<D>(a.out + row), own = pair_of<D>(a.v + key_row(t)), q = pair_of<D>(a.q + row);
  const bool open0 = is_nan(low(was)), open1 = is_nan(high(was));
  if (!any_lane((open0 && !is_nan(low(own))) || (open1 && !is_nan(high(own))))) return;
  float o0 = 0.f, o1 = 0.f, m = -INFINITY, l = 0.f;
  const int base = max(0, t - a.w + 1 - a.sinks), keys = t + 1 - base;
#pragma unroll 1
  for (int k0 = 0; k0 < keys; k0 += 64) {
    const bool in = k0 + lane < keys;
    const float x = row_dot<D>(a.k + key_row(seen_key(a, base, min(k0 + lane, keys - 1))), q) * a.scale_log2;
    const float s = in ? x : -INFINITY;
    if (any_lane(is_nan(s) || s == INFINITY)) return;   // all of the row is NaN, as it was stored
    float mn = fmaxf(m, s);
#pragma unroll
    for (int off = 32; off; off >>= 1) mn = fmaxf(mn, __shfl_xor(mn, off, 64));
    const float ref = mn == -INFINITY ? 0.f : mn;   // no weight so far: exp2(-Inf - 0) = 0
    const float c = exp2f(m - ref), p = exp2f(s - ref);
    l = l * c + wave_sum(p);
    o0 *= c;
    o1 *= c;
    m = mn;
    const int n = min(64, keys - k0);
#pragma unroll 1
    for (int i = 0; i < n; i += kAdd) {
      uint32_t v[kAdd];
#pragma unroll
      for (int u = 0; u < kAdd; ++u) v[u] = i + u < n ? pair_of<D>(a.v + key_row(seen_key(a, base, k0 + i + u))) : 0u;
#pragma unroll
      for (int u = 0; u < kAdd; ++u) {
        const float pu = lane_value(p, i + u);
        o0 += pu * low(v[u]);
        o1 += pu * high(v[u]);
      }
      if (!any_lane((open0 && !is_nan(o0)) || (open1 && !is_nan(o1)))) return;
    }
  }
  store_pair<D>(a.out + row, o0 / l, o1 / l);
  if (lane == 0) a.lse_out[static_cast<size_t>(hq) * a.T + s0 + t] = (m + log2f(l)) * kLn2;
}

__device__ const u32x4 kZeros = {0u, 0u, 0u, 0u};

// Accumulators of one column (rows: dims 32 x + 8 y + 4 hf + 0 .. 3 in registers 4 y .. of block x),
// times f, to the row's bf16 elements: the two lanes of the column exchange halves and each writes 16 bytes.
// Returns whether the column holds a NaN (in one of its lanes; also if it holds infinities of both signs).
template <int D>
__device__ inline bool store_row(__bf16* dst, const f32x16* o, float f, int hf, bool ok) {
  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
  float sum = 0.f;
#pragma unroll
  for (int x = 0; x < TileOf<D>::kDB; ++x)
#pragma unroll
    for (int y = 0; y < 4; y += 2) {
      u32x2 r[2];
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const f32x2 pr = {o[x][4 * (y + z) + 2 * e] * f, o[x][4 * (y + z) + 2 * e + 1] * f};
          const bf16x2 pb = __builtin_convertvector(pr, bf16x2);
          sum = __builtin_amdgcn_fdot2_f32_bf16(pb, ones, sum, false);
          r[z][e] = __builtin_bit_cast(uint32_t, pb);
        }
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const auto sw = __builtin_amdgcn_permlane32_swap(r[0][e], r[1][e], false, false);
        w[e] = sw[0];
        w[2 + e] = sw[1];
      }
      if (ok) *reinterpret_cast<u32x4*>(dst + 32 * x + 8 * y + 8 * hf) = w;
    }
  return is_nan(sum);
}

// ---------------------------------------------------------------------------
// Rows of a wave's 32 columns between memory and MFMA operands.  Column c of
// the block is row pl (Hq - g) + c past the block's first one (pl its position).
// Memory is read and written in whole 128-byte lines, 8 rows an instruction
// (lane l: row 8 m + l / 8, 16-byte piece l % 8 of a 64-element half), and the
// halves are turned in 4 KB of LDS of the wave's own, pieces permuted by row as
// in the tiles.  Read straight into operands (32 rows of 32 bytes an
// instruction) and written so, rows took 60 of the forward's 165 us (16384
// tokens of 8 x 5 heads, w = 256, 4 sinks).
// ---------------------------------------------------------------------------
constexpr int kTurn = 4096;   // LDS bytes of a wave's half rows
struct Rows {
  uint32_t off[4];   // bytes from the block's first row
  bool ok[4];
  uint32_t wr, rd;   // LDS offsets: this lane's piece of rows 8 m .. (m odd: ^ 32), of its column's row (k-step s: ^ 32 s)
};
template <int D>
__device__ inline Rows wave_rows(const WindowArgs& a, int wave, int lane, int positions) {
  Rows r;
  const int r8 = lane >> 3, c8 = lane & 7, col = lane & 31;
#pragma unroll
  for (int m = 0; m < 4; ++m) {
    const int c = wave * 32 + 8 * m + r8;
    const int pl = static_cast<int>(c * a.inv_g >> 16);
    r.ok[m] = pl < positions;
    r.off[m] = (r.ok[m] ? static_cast<uint32_t>(pl * (a.H - 1) * a.g + c) * TileOf<D>::kRowB : 0u) + 16 * c8;
  }
  r.wr = r8 * 128 + 16 * (c8 ^ row_flip<64>(r8));
  r.rd = col * 128 + 16 * ((lane >> 5) ^ piece_flip<64>(col));
  return r;
}
// Loads (not waited for) of the rows at `base`: piece set h * 4 + m is half h of rows 8 m ..
template <int D>
__device__ inline void load_rows(u32x4* x, const __bf16* base, const Rows& r) {
#pragma unroll
  for (int h = 0; h < D / 64; ++h)
#pragma unroll
    for (int m = 0; m < 4; ++m) x[4 * h + m] = ld16(reinterpret_cast<const char*>(base) + r.off[m] + 128 * h);
}
// Loaded rows to column operands, in place.
template <int D>
__device__ inline void to_operands(u32x4* x, const Rows& r, uint32_t turn) {
#pragma unroll
  for (int h = 0; h < D / 64; ++h) {
#pragma unroll
    for (int m = 0; m < 4; ++m)
      *reinterpret_cast<DMS_LDS u32x4*>(turn + 1024 * m + (r.wr ^ (32 * (m & 1)))) = x[4 * h + m];
#pragma unroll
    for (int s = 0; s < 4; ++s) x[4 * h + s] = *reinterpret_cast<DMS_LDS const u32x4*>(turn + (r.rd ^ (32 * s)));
  }
}
// Accumulators of the columns, times f (per column), to their bf16 rows.  Returns whether this lane's part of
// its column holds a NaN (also if it holds infinities of both signs).
template <int D>
__device__ inline bool store_rows(__bf16* base, const f32x16* o, float f, const Rows& r, uint32_t turn, int hf) {
  const bf16x2 ones = __builtin_bit_cast(bf16x2, 0x3F803F80u);
  float sum = 0.f;
#pragma unroll
  for (int h = 0; h < D / 64; ++h) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        u32x2 w;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const f32x2 pr = {o[2 * h + x][4 * y + 2 * e] * f, o[2 * h + x][4 * y + 2 * e + 1] * f};
          const bf16x2 pb = __builtin_convertvector(pr, bf16x2);
          sum = __builtin_amdgcn_fdot2_f32_bf16(pb, ones, sum, false);
          w[e] = __builtin_bit_cast(uint32_t, pb);
        }
        // piece 4 x + y of the half; the lane's 8 bytes of it (rd holds piece hf)
        *reinterpret_cast<DMS_LDS u32x2*>(turn + ((r.rd ^ (16 * hf)) ^ (16 * (4 * x + y))) + 8 * hf) = w;
      }
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const u32x4 v = *reinterpret_cast<DMS_LDS const u32x4*>(turn + 1024 * m + (r.wr ^ (32 * (m & 1))));
      if (r.ok[m]) *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(base) + r.off[m] + 128 * h) = v;
    }
  }
  return is_nan(sum);
}

// ---------------------------------------------------------------------------
// LDS ring of steps, each two 32-row tiles of 2 D bytes a row ([K | V] of 32
// keys): while one step is computed the next are on their way.  A window is few
// steps long, so that a workgroup spends as long waiting as computing unless its
// first copies leave together.  Wave x copies half x % 2 of tile x / 2.  Three
// slots (48 KB at d = 128) leave room for three workgroups per CU: 16384 tokens
// of 8 x 5 heads, w = 256, take 151 us, with four slots and two workgroups 165.
// ---------------------------------------------------------------------------
constexpr int kSlots = 3;
template <int D>
constexpr int kCopies = D / 32;   // copies of a step by one wave

// Wave x copies its half of tile i of the listed keys; only a tile that holds both the last sinks and the
// window's first keys takes each row by itself.
template <int D>
__device__ inline void copy_keys(const WindowArgs& a, const KeyTiles& kt, const char* kv, int i, int end, uint32_t stride,
                                 const LaneOffsets& lo, int lane, int wave, uint32_t dst) {
  dst += TileOf<D>::kUnit * (wave >> 1);
  const bool mixed = 32 * i < a.sinks && 32 * i + 32 > a.sinks && kt.base > 0;
  if (!mixed) {
    copy_tile<D, 2>(kv, 32 * i < a.sinks ? 32 * i : kt.base + 32 * i, end, stride, lo, lane, dst, &kZeros, wave & 1);
    return;
  }
  // both parts at the places of their rows, each lane in one of the two copies (a wait for the newest copies
  // counts them as one: it waits for more than it has to)
  constexpr int kRows = kCopyRows<D>;
  const int tr = fresh(lane) / (D / 8);
#pragma unroll
  for (int m0 = 0; m0 < 32 / kRows; m0 += 2) {
    const int m = m0 + (wave & 1), e = 32 * i + kRows * m;
    const uint32_t off = lo.src ^ copy_flip<D>(m);
    if (e + tr < a.sinks) lds_copy16(kv + static_cast<size_t>(e) * stride, off, dst + 1024 * m);
    else if (kt.base + e + tr < end) lds_copy16(kv + static_cast<size_t>(kt.base + e) * stride, off, dst + 1024 * m);
    else lds_copy16(&kZeros, dst + 1024 * m);
  }
}

// Of the steps after this one `left` are there to come and the first has been issued: this one has landed for
// every wave.
template <int D>
__device__ inline void step_ready(int left) {
  if (left >= 1) wait_copies_but<kCopies<D>>();
  else wait_copies();
  __syncthreads();
}

// f(step, slot) for steps 0 .. n - 1, the slot a constant.
template <typename F>
__device__ __forceinline__ void over_steps(int n, F f) {
  for (int i = 0; i < n; i += kSlots) {
    f(i, std::integral_constant<int, 0>{});
    if (i + 1 < n) f(i + 1, std::integral_constant<int, 1>{});
    if (i + 2 < n) f(i + 2, std::integral_constant<int, 2>{});
  }
}

// ---------------------------------------------------------------------------
// Forward.  Workgroup = (KV head, block of PB positions of one sequence);
// columns are (position, query head) pairs, the g heads of a position
// consecutive, 32 per wave.  The block's key tiles go through the LDS ring.
// 16384 tokens of 8 x 5 heads, d = 128, w = 256, 4 sinks (405 MB, 86 GFLOP) take
// 136 to 146 us among other calls (25 launches in a row from an idle clock 130 to
// 205, 160 to 170 on average), d = 64 77 to 80.  A steady tile's 16 products take 512
// cycles of a SIMD's matrix core beside 58 vector instructions and 16
// exponentials at a quarter of the rate, 488 cycles, and long walks run at the
// matrix core's rate (w = 4096: 1.0 ms, 1.2 PFLOP/s).  At w = 256 a walk is 9
// tiles, and what lies around its steady tiles (the sequence search, the rows'
// turns, edge masks, the first rescale) brings it to 162 vector instructions a
// tile and leaves the matrix core 38 % busy.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(kThreads, 3) void window_fwd_kernel(WindowArgs a) {
  using Tile = TileOf<D>;
  constexpr int kUnit = Tile::kUnit, kKS = Tile::kKS, kDB = Tile::kDB;
  // the last slot, idle until the first step, and its end (D = 64) also turn the waves' rows
  constexpr int kTurnAt = (kSlots - 1) * 2 * kUnit;
  __shared__ __attribute__((aligned(256))) char tile_lds[kTurnAt + (D == 128 ? 2 * kUnit : 4 * kTurn)];
  const int2 wg = xcd_order();
  const int h = wg.y;
  const Block blk = block_of(a, wg.x, a.PB, a.inv_pb);
  if (blk.p0 >= blk.len) return;
  const int s0 = blk.s0, p0 = blk.p0, p1 = min(blk.len, p0 + a.PB);
  const KeyTiles kt = key_tiles(a, p0, p1);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hf = lane >> 5;
  const int Hq = a.H * a.g;

  const uint32_t stride = a.H * Tile::kRowB;
  const LaneOffsets lo = lane_offsets<D>(lane, stride);
  const uint32_t tiles = lds_addr(tile_lds);
  const char* kv = reinterpret_cast<const char*>((wave >> 1 ? a.v : a.k) + (static_cast<size_t>(s0) * a.H + h) * D);
  auto issue = [&](int i, int slot) { copy_keys<D>(a, kt, kv, i, blk.len, stride, lo, lane, wave, tiles + slot * 2 * kUnit); };
#pragma unroll
  for (int i = 0; i < kSlots - 1; ++i)
    if (i < kt.nt) issue(i, i);

  const int col = wave * 32 + (lane & 31);
  const int pl = static_cast<int>(col * a.inv_g >> 16), qh = col - pl * a.g;
  const bool ok = pl < a.PB && p0 + pl < p1;
  const int t = ok ? p0 + pl : p0;
  const size_t first_row = static_cast<size_t>(s0 + p0) * Hq + h * a.g;
  const Rows rows = wave_rows<D>(a, wave, lane, p1 - p0);
  u32x4 qf[kKS];
  load_rows<D>(qf, a.q + first_row * D, rows);
  // positions of this wave's columns
  const int q0 = p0 + static_cast<int>(wave * 32 * a.inv_g >> 16);
  const WaveTiles wt = wave_tiles(a, kt, q0, min(p1 - 1, p0 + static_cast<int>((wave * 32 + 31) * a.inv_g >> 16)));
  const LaneAddresses<D> ad = lane_addresses<D>(tiles, lo);

  f32x16 o[kDB];
#pragma unroll
  for (int x = 0; x < kDB; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[x][i] = 0.f;
  to_operands<D>(qf, rows, tiles + kTurnAt + wave * kTurn);
  float m_ref = kMInit, l_run = 0.f;
  const float thr = kRescale / a.scale_log2;

  over_steps(kt.nt, [&](int i, auto slot_c) {
    constexpr int slot = decltype(slot_c)::value, tl = slot * 2 * kUnit;
    step_ready<D>(kt.nt - 1 - i);
    if (i + kSlots - 1 < kt.nt) issue(i + kSlots - 1, (slot + kSlots - 1) % kSlots);
    if (!tile_seen(wt, i)) return;
    f32x16 s;
#pragma unroll
    for (int x = 0; x < 16; ++x) s[x] = 0.f;
    u32x4 op[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) op[e] = row_operand(tl, ad, e);
#pragma unroll
    for (int e = 0; e < kKS; ++e) {
      __builtin_amdgcn_sched_barrier(0);
      s = mfma(op[e % kAhead], qf[e], s);
      if (e + kAhead < kKS) op[e % kAhead] = row_operand(tl, ad, e + kAhead);
    }
    __builtin_amdgcn_sched_barrier(0);
    hide(s, a, kt, wt, i, t, hf);
    // value product e: token half e / kDB, dim block e % kDB
    auto read_v = [&](int e) { return col_operand(tl + kUnit, ad, e % kDB, e / kDB); };
#pragma unroll
    for (int e = 0; e < kAhead; ++e) op[e] = read_v(e);
    float mx = max3(s[0], s[1], s[2]);
#pragma unroll
    for (int x = 3; x < 15; x += 2) mx = max3(mx, s[x], s[x + 1]);
    mx = col_max(fmaxf(mx, s[15]));
    const bool raise = mx > m_ref + thr;
    if (__builtin_amdgcn_ballot_w64(raise)) {
      const float m_new = raise ? mx : m_ref;
      const float f = __builtin_amdgcn_exp2f((m_ref - m_new) * a.scale_log2);
      l_run *= f;
#pragma unroll
      for (int x = 0; x < kDB; ++x) o[x] *= f;
      m_ref = m_new;
    }
    const float mb = m_ref * a.scale_log2;
    // the products take weights rounded to bf16 (half a step, 2^-8 of each, averaged over the row); the
    // denominator adds them unrounded, so that lse keeps float32 precision
    u32x4 pu[2];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const f32x2 pr = {__builtin_amdgcn_exp2f(fmaf(s[2 * j], a.scale_log2, -mb)),
                        __builtin_amdgcn_exp2f(fmaf(s[2 * j + 1], a.scale_log2, -mb))};
      l_run += pr[0] + pr[1];
      pu[j >> 2][j & 3] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, bf16x2));
    }
#pragma unroll
    for (int e = 0; e < 2 * kDB; ++e) {
      __builtin_amdgcn_sched_barrier(0);
      o[e % kDB] = mfma(op[e % kAhead], pu[e / kDB], o[e % kDB]);
      if (e + kAhead < 2 * kDB) op[e % kAhead] = read_v(e + kAhead);
    }
    __builtin_amdgcn_sched_barrier(0);
  });

  const float l = col_sum(l_run);
  const float inv = 1.0f / l;
  __syncthreads();   // every wave is done with the tiles
  // (weights that add to a NaN are those of visible scores: all of the row is NaN)
  const bool bad = (store_rows<D>(a.out + first_row * D, o, inv, rows, tiles + wave * kTurn, hf) || not_finite(inv)) && !is_nan(l);
  if (ok && hf == 0)
    a.lse_out[static_cast<size_t>(h * a.g + qh) * a.T + s0 + t] = (m_ref * a.scale_log2 + __log2f(l)) * kLn2;
  const uint64_t lanes = __builtin_amdgcn_ballot_w64(bad && ok);
  for (uint32_t cols = static_cast<uint32_t>(lanes | lanes >> 32); cols; cols &= cols - 1) {
    const int c = wave * 32 + __builtin_ctz(cols);
    exact_row<D>(a, s0, p0 + c / a.g, h * a.g + c % a.g);
  }
}

// ---------------------------------------------------------------------------
// dQ pass.  Workgroups, columns and tiles as in the forward.  Two walks over
// the key tiles, each S^T = K Q^T and dP^T = V dO^T over rows: the first sums
// D_t from P and dP, the second adds dQ^T += K^T dS^T over columns.  The pass
// also leaves -lse and -D of every row to the key-major pass.
// D_t from dO and the rounded `out` costs no walk, but errors of up to 5 times a
// row's own dQ where its weights are peaked (queries of scale 8, w = 256), with
// dS in two bf16 parts in the last product already.  The walk makes a backward
// of 16384 tokens of 8 x 5 heads take 573 us instead of 531 at w = 256, 1499
// instead of 1328 at w = 1024.  The pass takes 290 to 330 us of the former (two
// waves of 237 registers per SIMD, matrix core 44 % busy).
// ---------------------------------------------------------------------------
// A dQ row as exact_row above, whose lse is no NaN; the row's values for the key-major pass go with it.
template <int D>
__device__ inline void exact_dq_row(const WindowArgs& a, int s0, int t, int hq) {
  const int lane = threadIdx.x & 63, Hq = a.H * a.g, h = hq / a.g;
  auto key_row = [&](int j) { return (static_cast<size_t>(s0 + j) * a.H + h) * D; };
  const size_t row = (static_cast<size_t>(s0 + t) * Hq + hq) * D;
  after_stores();
  const uint32_t was = pair_of<D>(a.dq + row), own = pair_of<D>(a.v + key_row(t));
  const uint32_t q = pair_of<D>(a.q + row), dO = pair_of<D>(a.dout + row);
  const bool open0 = is_nan(low(was)), open1 = is_nan(high(was));
  // a NaN D makes all of the row NaN, as it was stored
  if (any_lane(is_nan(low(own)) || is_nan(high(own)) || is_nan(low(dO)) || is_nan(high(dO)))) return;
  const float lse2 = a.lse[static_cast<size_t>(hq) * a.T + s0 + t] * kLog2e;
  float dq0 = 0.f, dq1 = 0.f, d = 0.f, sum = 0.f;
  const int base = max(0, t - a.w + 1 - a.sinks), keys = t + 1 - base;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
    for (int k0 = 0; k0 < keys; k0 += 64) {
      const bool in = k0 + lane < keys;
      const size_t kr = key_row(seen_key(a, base, min(k0 + lane, keys - 1)));
      const float x = exp2f(row_dot<D>(a.k + kr, q) * a.scale_log2 - lse2), dp = row_dot<D>(a.v + kr, dO);
      if (!pass) {
        d += wave_sum(in ? x * dp : 0.f);
        sum += wave_sum(in ? x : 0.f);
        if (is_nan(d)) return;
        continue;
      }
      const float ds = x * (dp - d);
      const int n = min(64, keys - k0);
#pragma unroll 1
      for (int i = 0; i < n; i += kAdd) {
        uint32_t k[kAdd];
#pragma unroll
        for (int u = 0; u < kAdd; ++u) k[u] = i + u < n ? pair_of<D>(a.k + key_row(seen_key(a, base, k0 + i + u))) : 0u;
#pragma unroll
        for (int u = 0; u < kAdd; ++u) {
          const float du = i + u < n ? lane_value(ds, i + u) : 0.f;
          dq0 += du * low(k[u]);
          dq1 += du * high(k[u]);
        }
        if (!any_lane((open0 && !is_nan(dq0)) || (open1 && !is_nan(dq1)))) return;
      }
    }
    if (!pass) {
      d /= sum;
      if (lane == 0) {
        a.nlse[hq * a.Ts + s0 + t] = -lse2 / a.scale_log2;
        a.nsum[hq * a.Ts + s0 + t] = -d;
      }
    }
  }
  const float scale = a.scale_log2 / kLog2e;
  store_pair<D>(a.dq + row, a.single ? 0.f : dq0 * scale, a.single ? 0.f : dq1 * scale);
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void window_dq_kernel(WindowArgs a) {
  using Tile = TileOf<D>;
  constexpr int kUnit = Tile::kUnit, kKS = Tile::kKS, kDB = Tile::kDB;
  // [K | V] of two tiles, twice; the second pair of tiles, idle until the first step, also turns the waves' rows
  __shared__ __attribute__((aligned(256))) char tile_lds[2][4 * kUnit];
  const int2 wg = xcd_order();
  const int h = wg.y;
  const Block blk = block_of(a, wg.x, a.PB, a.inv_pb);
  if (blk.p0 >= blk.len) return;
  const int s0 = blk.s0, p0 = blk.p0, p1 = min(blk.len, p0 + a.PB);
  const KeyTiles kt = key_tiles(a, p0, p1);
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hf = lane >> 5;
  const int Hq = a.H * a.g;

  const uint32_t stride = a.H * Tile::kRowB;
  const LaneOffsets lo = lane_offsets<D>(lane, stride);
  const uint32_t tiles = lds_addr(tile_lds);
  const char* kv = reinterpret_cast<const char*>((wave >> 1 ? a.v : a.k) + (static_cast<size_t>(s0) * a.H + h) * D);
  const int steps = (kt.nt + 1) >> 1;
  auto issue = [&](int st, int buf) {
    copy_keys<D>(a, kt, kv, 2 * st, blk.len, stride, lo, lane, wave, tiles + buf * 4 * kUnit);
    if (2 * st + 1 < kt.nt)
      copy_keys<D>(a, kt, kv, 2 * st + 1, blk.len, stride, lo, lane, wave, tiles + buf * 4 * kUnit + 2 * kUnit);
  };
  issue(0, 0);

  const int col = wave * 32 + (lane & 31);
  const int pl = static_cast<int>(col * a.inv_g >> 16), qh = col - pl * a.g;
  const bool ok = pl < a.PB && p0 + pl < p1;
  const int t = ok ? p0 + pl : p0;
  const size_t first_row = static_cast<size_t>(s0 + p0) * Hq + h * a.g;
  const Rows rows = wave_rows<D>(a, wave, lane, p1 - p0);
  const uint32_t turn = tiles + 4 * kUnit + wave * kTurn;
  u32x4 qf[kKS], df[kKS];
  load_rows<D>(qf, a.q + first_row * D, rows);
  load_rows<D>(df, a.dout + first_row * D, rows);
  float dcol = 0.f, psum = 0.f;
  to_operands<D>(qf, rows, turn);
  to_operands<D>(df, rows, turn);
  const size_t at = static_cast<size_t>(h * a.g + qh) * a.T + s0 + t;
  const float lse2 = ok ? a.lse[at] * kLog2e : 0.f;
  const int q0 = p0 + static_cast<int>(wave * 32 * a.inv_g >> 16);
  const WaveTiles wt = wave_tiles(a, kt, q0, min(p1 - 1, p0 + static_cast<int>((wave * 32 + 31) * a.inv_g >> 16)));
  const LaneAddresses<D> ad = lane_addresses<D>(tiles, lo);

  f32x16 dqa[kDB], start;   // -D in every row starts the dP products
  auto attend = [&](int st, auto buf_c, auto sum_c) {
    constexpr int buf = decltype(buf_c)::value;
    constexpr bool kSum = decltype(sum_c)::value;   // only summing D
    wait_copies();
    __syncthreads();
    if (st + 1 < steps) issue(st + 1, buf ^ 1);
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
      const int i = 2 * st + sub;
      const int tl = buf * 4 * kUnit + 2 * kUnit * sub;
      if (i >= kt.nt || !tile_seen(wt, i)) continue;
      f32x16 s, dp;
      u32x4 op[kAhead];
      // product e: scores (keys) and dP (values) take turns, k-step e / 2
#pragma unroll
      for (int e = 0; e < kAhead; ++e) op[e] = row_operand(tl + kUnit * (e & 1), ad, e >> 1);
#pragma unroll
      for (int e = 0; e < 2 * kKS; ++e) {
        __builtin_amdgcn_sched_barrier(0);
        if (e & 1) dp = mfma(op[e % kAhead], df[e >> 1], e > 1 ? dp : kSum ? f32x16{} : start);
        else s = mfma(op[e % kAhead], qf[e >> 1], e ? s : f32x16{});
        if (e + kAhead < 2 * kKS) op[e % kAhead] = row_operand(tl + kUnit * (e & 1), ad, (e + kAhead) >> 1);
      }
      __builtin_amdgcn_sched_barrier(0);
      hide(s, a, kt, wt, i, t, hf);
      if constexpr (kSum) {
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[x], a.scale_log2, -lse2));
          dcol += p * dp[x];
          psum += p;
        }
      } else {
#pragma unroll
        for (int e = 0; e < kAhead; ++e) op[e] = col_operand(tl, ad, e % kDB, e / kDB);
        float ds[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) ds[x] = __builtin_amdgcn_exp2f(fmaf(s[x], a.scale_log2, -lse2)) * dp[x];
        const u32x4 du[2] = {pack_bf16(ds), pack_bf16(ds + 8)};   // half a step, 2^-8 of each, averaged over the row
#pragma unroll
        for (int e = 0; e < 2 * kDB; ++e) {
          __builtin_amdgcn_sched_barrier(0);
          dqa[e % kDB] = mfma(op[e % kAhead], du[e / kDB], dqa[e % kDB]);
          if (e + kAhead < 2 * kDB) op[e % kAhead] = col_operand(tl, ad, (e + kAhead) % kDB, (e + kAhead) / kDB);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  auto walk = [&](auto sum_c) {
    for (int st = 0; st < steps; st += 2) {
      attend(st, std::integral_constant<int, 0>{}, sum_c);
      if (st + 1 < steps) attend(st + 1, std::integral_constant<int, 1>{}, sum_c);
    }
  };
  walk(std::true_type{});
  dcol = col_sum(dcol) / col_sum(psum);
  __syncthreads();   // every wave is done with the tiles
  issue(0, 0);
#pragma unroll
  for (int i = 0; i < 16; ++i) start[i] = -dcol;
#pragma unroll
  for (int x = 0; x < kDB; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) dqa[x][i] = 0.f;
  walk(std::false_type{});

  if (ok) (hf ? a.nsum : a.nlse)[static_cast<size_t>(h * a.g + qh) * a.Ts + s0 + t] = hf ? -dcol : -lse2 / a.scale_log2;
  const float scale = a.single ? 0.f : a.scale_log2 / kLog2e;
  __syncthreads();   // every wave is done with the tiles
  const bool bad = (store_rows<D>(a.dq + first_row * D, dqa, scale, rows, tiles + wave * kTurn, hf) || not_finite(dcol)) && !is_nan(lse2);
  const uint64_t lanes = __builtin_amdgcn_ballot_w64(bad && ok);
  for (uint32_t cols = static_cast<uint32_t>(lanes | lanes >> 32); cols; cols &= cols - 1) {
    const int c = wave * 32 + __builtin_ctz(cols);
    exact_dq_row<D>(a, s0, p0 + c / a.g, h * a.g + c % a.g);
  }
}

// ---------------------------------------------------------------------------
// dK / dV pass.  Workgroup = (KV head, 128 keys of one sequence, share of the
// steps); wave x owns 32 of the keys as the columns of its products, with their
// K and V operands in registers, and walks the query tiles (32 positions) that
// see the block, every head of the group: dV^T += dO^T P, dK^T += Q^T dS with
// P, dS [query, key] from S = Q K^T, dP = dO V^T.
// At d = 128 sums, operands and one step's scores fill the 256 registers of two
// waves per SIMD, so that a wave takes one step at a time, with operands read two
// ahead: while one wave forms weights the other has the matrix core.  16384 tokens
// of 8 x 5 heads, w = 256, 4 sinks: 290 to 300 us at the shortest, 333 on average of 25
// launches in a row, matrix core 39 % busy.  One wave of 512 registers that takes
// two steps together, operands read six ahead, ran 400 us against 300; three and
// four ahead spill in this form (+80 us).  Every step clears hidden weights, 48 of
// its 126 vector instructions, and a wave waits through 3 of the 12 query tiles
// that its block walks.
// A sink is seen by every later query.  A block that holds sinks walks on to
// position `far`; what lies further is shared out to workgroups of `far`
// positions, whose waves take the steps in turn.
// When the call has too few blocks to fill the chip, each block's steps are
// split over `splits` workgroups.  Sums that several workgroups hold are added,
// in order, by window_sum_kernel.
// ---------------------------------------------------------------------------
constexpr int kKeys = 128;
constexpr int kSplitTarget = 256;   // key blocks below which their steps are split
constexpr int kMaxSplits = 8;
constexpr int kStages = 2;     // pairs of steps in LDS (four single ones, a barrier each: 46 us more of 652)
constexpr int kDeep = 2;        // operands are read this many products ahead

// First position (a multiple of 32) that the block of keys from j0 on leaves to others.
__device__ inline int far_begin(const WindowArgs& a, int j0) {
  const int end = j0 + ((kKeys + a.w + 31) & ~31);
  return j0 < a.sinks ? max(end, a.far) : end;
}

// dK and dV of key j as exact_row above, from the queries that see it.
template <int D>
__device__ inline void exact_key(const WindowArgs& a, int s0, int len, int j, int h) {
  const int lane = threadIdx.x & 63, Hq = a.H * a.g;
  // row r: query j + r / g, head r % g of the group
  auto query_row = [&](int r) { return (static_cast<size_t>(s0 + j + r / a.g) * Hq + h * a.g + r % a.g) * D; };
  auto value_at = [&](int r) { return (h * a.g + r % a.g) * a.Ts + s0 + j + r / a.g; };
  const size_t kr = (static_cast<size_t>(s0 + j) * a.H + h) * D;
  after_stores();
  const uint32_t was_k = pair_of<D>(a.dk + kr), was_v = pair_of<D>(a.dv + kr), own = pair_of<D>(a.dout + query_row(0));
  const bool no_p = is_nan(a.nlse[value_at(0)]), no_ds = no_p || is_nan(a.nsum[value_at(0)]);
  const bool open_k0 = is_nan(low(was_k)) && !no_ds, open_k1 = is_nan(high(was_k)) && !no_ds;
  const bool open_v0 = is_nan(low(was_v)) && !no_p && !is_nan(low(own)), open_v1 = is_nan(high(was_v)) && !no_p && !is_nan(high(own));
  if (!any_lane(open_k0 || open_k1 || open_v0 || open_v1)) return;
  if (j < a.sinks) {
    // The only queries that its sums met unseen are those before it in its tile of 32: where these are finite
    // every NaN comes from a visible one (its walk would take all of a long sequence to tell).
    bool met = false;
    const int before = (j & 31) * a.g;
#pragma unroll 1
    for (int r = 0; r < before; ++r) {
      const size_t qr = (static_cast<size_t>(s0 + (j & ~31) + r / a.g) * Hq + h * a.g + r % a.g) * D;
      const uint32_t q = pair_of<D>(a.q + qr), dO = pair_of<D>(a.dout + qr);
      met |= not_finite(low(q)) || not_finite(high(q)) || not_finite(low(dO)) || not_finite(high(dO));
    }
    if (!any_lane(met)) return;
  }
  const uint32_t k = pair_of<D>(a.k + kr), v = pair_of<D>(a.v + kr);
  float dk0 = 0.f, dk1 = 0.f, dv0 = 0.f, dv1 = 0.f;
  const int end = j < a.sinks ? len : static_cast<int>(min<int64_t>(len, static_cast<int64_t>(j) + a.w));
  const int rows = (end - j) * a.g;
#pragma unroll 1
  for (int r0 = 0; r0 < rows; r0 += 64) {
    const int mine = min(r0 + lane, rows - 1);
    const size_t qr = query_row(mine), at = value_at(mine);
    const float p = exp2f((row_dot<D>(a.q + qr, k) + a.nlse[at]) * a.scale_log2);
    const float ds = p * (row_dot<D>(a.dout + qr, v) + a.nsum[at]);
    const int n = min(64, rows - r0);
#pragma unroll 1
    for (int i = 0; i < n; i += kAdd) {
      uint32_t q[kAdd], dO[kAdd];
#pragma unroll
      for (int u = 0; u < kAdd; ++u) {
        const size_t x = query_row(min(r0 + i + u, rows - 1));
        q[u] = i + u < n ? pair_of<D>(a.q + x) : 0u;
        dO[u] = i + u < n ? pair_of<D>(a.dout + x) : 0u;
      }
#pragma unroll
      for (int u = 0; u < kAdd; ++u) {
        const float pu = i + u < n ? lane_value(p, i + u) : 0.f, du = i + u < n ? lane_value(ds, i + u) : 0.f;
        dv0 += pu * low(dO[u]);
        dv1 += pu * high(dO[u]);
        dk0 += du * low(q[u]);
        dk1 += du * high(q[u]);
      }
      if (!any_lane((open_k0 && !is_nan(dk0)) || (open_k1 && !is_nan(dk1)) || (open_v0 && !is_nan(dv0)) ||
                    (open_v1 && !is_nan(dv1))))
        return;
    }
  }
  const float scale = a.scale_log2 / kLog2e;
  store_pair<D>(a.dk + kr, a.single ? 0.f : dk0 * scale, a.single ? 0.f : dk1 * scale);
  store_pair<D>(a.dv + kr, dv0, dv1);
}

// Sums of the far queries of slot b: positions far c .. of the sequence that starts in the packed tokens'
// (b - c)-th `far`, c >= 1.  Only sequences longer than that have any, so that no two share a slot.
__device__ inline float* far_sums(const WindowArgs& a, int slot, int tile, int h, int D) {
  return a.far_part + ((static_cast<size_t>(slot) * a.sink_tiles + tile) * a.H + h) * 64 * D;
}
// Sums of a tile of sinks from its key block, where nothing else is shared: of the sequence that starts in the
// packed tokens' slot-th `far`.
__device__ inline float* near_sums(const WindowArgs& a, int slot, int tile, int h, int D) {
  return far_sums(a, divide(a.T, a.far, a.inv_far) + 1 + slot, tile, h, D);
}
// Sums of one share of a key block: row of packed token t.
__device__ inline float* share_sums(const WindowArgs& a, int split, int t, int h, int D) {
  return a.part + ((static_cast<size_t>(split) * a.T + t) * a.H + h) * 2 * D;
}

// The list of (query tile, head) steps of a workgroup: `tiles` tiles of positions from pos0 on, beginning with
// tile `start` and around to the one before it, heads inside a tile.  Key blocks begin with the tile whose
// number is a multiple of the tiles that a block sees: blocks of one sequence that run together then read the
// same tile at about the same time, and each XCD's L2 serves most of them (each block beginning with its own
// first tile, copies took 1.1 GB past the L2s and 180 us).
struct StepList {
  int pos0, tiles, start, g;
  int qh, tile;           // current step
  __device__ void seek(int step) {
    qh = step % g;
    tile = start + step / g;
    while (tile >= tiles) tile -= tiles;
  }
  __device__ void skip(int n) {
    qh += n;
    while (qh >= g) {
      qh -= g;
      if (++tile >= tiles) tile -= tiles;
    }
  }
  __device__ int pos() const { return pos0 + 32 * tile; }
};

// Copies the steps, two at a time, through a ring of stages: [Q | dO] of both steps, then their rows' -lse and -D.
template <int D>
struct QuerySteps {
  static constexpr int kUnit = TileOf<D>::kUnit;
  static constexpr int kBytes = 4 * kUnit;             // tiles of a stage
  const char* src;        // this wave's tensor (queries or output gradients): first head, first token
  const float* rows;      // this wave's row values
  int64_t head_step;
  int len, wave, lane;
  uint32_t stride, tiles, row_lds;
  StepList ld;            // this wave's next step

  __device__ QuerySteps(const WindowArgs& a, int s0, int len_, int h, const StepList& list, int first, int wave_,
                        int lane_, uint32_t tiles_, uint32_t row_lds_)
      : len(len_), wave(wave_), lane(lane_), tiles(tiles_), row_lds(row_lds_), ld(list) {
    const int Hq = a.H * a.g;
    stride = Hq * TileOf<D>::kRowB;
    // wave x copies tensor x / 2 and row values x / 2 of step 2 st + x % 2
    src = reinterpret_cast<const char*>((wave >> 1 ? a.dout : a.q) + (static_cast<size_t>(s0) * Hq + h * a.g) * D);
    rows = (wave >> 1 ? a.nsum : a.nlse) + h * a.g * a.Ts + s0;
    head_step = a.Ts;
    ld.seek(first + (wave & 1));
  }
  __device__ void issue(int stage, const LaneOffsets& lo) {
    // (a step past the last is copied like the others, so that waits can count copies, and read by nobody)
    copy_tile<D>(src + static_cast<size_t>(ld.qh) * TileOf<D>::kRowB, ld.pos(), len, stride, lo, lane,
                 tiles + stage * kBytes + 2 * kUnit * (wave & 1) + kUnit * (wave >> 1), &kZeros);
    lds_copy4(rows + ld.qh * head_step + ld.pos(), 4 * fresh(lane), row_lds + 1024 * stage + 512 * (wave & 1) + 256 * (wave >> 1));
    ld.skip(2);
  }
};

// One step for one wave's 32 keys from key0 on: its tiles from LDS address `tl` on, its rows' values from `rows`
// on, its queries from position tq on.
template <int D>
__device__ __forceinline__ void key_step(const WindowArgs& a, LaneOffsets lo, uint32_t tl, uint32_t rows, int tq,
                                         int key0, int len, int lane, const u32x4* kf, const u32x4* vf, f32x16* dka,
                                         f32x16* dva) {
  constexpr int kUnit = TileOf<D>::kUnit, kKS = TileOf<D>::kKS, kDB = TileOf<D>::kDB;
  const int hf = lane >> 5;
  f32x16 s, dp;
  // -lse and -D of the rows start the products: register i of a lane is query tq + 16 (i / 8) + 8 hf + i % 8
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t r = rows + 32 * hf + 4 * (16 * (i >> 1) + 4 * (i & 1));
    const f32x4 l = *reinterpret_cast<DMS_LDS const f32x4*>(r), d = *reinterpret_cast<DMS_LDS const f32x4*>(r + 256);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[4 * i + e] = l[e];
      dp[4 * i + e] = d[e];
    }
  }
  // addresses are formed here, by an exclusive or each: held ahead of the loop they do not fit the registers
  refresh(lo);
  const uint32_t row0 = tl + lo.row, col0 = tl + lo.col;
  // product e: scores (Q rows) and dP (dO rows) take turns
  auto read_row = [&](int e) {
    return *reinterpret_cast<DMS_LDS const u32x4*>((row0 ^ (32 * (e >> 1))) + (e & 1) * kUnit);
  };
  constexpr int kProd = 2 * kKS, kSum = 4 * kDB;
  u32x4 op[kDeep];
#pragma unroll
  for (int e = 0; e < kDeep; ++e) op[e] = read_row(e);
#pragma unroll
  for (int e = 0; e < kProd; ++e) {
    __builtin_amdgcn_sched_barrier(0);
    if (e & 1) dp = mfma(op[e % kDeep], vf[e >> 1], dp);
    else s = mfma(op[e % kDeep], kf[e >> 1], s);
    if (e + kDeep < kProd) op[e % kDeep] = read_row(e + kDeep);
  }
  __builtin_amdgcn_sched_barrier(0);
  // sum e: dV (dO columns) and dK (Q columns) take turns
  auto read_col = [&](int e) {
    const int x = e >> 1;   // dim block x % kDB, query half x / kDB
    const uint32_t at = (col0 ^ (64 * (x % kDB))) + (e & 1 ? 0 : kUnit) + 16 * (x / kDB) * TileOf<D>::kRowB;
    const uint32_t at4 = (col0 ^ (64 * (x % kDB)) ^ 16) + (e & 1 ? 0 : kUnit) + (16 * (x / kDB) + 4) * TileOf<D>::kRowB;
    const u32x2 l = tr_read16(at), h = tr_read16(at4);
    return u32x4{l[0], l[1], h[0], h[1]};
  };
#pragma unroll
  for (int e = 0; e < kDeep; ++e) op[e] = read_col(e);
  // bit c of a lane's mask: query tq + 8 hf + c sees its key.  Hidden weights are cleared in their packed words,
  // whatever they are (rows of no sequence have any values).
  const int j = key0 + (lane & 31), t0 = tq + 8 * hf;
  const int end = min(len - t0, j < a.sinks ? len - t0 : j - t0 + a.w);
  const uint32_t seen = ((1u << min(max(end, 0), 24)) - 1) & ~((1u << min(max(j - t0, 0), 24)) - 1);
  u32x4 pu[2], du[2];   // P = exp(s - lse) and dS = P dP, rounded to bf16
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const f32x2 p = {__builtin_amdgcn_exp2f(s[2 * e] * a.scale_log2), __builtin_amdgcn_exp2f(s[2 * e + 1] * a.scale_log2)};
    const int c = 16 * (e >> 2) + 2 * (e & 3);
    const uint32_t lo_m = __builtin_amdgcn_sbfe(seen, c, 1), hi_m = __builtin_amdgcn_sbfe(seen, c + 1, 1);
    const uint32_t m = (lo_m & 0xFFFFu) | (hi_m & 0xFFFF0000u);
    pu[e >> 2][e & 3] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2)) & m;
    const f32x2 d = {p[0] * dp[2 * e], p[1] * dp[2 * e + 1]};
    du[e >> 2][e & 3] = __builtin_bit_cast(uint32_t, __builtin_convertvector(d, bf16x2)) & m;
  }
#pragma unroll
  for (int e = 0; e < kSum; ++e) {
    __builtin_amdgcn_sched_barrier(0);
    const int x = e >> 1, b = x % kDB, half = x / kDB;
    if (e & 1) dka[b] = mfma(op[e % kDeep], du[half], dka[b]);
    else dva[b] = mfma(op[e % kDeep], pu[half], dva[b]);
    if (e + kDeep < kSum) op[e % kDeep] = read_col(e + kDeep);
  }
  __builtin_amdgcn_sched_barrier(0);
}

// Accumulators of one key (column) to float32 rows.
template <int D>
__device__ inline void store_sums(float* dst, const f32x16* o, int hf) {
#pragma unroll
  for (int x = 0; x < TileOf<D>::kDB; ++x)
#pragma unroll
    for (int y = 0; y < 4; ++y)
      *reinterpret_cast<f32x4*>(dst + 32 * x + 8 * y + 4 * hf) =
          f32x4{o[x][4 * y], o[x][4 * y + 1], o[x][4 * y + 2], o[x][4 * y + 3]};
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void window_dkv_kernel(WindowArgs a) {
  using Tile = TileOf<D>;
  using Steps = QuerySteps<D>;
  constexpr int kUnit = Tile::kUnit, kKS = Tile::kKS, kDB = Tile::kDB;
  __shared__ __attribute__((aligned(256))) char tile_lds[kStages * Steps::kBytes];
  __shared__ __attribute__((aligned(16))) float row_lds[kStages][2][2][64];               // [step][-lse, -D][row]
  const int2 wg = xcd_order();
  const int h = wg.y;
  const int lane = threadIdx.x & 63, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t tiles = lds_addr(tile_lds), rows = lds_addr(row_lds);
  // the key blocks of `far` tokens, each in its shares, then the far queries of as many positions, once per
  // tile of sinks
  const int near = a.far / kKeys * a.splits;
  const int group = wg.x / (near + a.sink_tiles), in_group = wg.x % (near + a.sink_tiles);
  const bool far = in_group >= near;
  int s0, len, key0, pos0, first = 0, total;   // sequence, this wave's keys, the steps' first position, this share of them
  StepList list;
  list.g = a.g;
  list.start = 0;
  if (far) {
    // positions far c .. (c >= 1) of the last sequence that starts before this `far` of the packed tokens
    if (group == 0) return;
    const Block f = block_of(a, group - 1, a.far, a.inv_far, 0);
    s0 = f.s0;
    len = f.len;
    key0 = 32 * (in_group - near);
    pos0 = max(f.p0 + a.far, far_begin(a, key0 & ~(kKeys - 1)));
    const int last = static_cast<int>(min<int64_t>(len, f.p0 + 2 * static_cast<int64_t>(a.far)));
    if (pos0 >= last || key0 >= len) return;
    list.tiles = (last - pos0 + 31) / 32;
    total = list.tiles * a.g;
  } else {
    const Block b = block_of(a, a.far / kKeys * group + in_group / a.splits, kKeys, inverse(kKeys));
    if (b.p0 >= b.len) return;
    s0 = b.s0;
    len = b.len;
    key0 = b.p0 + 32 * wave;
    pos0 = b.p0;
    list.tiles = (min(len, far_begin(a, pos0)) - pos0 + 31) / 32;
    const int see = (kKeys + a.w + 31) >> 5;   // tiles of a block inside the sequence
    list.start = (see - (pos0 >> 5) % see) % see;
    if (list.start >= list.tiles) list.start = 0;
    const int64_t all = static_cast<int64_t>(list.tiles) * a.g;
    const int split = in_group % a.splits;
    first = static_cast<int>(all * split / a.splits);
    total = static_cast<int>(all * (split + 1) / a.splits) - first;
  }
  list.pos0 = pos0;
  Steps qs(a, s0, len, h, list, first, wave, lane, tiles, rows);
  const LaneOffsets lo = lane_offsets<D>(lane, qs.stride);
  const int stages = (total + 1) >> 1;
  qs.issue(0, lo);

  const int j = key0 + (lane & 31);          // this lane's key
  const bool jok = j < len;
  const size_t krow = (static_cast<size_t>(s0 + (jok ? j : 0)) * a.H + h) * D;
  u32x4 kf[kKS], vf[kKS];
#pragma unroll
  for (int x = 0; x < kKS; ++x) {
    kf[x] = jok ? ld16(a.k + krow + 16 * x + 8 * hf) : u32x4{0u, 0u, 0u, 0u};
    vf[x] = jok ? ld16(a.v + krow + 16 * x + 8 * hf) : u32x4{0u, 0u, 0u, 0u};
  }
  f32x16 dka[kDB], dva[kDB];
#pragma unroll
  for (int x = 0; x < kDB; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) dka[x][i] = dva[x][i] = 0.f;
  StepList at = list;       // steps 2 st and 2 st + 1, one after the other
  at.seek(first);
  for (int st = 0; st < stages; ++st) {
    wait_copies();
    __syncthreads();
    if (st + 1 < stages) qs.issue((st & 1) ^ 1, lo);
#pragma unroll 1
    for (int sub = 0; sub < 2; ++sub) {
      const int tq = at.pos();
      const uint32_t t = tiles + (st & 1) * Steps::kBytes + 2 * kUnit * sub, r = rows + 1024 * (st & 1) + 512 * sub;
      const bool seen = tq + 31 >= key0 && (tq < key0 + 31 + a.w || key0 < a.sinks) && key0 < len && 2 * st + sub < total;
      if (seen && (!far || wave == ((2 * st + sub) & 3)))
        key_step<D>(a, lo, t, r, tq, key0, len, lane, kf, vf, dka, dva);
      at.skip(1);
    }
  }

  const int je = key0 + (fresh(lane) & 31);
  if (far) {
    // the waves took a step in four each: the four sums of a value meet in LDS, whose tiles nothing reads any more
    float* sum = reinterpret_cast<float*>(tile_lds);
    float* dst = far_sums(a, group, key0 >> 5, h, D);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      __syncthreads();
      store_sums<D>(sum + (32 * wave + je - key0) * D, x ? dva : dka, hf);
      __syncthreads();
      for (int i = 4 * threadIdx.x; i < 32 * D; i += 4 * kThreads) {
        f32x4 all = *reinterpret_cast<const f32x4*>(sum + i);
        for (int n = 1; n < kThreads / 64; ++n) all += *reinterpret_cast<const f32x4*>(sum + 32 * D * n + i);
        *reinterpret_cast<f32x4*>(dst + 32 * D * x + i) = all;
      }
    }
    return;
  }
  if (a.splits > 1) {   // others hold sums of these keys, too
    if (je < len) {
      float* dst = share_sums(a, in_group % a.splits, s0 + je, h, D);
      store_sums<D>(dst, dka, hf);
      store_sums<D>(dst + D, dva, hf);
    }
    return;
  }
  if (a.sink_tiles && key0 < a.sinks && far_begin(a, pos0) < len) {
    float* dst = near_sums(a, divide(s0, a.far, a.inv_far), key0 >> 5, h, D) + (je - key0) * D;
    store_sums<D>(dst, dka, hf);
    store_sums<D>(dst + 32 * D, dva, hf);
    return;
  }
  const bool jo = je < len;
  const size_t out = (static_cast<size_t>(s0 + (jo ? je : 0)) * a.H + h) * D;
  bool bad = store_row<D>(a.dk + out, dka, a.single ? 0.f : a.scale_log2 / kLog2e, hf, jo);
  bad |= store_row<D>(a.dv + out, dva, 1.0f, hf, jo);
  const uint64_t lanes = __builtin_amdgcn_ballot_w64(bad && jo);
  for (uint32_t cols = static_cast<uint32_t>(lanes | lanes >> 32); cols; cols &= cols - 1)
    exact_key<D>(a, s0, len, key0 + __builtin_ctz(cols), h);
}

// Keys whose sums lie with several workgroups, a wave each: the shares of their block in order, then, for a
// sink, the far queries in order of position.  Workgroup (x, head): keys 4 x .. of the packed tokens (splits > 1),
// or of the sinks of the sequence that starts in a `far` of them.
template <int D>
__global__ __launch_bounds__(kThreads) void window_sum_kernel(WindowArgs a) {
  constexpr int E = D / 64;
  const int h = blockIdx.y, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  Block blk;
  int j;                    // the wave's key
  if (a.splits > 1) {
    const int t = blockIdx.x * (kThreads / 64) + wave;
    if (t >= a.T) return;
    blk = block_of(a, t, 1, 0, 0);
    j = t - blk.s0;
  } else {
    const int per = 8 * a.sink_tiles;   // workgroups of a sequence's sinks
    blk = block_of(a, blockIdx.x / per, a.far, a.inv_far, 0);
    if (blk.p0 != 0) return;
    j = blockIdx.x % per * (kThreads / 64) + wave;
  }
  if (j < 0 || j >= blk.len) return;
  const int begin = far_begin(a, j & ~(kKeys - 1));
  const bool far = a.sink_tiles && (j & ~31) < a.sinks && begin < blk.len;   // the tile has far queries
  if (a.splits == 1 && !far) return;                                         // stored by its block
  float dk[E], dv[E];
#pragma unroll
  for (int e = 0; e < E; ++e) dk[e] = dv[e] = 0.f;
  auto add = [&](const float* p, int to_v) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      dk[e] += p[E * lane + e];
      dv[e] += p[to_v + E * lane + e];
    }
  };
  const int slot = divide(blk.s0, a.far, a.inv_far);
  if (a.splits == 1) add(near_sums(a, slot, j >> 5, h, D) + (j & 31) * D, 32 * D);
  else
#pragma unroll 4
    for (int sp = 0; sp < a.splits; ++sp) add(share_sums(a, sp, blk.s0 + j, h, D), D);
  if (far) {
    const int end = divide(blk.len - 1, a.far, a.inv_far) + 1;
#pragma unroll 4
    for (int c = divide(begin, a.far, a.inv_far); c < end; ++c) add(far_sums(a, slot + c, j >> 5, h, D) + (j & 31) * D, 32 * D);
  }
  bool bad = false;
  const size_t out = (static_cast<size_t>(blk.s0 + j) * a.H + h) * D + E * lane;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    bad |= not_finite(dk[e]) || not_finite(dv[e]);
    a.dk[out + e] = static_cast<__bf16>(a.single ? 0.f : dk[e] * a.scale_log2 / kLog2e);
    a.dv[out + e] = static_cast<__bf16>(dv[e]);
  }
  if (__builtin_amdgcn_ballot_w64(bad)) exact_key<D>(a, blk.s0, blk.len, j, h);
}

WindowArgs window_args(const dms_window_config& c, const int32_t* cu, const void* q, const void* k, const void* v) {
  WindowArgs a{};
  a.cu = cu;
  a.q = static_cast<const __bf16*>(q);
  a.k = static_cast<const __bf16*>(k);
  a.v = static_cast<const __bf16*>(v);
  a.n = c.num_seqs;
  a.T = c.total_tokens;
  a.H = c.num_kv_heads;
  a.g = c.group_size;
  a.w = std::min(c.window, std::max(1, c.max_seqlen));   // no query is further from a key
  a.sinks = std::min(c.sinks, c.max_seqlen);
  a.PB = kCols / a.g;
  a.inv_pb = inverse(a.PB);
  a.inv_g = 65536 / a.g + 1;
  a.single = a.w == 1 && (a.sinks == 0 || c.max_seqlen == 1);
  const float scale = c.softmax_scale > 0.f ? c.softmax_scale : 1.0f / sqrtf(static_cast<float>(c.head_dim));
  a.scale_log2 = scale * kLog2e;
  return a;
}

// Row values of the queries, then sums that workgroups leave to others: shares of key blocks' steps and far
// queries of sinks.
struct WindowLayout {
  size_t nlse, nsum, part, far_part, bytes;
  int64_t Ts;
  int far, sink_tiles, splits;
};
WindowLayout window_layout(const dms_window_config& c) {
  WindowLayout l{};
  const size_t T = c.total_tokens, H = c.num_kv_heads, D = c.head_dim;
  l.Ts = static_cast<int64_t>(T) + 128;
  const int64_t blocks = (static_cast<int64_t>(T) + kKeys - 1) / kKeys * c.num_kv_heads;
  // fewer blocks than CUs: shares of their steps, and shorter lists of far queries.  28 blocks (1777 tokens of 2
  // x 6 heads, w = 256, 16 sinks): forward and backward take 68 us, without shares 48 more, with far lists of 512
  // positions 49; 1024 blocks (16384 tokens of 8 x 5 heads, 4 sinks): 726 us, with far lists of 128 positions 82 more.
  l.splits = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kMaxSplits, kSplitTarget / std::max<int64_t>(1, blocks))));
  const int sinks = std::min(c.sinks, c.max_seqlen);
  // Far lists as long as the sinks (a fourth of them where blocks are few) at least: their sums, T / far lists for
  // each 32 sinks, then take no more than 32 D bytes of each token and KV head, and where all tokens are sinks
  // (full attention) there are none.  16384 tokens of 8 x 5 heads, w = 256, 4096 sinks: 0.3 GB of workspace, backward
  // 6.7 ms (lists of 512: 2.2 GB, 7.3 ms); all sinks: 5 MB, 13.0 ms (8.9 GB, 16.9 ms).
  const bool few = blocks < kSplitTarget;
  l.far = std::max(few ? kKeys : 4 * kKeys, static_cast<int>(align_up(few ? sinks / 4 : sinks, kKeys)));
  l.sink_tiles = c.max_seqlen > l.far ? (sinks + 31) / 32 : 0;
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, kAlign); return o; };
  l.nlse = take(H * c.group_size * l.Ts * 4);
  l.nsum = take(H * c.group_size * l.Ts * 4);
  l.part = take(l.splits > 1 ? l.splits * T * H * 2 * D * 4 : 0);
  l.far_part = take((l.splits > 1 ? 1 : 2) * (T / l.far + 1) * l.sink_tiles * H * 64 * D * 4);
  l.bytes = off;
  return l;
}

// Workgroups of a KV head in each launch.
struct WindowGrids {
  int64_t rows, keys, sums;   // query blocks; key blocks' shares and far queries; sums (0: no launch)
};
WindowGrids window_grids(const dms_window_config& c, const WindowLayout& l) {
  const int64_t T = c.total_tokens, n = c.num_seqs, per = l.far / kKeys;
  WindowGrids w{};
  w.rows = T / (kCols / c.group_size) + n;
  w.keys = (T / kKeys + n + per - 1) / per * (per * l.splits + l.sink_tiles);
  w.sums = l.splits > 1 ? (T + 3) / 4 : l.sink_tiles ? (T / l.far + 1) * 8 * l.sink_tiles : 0;
  return w;
}

template <int D>
void launch_backward(const WindowArgs& a, const WindowGrids& w, hipStream_t st) {
  auto grid = [&](int64_t x) { return dim3(static_cast<unsigned>(x), a.H); };
  hipLaunchKernelGGL(window_dq_kernel<D>, grid(w.rows), dim3(kThreads), 0, st, a);
  hipLaunchKernelGGL(window_dkv_kernel<D>, grid(w.keys), dim3(kThreads), 0, st, a);
  if (w.sums) hipLaunchKernelGGL(window_sum_kernel<D>, grid(w.sums), dim3(kThreads), 0, st, a);
}

}  // namespace

size_t window_workspace_bytes(const dms_window_config& c) { return window_layout(c).bytes; }

// A grid holds fewer than 2^32 threads.  Tokens times sinks have the limit that lists of 512 queries set.
bool window_grids_fit(const dms_window_config& c) {
  const WindowGrids w = window_grids(c, window_layout(c));
  const int64_t sinks = c.max_seqlen > 512 ? (static_cast<int64_t>(std::min(c.sinks, c.max_seqlen)) + 31) / 32 : 0;
  return std::max({w.rows, w.keys, w.sums, (c.total_tokens / 512 + int64_t(1)) * 8 * sinks}) < (int64_t(1) << 32) / kThreads;
}

hipError_t launch_window_fwd(const dms_window_config& c, const int32_t* cu, const void* q, const void* k,
                             const void* v, void* out, float* lse, void*, hipStream_t st) {
  WindowArgs a = window_args(c, cu, q, k, v);
  a.out = static_cast<__bf16*>(out);
  a.lse_out = lse;
  const dim3 grid(static_cast<unsigned>(window_grids(c, window_layout(c)).rows), a.H);
  if (c.head_dim == 64) hipLaunchKernelGGL(window_fwd_kernel<64>, grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(window_fwd_kernel<128>, grid, dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_window_bwd(const dms_window_config& c, const int32_t* cu, const void* q, const void* k,
                             const void* v, const float* lse, const void* dout, void* dq,
                             void* dk, void* dv, void* ws, hipStream_t st) {
  WindowArgs a = window_args(c, cu, q, k, v);
  const WindowLayout l = window_layout(c);
  char* w = static_cast<char*>(ws);
  a.nlse = reinterpret_cast<float*>(w + l.nlse);
  a.nsum = reinterpret_cast<float*>(w + l.nsum);
  a.part = reinterpret_cast<float*>(w + l.part);
  a.far_part = reinterpret_cast<float*>(w + l.far_part);
  a.Ts = l.Ts;
  a.far = l.far;
  a.inv_far = inverse(l.far);
  a.sink_tiles = l.sink_tiles;
  a.splits = l.splits;
  a.lse = lse;
  a.dout = static_cast<const __bf16*>(dout);
  a.dq = static_cast<__bf16*>(dq);
  a.dk = static_cast<__bf16*>(dk);
  a.dv = static_cast<__bf16*>(dv);
  const WindowGrids grids = window_grids(c, l);
  if (c.head_dim == 64) launch_backward<64>(a, grids, st);
  else launch_backward<128>(a, grids, st);
  return hipGetLastError();
}

}  // namespace dms
