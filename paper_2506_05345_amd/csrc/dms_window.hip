// Attention with a sliding window and sinks over packed sequences, gfx950.
//
// Key j is visible to query t iff j <= t and (j > t - w or j < sinks).
//   fwd: s = scale q.k, out = sum exp(s - m) v / l, lse = m + log l;
//   bwd: P = exp(s - lse), dP = dO V^T, D_t = dO.out, dS = P (dP - D),
//        dQ = scale dS K, dK = scale dS^T Q, dV = P^T dO.
// D_t is formed as sum_j P_j dP_j / sum_j P_j: from the rounded `out` it would be
// off by 2^-9 of |dO||out|, which dS = P (dP - D) of a row with few keys does not
// forgive (where one key takes nearly all the weight dP - D is nearly 0).
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
  float* row;              // [Hq][T] D_t (workspace)
  int n, T, H, g, w, sinks;
  int single;              // every row sees one key: P = 1 and dS = 0
  int PB;                  // positions of a query block: kCols / g
  float scale_log2;
};

// Bounds of sequence i inside the packed tensors, whatever cu holds.
__device__ inline int2 bounds_of(const WindowArgs& a, int i) {
  const int lo = min(max(a.cu[i], 0), a.T);
  return make_int2(lo, min(max(a.cu[i + 1], lo), a.T));
}

// Bounds of the sequence that owns packed token t (x > t: none).
__device__ inline int2 sequence_of(const WindowArgs& a, int t) {
  int lo = 0, hi = a.n;   // first i with cu[i + 1] > t
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a.cu[mid + 1] > t) hi = mid; else lo = mid + 1;
  }
  if (lo == a.n) return make_int2(t + 1, t + 1);
  const int2 b = bounds_of(a, lo);
  return b.x <= t && t < b.y ? b : make_int2(t + 1, t + 1);
}

__device__ inline float wave_sum(float x) {
#pragma unroll
  for (int off = 32; off; off >>= 1) x += __shfl_xor(x, off, 64);
  return x;
}

// Block b of a packed launch whose blocks hold PB tokens each: sequence i owns blocks
// cu[i] / PB + i .. cu[i + 1] / PB + i, at least as many as it needs, so that a block finds its sequence
// by a search over cu (64 candidates a round) and the host needs no prefix sums.
struct Block {
  int s0, len, p0;   // first token and length of the sequence, first position of the block (>= len: no block)
};
__device__ inline Block block_of(const WindowArgs& a, int b, int PB) {
  const int lane = threadIdx.x & 63;
  int lo = 0, cnt = a.n;
  while (cnt > 1) {
    const int step = (cnt + 63) >> 6;
    const int i = min(lo + lane * step, a.n);
    const bool le = lane * step < cnt && min(max(a.cu[i], 0), a.T) / PB + i <= b;
    const int k = max(1, __builtin_popcountll(__builtin_amdgcn_ballot_w64(le)));
    lo += (k - 1) * step;
    cnt = min(step, cnt - (k - 1) * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  const int2 r = bounds_of(a, lo);
  return Block{r.x, r.y - r.x, max(b - (r.x / PB + lo), 0) * PB};
}

// Keys that queries [p0, p1) of a sequence see, as tiles of 32: `nsk` tiles of sinks from position 0
// where a gap separates them from the window, then tiles from b0 on.
struct KeyTiles {
  int nsk, b0, nt;
  __device__ int first(int i) const { return i < nsk ? 32 * i : b0 + 32 * (i - nsk); }
};
__device__ inline KeyTiles key_tiles(const WindowArgs& a, int p0, int p1) {
  const int b0 = max(0, p0 - a.w + 1);
  KeyTiles t;
  t.nsk = a.sinks >= b0 ? 0 : (a.sinks + 31) >> 5;
  t.b0 = a.sinks >= b0 ? 0 : b0;
  t.nt = t.nsk + ((p1 - t.b0 + 31) >> 5);
  return t;
}

enum { kAll, kSome, kNone };
// What queries [q0, q1] (positions) see of tile i, whose first key is j0.
__device__ inline int mask_class(const WindowArgs& a, const KeyTiles& kt, int i, int j0, int q0, int q1) {
  if (i >= kt.nt || j0 > q1 || q0 > q1) return kNone;
  if (i < kt.nsk) return j0 + 32 <= a.sinks ? kAll : kSome;
  if (j0 + 31 <= q0 - a.w && j0 >= a.sinks) return kNone;
  return j0 + 31 <= q0 && (j0 > q1 - a.w || j0 + 32 <= a.sinks) ? kAll : kSome;
}
// Hides what position t does not see: register i of a lane is key j0 + 16 (i / 8) + 8 hf + i % 8.
__device__ inline void hide(f32x16& s, const WindowArgs& a, bool sink_tile, int j0, int t, int hf) {
  const int first = j0 + 8 * hf;
  const int hi = sink_tile ? a.sinks - 1 - first : t - first;   // last key seen
  const int lo = sink_tile ? -1 : t - a.w - first;              // last one before the window
  const int sn = a.sinks - first;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int k = 16 * (i >> 3) + (i & 7);
    s[i] = k <= hi && (k > lo || k < sn) ? s[i] : -INFINITY;
  }
}

__device__ inline float max3(float a, float b, float c) {   // scores of visible NaN keys are ignored here
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}
__device__ inline bool not_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }

// Row (position t of the sequence at s0, query head hq) by one wave, lanes over the head's elements and
// only visible keys read: rows whose sums are not finite, where a product may have met an Inf or NaN of
// a hidden key.
template <int D>
__device__ inline void exact_row(const WindowArgs& a, int s0, int t, int hq) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63, Hq = a.H * a.g, h = hq / a.g;
  const size_t row = (static_cast<size_t>(s0 + t) * Hq + hq) * D + E * lane;
  float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) q[e] = static_cast<float>(a.q[row + e]);
  const int band = max(0, t - a.w + 1);
  int j = a.sinks > 0 ? 0 : band;
#pragma unroll 1
  while (j <= t) {
    const size_t kr = (static_cast<size_t>(s0 + j) * a.H + h) * D + E * lane;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s += q[e] * static_cast<float>(a.k[kr + e]);
    s = wave_sum(s) * a.scale_log2;
    const float mn = fmaxf(m, s), c = exp2f(m - mn), p = exp2f(s - mn);
    l = l * c + p;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = o[e] * c + p * static_cast<float>(a.v[kr + e]);
    m = mn;
    j = j + 1 >= a.sinks ? max(j + 1, band) : j + 1;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) a.out[row + e] = static_cast<__bf16>(o[e] / l);
  if (lane == 0) a.lse_out[static_cast<size_t>(hq) * a.T + s0 + t] = (m + log2f(l)) * kLn2;
}

__device__ const u32x4 kZeros = {0u, 0u, 0u, 0u};

// Accumulators of one column (rows: dims 32 x + 8 y + 4 hf + 0 .. 3 in registers 4 y .. of block x),
// times f, to the row's bf16 elements: the two lanes of the column exchange halves and each writes 16 bytes.
template <int D>
__device__ inline void store_row(__bf16* dst, const f32x16* o, float f, int hf, bool ok) {
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
          r[z][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, bf16x2));
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
}

// ---------------------------------------------------------------------------
// Forward.  Workgroup = (KV head, block of PB positions of one sequence);
// columns are (position, query head) pairs, the g heads of a position
// consecutive, 32 per wave.  The block's key tiles go through LDS two at a
// time, the next two being copied while these are attended.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(kThreads, 2) void window_fwd_kernel(WindowArgs a) {
  using Tile = TileOf<D>;
  constexpr int kUnit = Tile::kUnit, kStage = 4 * kUnit, kKS = Tile::kKS, kDB = Tile::kDB;
  __shared__ __attribute__((aligned(256))) char tile_lds[2][kStage];   // [K tile | V tile] x 2
  const int2 wg = xcd_order();
  const int h = wg.y;
  const Block blk = block_of(a, wg.x, a.PB);
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
  auto issue = [&](int st, int buf) {   // a second tile past the last has zero rows
    const int i = 2 * st + (wave & 1);
    copy_tile<D>(kv, i < kt.nt ? kt.first(i) : p1, p1, stride, lo, lane,
                 tiles + buf * kStage + 2 * kUnit * (wave & 1) + kUnit * (wave >> 1), &kZeros);
  };
  issue(0, 0);

  const int col = wave * 32 + (lane & 31);
  const int pl = col / a.g, qh = col % a.g;
  const bool ok = pl < a.PB && p0 + pl < p1;
  const int t = ok ? p0 + pl : p0;
  const size_t row = static_cast<size_t>(s0 + t) * Hq + h * a.g + qh;
  u32x4 qf[kKS];
#pragma unroll
  for (int x = 0; x < kKS; ++x)
    qf[x] = ok ? ld16(a.q + row * D + 16 * x + 8 * hf) : u32x4{0u, 0u, 0u, 0u};
  // positions of this wave's columns
  const int q0 = p0 + wave * 32 / a.g, q1 = min(p1 - 1, p0 + (wave * 32 + 31) / a.g);
  const LaneAddresses<D> ad = lane_addresses<D>(tiles, lo);

  f32x16 o[kDB];
#pragma unroll
  for (int x = 0; x < kDB; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[x][i] = 0.f;
  float m_ref = kMInit, l_run = 0.f;
  const float thr = kRescale / a.scale_log2;

  const int steps = (kt.nt + 1) >> 1;
  auto attend = [&](int st, auto buf_c) {
    constexpr int buf = decltype(buf_c)::value;
    wait_copies();
    __syncthreads();
    if (st + 1 < steps) issue(st + 1, buf ^ 1);
    constexpr int tl = buf * kStage;
    const int j0 = kt.first(2 * st), j1 = kt.first(2 * st + 1);
    const int c0 = mask_class(a, kt, 2 * st, j0, q0, q1), c1 = mask_class(a, kt, 2 * st + 1, j1, q0, q1);
    if (c0 == kNone && c1 == kNone) return;
    f32x16 s[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[0][i] = s[1][i] = 0.f;
    u32x4 op[kAhead];
    // score product e: tile e % 2, k-step e / 2 (the two chains take turns)
#pragma unroll
    for (int e = 0; e < kAhead; ++e) op[e] = row_operand(tl + 2 * kUnit * (e & 1), ad, e >> 1);
#pragma unroll
    for (int e = 0; e < 2 * kKS; ++e) {
      __builtin_amdgcn_sched_barrier(0);
      s[e & 1] = mfma(op[e % kAhead], qf[e >> 1], s[e & 1]);
      if (e + kAhead < 2 * kKS) op[e % kAhead] = row_operand(tl + 2 * kUnit * (e & 1), ad, (e + kAhead) >> 1);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (c0 != kAll) hide(s[0], a, 2 * st < kt.nsk, j0, c0 == kNone ? j0 - 1 : t, hf);
    if (c1 != kAll) hide(s[1], a, 2 * st + 1 < kt.nsk, j1, c1 == kNone ? j1 - 1 : t, hf);
    float mx = max3(s[0][0], s[1][0], s[0][1]);
#pragma unroll
    for (int i = 1; i < 15; ++i) mx = max3(mx, s[1][i], s[0][i + 1]);
    mx = col_max(fmaxf(mx, s[1][15]));
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
    u32x4 pu[2][2];
    auto weight_pair = [&](int u, int j) {
      const f32x2 pr = {__builtin_amdgcn_exp2f(fmaf(s[u][2 * j], a.scale_log2, -mb)),
                        __builtin_amdgcn_exp2f(fmaf(s[u][2 * j + 1], a.scale_log2, -mb))};
      l_run += pr[0] + pr[1];
      pu[u][j >> 2][j & 3] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, bf16x2));
    };
#pragma unroll
    for (int j = 0; j < 8; ++j) weight_pair(0, j);
    // value product e: tile e / (2 kDB), token half (e / kDB) % 2, dim block e % kDB; the second
    // tile's weights are formed beside the first one's products
    auto read_v = [&](int e) {
      return col_operand(tl + 2 * kUnit * (e / (2 * kDB)) + kUnit, ad, e % kDB, (e / kDB) % 2);
    };
#pragma unroll
    for (int e = 0; e < kAhead; ++e) op[e] = read_v(e);
#pragma unroll
    for (int e = 0; e < 4 * kDB; ++e) {
      __builtin_amdgcn_sched_barrier(0);
      o[e % kDB] = mfma(op[e % kAhead], pu[e / (2 * kDB)][(e / kDB) % 2], o[e % kDB]);
      if (e + kAhead < 4 * kDB) op[e % kAhead] = read_v(e + kAhead);
      if (e < 2 * kDB)
#pragma unroll
        for (int j = 0; j < 4 / kDB; ++j) weight_pair(1, 4 / kDB * e + j);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  for (int st = 0; st < steps; st += 2) {
    attend(st, std::integral_constant<int, 0>{});
    if (st + 1 < steps) attend(st + 1, std::integral_constant<int, 1>{});
  }

  const float l = col_sum(l_run);
  const float inv = 1.0f / l;
  store_row<D>(a.out + row * D, o, inv, hf, ok);
  if (ok && hf == 0)
    a.lse_out[static_cast<size_t>(h * a.g + qh) * a.T + s0 + t] = (m_ref * a.scale_log2 + __log2f(l)) * kLn2;
  bool bad = not_finite(inv);
#pragma unroll
  for (int x = 0; x < kDB; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i) bad |= not_finite(o[x][i]);
  const uint64_t lanes = __builtin_amdgcn_ballot_w64(bad && ok);
  for (uint32_t cols = static_cast<uint32_t>(lanes | lanes >> 32); cols; cols &= cols - 1) {
    const int c = wave * 32 + __builtin_ctz(cols);
    exact_row<D>(a, s0, p0 + c / a.g, h * a.g + c % a.g);
  }
}

template <int D>
__global__ __launch_bounds__(kThreads) void window_dq_kernel(WindowArgs a) {
  constexpr int E = D / 64;
  const int Hq = a.H * a.g, lane = threadIdx.x & 63;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
  if (row >= static_cast<int64_t>(a.T) * Hq) return;
  const int t = static_cast<int>(row / Hq), hq = static_cast<int>(row % Hq), h = hq / a.g;
  const int2 b = sequence_of(a, t);
  if (b.x > t) return;
  float q[E], dO[E], dq[E] = {}, d = 0.f, sum = 0.f;
  for (int e = 0; e < E; ++e) {
    q[e] = static_cast<float>(a.q[row * D + E * lane + e]);
    dO[e] = static_cast<float>(a.dout[row * D + E * lane + e]);
  }
  const float lse2 = a.lse[static_cast<size_t>(hq) * a.T + t] * kLog2e;
  bool second = false;
  auto key = [&](int j) {
    const size_t kr = (static_cast<size_t>(j) * a.H + h) * D + E * lane;
    float s = 0.f, dp = 0.f;
    for (int e = 0; e < E; ++e) {
      s += q[e] * static_cast<float>(a.k[kr + e]);
      dp += dO[e] * static_cast<float>(a.v[kr + e]);
    }
    const float p = exp2f(wave_sum(s) * a.scale_log2 - lse2);
    dp = wave_sum(dp);
    if (second) {
      const float ds = p * (dp - d);
      for (int e = 0; e < E; ++e) dq[e] += ds * static_cast<float>(a.k[kr + e]);
    } else {
      d += p * dp;
      sum += p;
    }
  };
  const int band = max(b.x, t - a.w + 1);
  for (int pass = 0; pass < 2; ++pass) {
    for (int j = b.x; j < min(band, b.x + a.sinks); ++j) key(j);
    for (int j = band; j <= t; ++j) key(j);
    if (!second) d /= sum;
    second = true;
  }
  if (lane == 0) a.row[static_cast<size_t>(hq) * a.T + t] = d;
  for (int e = 0; e < E; ++e) a.dq[row * D + E * lane + e] = static_cast<__bf16>(a.single ? 0.f : dq[e] * a.scale_log2 / kLog2e);
}

// A wave per key; it walks the queries that see the key, every head of the group.
template <int D>
__global__ __launch_bounds__(kThreads) void window_dkv_kernel(WindowArgs a) {
  constexpr int E = D / 64;
  const int Hq = a.H * a.g, lane = threadIdx.x & 63;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
  if (row >= static_cast<int64_t>(a.T) * a.H) return;
  const int j = static_cast<int>(row / a.H), h = static_cast<int>(row % a.H);
  const int2 b = sequence_of(a, j);
  if (b.x > j) return;
  float k[E], v[E], dk[E] = {}, dv[E] = {};
  for (int e = 0; e < E; ++e) {
    k[e] = static_cast<float>(a.k[row * D + E * lane + e]);
    v[e] = static_cast<float>(a.v[row * D + E * lane + e]);
  }
  const int end = j - b.x < a.sinks ? b.y : static_cast<int>(min<int64_t>(b.y, static_cast<int64_t>(j) + a.w));
  for (int t = j; t < end; ++t)
    for (int hq = h * a.g; hq < (h + 1) * a.g; ++hq) {
      const size_t qr = (static_cast<size_t>(t) * Hq + hq) * D + E * lane;
      float s = 0.f, dp = 0.f;
      for (int e = 0; e < E; ++e) {
        const float dO = static_cast<float>(a.dout[qr + e]);
        s += k[e] * static_cast<float>(a.q[qr + e]);
        dp += v[e] * dO;
      }
      const float p = exp2f(wave_sum(s) * a.scale_log2 - a.lse[static_cast<size_t>(hq) * a.T + t] * kLog2e);
      const float ds = p * (wave_sum(dp) - a.row[static_cast<size_t>(hq) * a.T + t]);
      for (int e = 0; e < E; ++e) {
        dv[e] += p * static_cast<float>(a.dout[qr + e]);
        dk[e] += ds * static_cast<float>(a.q[qr + e]);
      }
    }
  for (int e = 0; e < E; ++e) {
    a.dk[row * D + E * lane + e] = static_cast<__bf16>(a.single ? 0.f : dk[e] * a.scale_log2 / kLog2e);
    a.dv[row * D + E * lane + e] = static_cast<__bf16>(dv[e]);
  }
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
  a.single = a.w == 1 && (a.sinks == 0 || c.max_seqlen == 1);
  const float scale = c.softmax_scale > 0.f ? c.softmax_scale : 1.0f / sqrtf(static_cast<float>(c.head_dim));
  a.scale_log2 = scale * kLog2e;
  return a;
}

unsigned row_blocks(int64_t rows) { return static_cast<unsigned>((rows + kThreads / 64 - 1) / (kThreads / 64)); }

}  // namespace

size_t window_workspace_bytes(const dms_window_config& c) {
  return align_up(static_cast<size_t>(c.total_tokens) * c.num_kv_heads * c.group_size * 4 + 4, kAlign);
}

hipError_t launch_window_fwd(const dms_window_config& c, const int32_t* cu, const void* q, const void* k,
                             const void* v, void* out, float* lse, void*, hipStream_t st) {
  WindowArgs a = window_args(c, cu, q, k, v);
  a.out = static_cast<__bf16*>(out);
  a.lse_out = lse;
  const dim3 grid(a.T / a.PB + a.n, a.H);
  if (c.head_dim == 64) hipLaunchKernelGGL(window_fwd_kernel<64>, grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL(window_fwd_kernel<128>, grid, dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_window_bwd(const dms_window_config& c, const int32_t* cu, const void* q, const void* k,
                             const void* v, const void*, const float* lse, const void* dout, void* dq,
                             void* dk, void* dv, void* ws, hipStream_t st) {
  WindowArgs a = window_args(c, cu, q, k, v);
  a.row = static_cast<float*>(ws);
  a.lse = lse;
  a.dout = static_cast<const __bf16*>(dout);
  a.dq = static_cast<__bf16*>(dq);
  a.dk = static_cast<__bf16*>(dk);
  a.dv = static_cast<__bf16*>(dv);
  const dim3 gq(row_blocks(static_cast<int64_t>(a.T) * a.H * a.g)), gk(row_blocks(static_cast<int64_t>(a.T) * a.H));
  if (c.head_dim == 64) {
    hipLaunchKernelGGL(window_dq_kernel<64>, gq, dim3(kThreads), 0, st, a);
    hipLaunchKernelGGL(window_dkv_kernel<64>, gk, dim3(kThreads), 0, st, a);
  } else {
    hipLaunchKernelGGL(window_dq_kernel<128>, gq, dim3(kThreads), 0, st, a);
    hipLaunchKernelGGL(window_dkv_kernel<128>, gk, dim3(kThreads), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace dms
