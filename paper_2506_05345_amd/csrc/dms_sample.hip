// One token per row of logits, gfx950: temperature, top-k, top-p and min-p, and
// the token that a given uniform number picks.
//
// The weight of a token is an integer,
//   w = round(2^43 exp((x - max x) / T)),
// formed in float64: sums of a row are exact in 64 bits whatever their order
// (at most 2^20 tokens), so that borders and picks depend on neither the split of a
// row nor the order of atomics.  Tokens of weight 0 are never taken.
//
// Rows of more than kSmallVocab logits are cut into parts, so that few rows fill the
// chip too, and take four launches:
//   sample_max_kernel   the largest values of the parts and of up to 2048 groups of a
//                       row's tokens (reads the logits from memory; the passes after
//                       it find them in the caches);
//   sample_hist_kernel  top-k of at most half the groups: the k-th largest of the
//                       groups' values, which k tokens reach.  Else the parts' weights,
//                       and each row's counts and weights by distance from its largest
//                       value (bins of 1/32 octave of weight); the row's last workgroup
//                       finds the bins that hold the borders of top-k and top-p;
//   sample_cut_kernel   lists the tokens that reach that value, or those of the borders'
//                       bins, with the weights ahead of them by part;
//   sample_pick_kernel  a workgroup a row sorts the listed tokens, cuts them, and finds
//                       the picked one: among them, if few are kept and all are
//                       listed, else in the part that holds it, by walking that.
// A row whose borders' bins hold too many tokens is done by the last launch alone, as
// shorter rows are (sample_row): equal logits, and flat rows with a few large ones, for
// bins are as fine as the range of a row allows.  Deviation 0.5 and eight logits 6 higher,
// T = 1, top-p 0.8: 151936 logits 390 us of that launch, 64 such rows 700; 262144 logits
// 660, 64 rows 1190.
//
// Kernel times on one MI355X in this order: 1 x 151936 float32, T = 0.6, top-p 0.95: 4.1 +
// 11.7 + 3.9 + 7.3 us, chains of dependent loads; 128 x 152064 of those: 14.3 (5.4 TB/s) +
// 37.3 + 15.0 + 11.0; 500 x 151936 bf16, every row its own settings: 29.0 (5.2 TB/s) + 55.8 +
// 39.5 + 19.0.  The second pass is bound by forming weights (18 float64 instructions a token;
// all vector instructions keep its units busy three quarters of the time), the third by the
// workgroups of rows that keep much of the vocabulary.  Before the groups, with counts for
// every top-k and the borders found by every workgroup of the third pass: 106, 81 and 69 us
// for the last three of the 500 rows.
#include <math.h>

#include <algorithm>

#include "dms_common.h"
#include "dms_draft.h"

namespace dms {
namespace {

typedef unsigned long long u64;

struct RowState;

struct SampleArgs {
  const void* logits;
  int64_t stride;
  const float* temperature;   // [rows], or null: the configuration's
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* u;
  int32_t* tokens;
  float* logprobs;            // or null
  int rows, vocab;
  float temperature0, top_p0, min_p0;
  int top_k0;
  RowState* state;            // [rows], rows in parts
  int parts;
};

// Settings of one row.
struct RowSetting {
  double t, c;       // temperature; log2(e) / temperature
  double p, least;   // top-p (1 and more: off), least weight that min-p keeps
  int k;             // top-k (vocab: off)
  float u;
};

__device__ inline RowSetting row_setting(const SampleArgs& a, int row) {
  RowSetting s;
  const float t = a.temperature ? a.temperature[row] : a.temperature0;
  const int k = a.top_k ? a.top_k[row] : a.top_k0;
  const float p = a.top_p ? a.top_p[row] : a.top_p0, m = a.min_p ? a.min_p[row] : a.min_p0;
  const bool greedy = !(t > 0.f);           // (NaN too)
  s.t = greedy ? 1.0 : static_cast<double>(t);
  s.c = 1.4426950408889634 / s.t;
  s.k = greedy ? 1 : k <= 0 ? a.vocab : min(k, a.vocab);
  s.p = p < 1.f ? static_cast<double>(p) : 1.0;
  s.least = (m > 0.f ? fmin(static_cast<double>(m), 1.0) : 0.0) * 0x1p43;
  const float u = a.u[row];
  s.u = u >= 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
  return s;
}

// A logit as it counts: NaN as -inf, +inf as the largest finite value, -0 as 0.
__device__ inline float counted(float x) {
  x = x != x ? -INFINITY : fminf(x, 0x1.fffffep127f);
  return x + 0.0f;
}
// The same but for NaN and -0, in two instructions of five: NaN has no weight and lies
// nowhere (comparisons are false), -0 weighs what 0 does.
__device__ inline float finite(float x) { return x == INFINITY ? 0x1.fffffep127f : x; }
// And with NaN such as fmaxf passes over: it answers a signalling one with NaN.
__device__ inline float quiet(float x) { return __builtin_canonicalizef(finite(x)); }
template <bool BF16>
__device__ inline float logit(const void* row, int i) {
  if constexpr (BF16)
    return counted(__uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(row)[i]) << 16));
  else
    return counted(static_cast<const float*>(row)[i]);
}
// Larger for larger values.
__device__ inline uint32_t order_key(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float key_value(uint32_t k) {
  return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k);
}
constexpr uint32_t kKeyNone = 0x007FFFFFu;   // -inf

// 2^43 2^((x - top) c), rounded.  2^f for |f| <= 1/2 is 1 + f P(f), P the polynomial of
// degree 9 that meets (2^f - 1) / f at the ten Chebyshev nodes of the range: 6.4e-16 off
// with its roundings, 0.006 of a unit.  No branches: several weights are formed side by side.
__device__ inline u64 weight(float x, float top, double c) {
  const double t = fmax((static_cast<double>(x) - static_cast<double>(top)) * c, -64.0);   // (NaN too: weight 0)
  // t + 1.5 2^52 has t's nearest integer in its low bits (a conversion and a rounding
  // instruction take four additions' time each)
  const double shifted = t + 0x1.8p52, f = t - (shifted - 0x1.8p52);
  constexpr double kTerms[10] = {7.070977866508138e-09,  1.0205905413765595e-07, 1.3215451633221434e-06,
                                 1.5252672924850737e-05, 0.00015403530424776529, 0.0013333558200794592,
                                 0.009618129107618665,   0.05550410866465167,    0.24022650695910075,
                                 0.6931471805599462};
  double p = kTerms[0];
#pragma unroll
  for (int i = 1; i < 10; ++i) {
    double term = kTerms[i];
    asm("" : "+s"(term));      // in scalar registers: an addend is no move of its own
    p = fma(p, f, term);
  }
  p = fma(p, f, 1.0);
  const double scale = __hiloint2double((1023 + 43 + __double2loint(shifted)) << 20, 0);
  // 2^52 and more have no fraction bits: the sum is rounded to an integer, half to even
  const u64 b = static_cast<u64>(__double_as_longlong(fma(p, scale, 0x1p52)));
  return b & ((1ull << 52) - 1);
}

// ---------------------------------------------------------------------------
// A row by one workgroup: right for every row.  The borders of top-k and top-p
// are found by their keys' digits (11, 11 and 10 bits), from the counts and
// weights of each digit's values.
// ---------------------------------------------------------------------------
// 512: two to three workgroups of the last launch fit a compute unit (of 1024, one: 500
// mixed rows 40 us against 25, one row 13.4 against 10.2).
constexpr int kRowThreads = 512, kWaves = kRowThreads / 64, kBins = 2048;

struct RowLds {
  u64 mass[kBins];
  uint32_t count[kBins];
  u64 wave_mass[kWaves];
  uint32_t wave_count[kWaves];
  u64 above_mass;
  uint32_t above_count, digit, key;
};

__device__ inline u64 wave_sum64(u64 v) {
  for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}
__device__ inline uint32_t wave_sum32(uint32_t v) {
  for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off, 64);
  return v;
}

// Border of a sorted prefix: values above `key`, and the first `ties` of those
// equal to it; mass: of the prefix.
struct Border {
  uint32_t key, ties;
  u64 mass;
};

// The shortest prefix of at least `want` tokens (by_mass: of at least `least`
// weight); the row has as many.
template <bool BF16>
__device__ Border find_border(const SampleArgs& a, const void* row, float top, double c, bool by_mass, uint32_t want,
                              double least, RowLds& s) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t prefix = 0, mask = 0, above_count = 0, in_bin = 0;
  u64 above_mass = 0;
  constexpr int kShift[3] = {21, 10, 0};
#pragma unroll
  for (int level = 0; level < 3; ++level) {
    for (int x = tid; x < kBins; x += kRowThreads) s.mass[x] = 0, s.count[x] = 0;
    if (tid == 0) s.digit = 0;
    __syncthreads();
    const uint32_t digits = level == 2 ? 1023u : 2047u;
    for (int i = tid; i < a.vocab; i += kRowThreads) {
      const float x = logit<BF16>(row, i);
      const uint32_t key = order_key(x);
      if ((key & mask) != prefix) continue;
      const u64 w = weight(x, top, c);
      if (w == 0) continue;
      atomicAdd(&s.mass[(key >> kShift[level]) & digits], w);
      atomicAdd(&s.count[(key >> kShift[level]) & digits], 1u);
    }
    __syncthreads();
    // thread t: bins 2047 - BINS t, .. in falling order
    constexpr int BINS = kBins / kRowThreads;
    const int b0 = kBins - 1 - BINS * tid;
    uint32_t nb[BINS], num = 0;
    u64 mb[BINS], sum = 0;
#pragma unroll
    for (int x = 0; x < BINS; ++x) num += nb[x] = s.count[b0 - x], sum += mb[x] = s.mass[b0 - x];
    uint32_t n = num;
    u64 m = sum;
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t un = __shfl_up(n, off, 64);
      const u64 um = __shfl_up(m, off, 64);
      if (lane >= off) n += un, m += um;
    }
    if (lane == 63) s.wave_count[wave] = n, s.wave_mass[wave] = m;
    __syncthreads();
    uint32_t en = n - num + above_count;
    u64 em = m - sum + above_mass;
    for (int x = 0; x < wave; ++x) en += s.wave_count[x], em += s.wave_mass[x];
    // the first bin whose end reaches the border
    auto reached = [&](uint32_t cn, u64 cm) { return cn > 0 && (by_mass ? static_cast<double>(cm) >= least : cn >= want); };
    bool before = reached(en, em);
#pragma unroll
    for (int x = 0; x < BINS; ++x) {
      const bool now = reached(en + nb[x], em + mb[x]);
      if (!before && now) {
        s.digit = b0 - x;
        s.above_count = en;
        s.above_mass = em;
      }
      before = now;
      en += nb[x];
      em += mb[x];
    }
    __syncthreads();
    prefix |= s.digit << kShift[level];
    mask |= digits << kShift[level];
    above_count = s.above_count;
    above_mass = s.above_mass;
    in_bin = s.count[s.digit];
    __syncthreads();
  }
  const u64 w = weight(key_value(prefix), top, c);
  uint32_t ties = want - above_count;
  if (by_mass) {
    const double miss = least - static_cast<double>(above_mass);
    ties = miss > 0.0 ? static_cast<uint32_t>(fmin(ceil(miss / static_cast<double>(w)), 2.0 * kSampleMaxVocab)) : 1u;
    ties = max(1u, min(ties, in_bin));
    while (ties > 1 && static_cast<double>(above_mass + (ties - 1) * w) >= least) --ties;
    while (ties < in_bin && static_cast<double>(above_mass + ties * w) < least) ++ties;
  }
  return Border{prefix, ties, above_mass + ties * w};
}

template <bool BF16>
__device__ void sample_row(const SampleArgs& a, int r, RowLds& s) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.vocab;
  const char* row = static_cast<const char*>(a.logits) + static_cast<int64_t>(r) * a.stride * (BF16 ? 2 : 4);
  const RowSetting set = row_setting(a, r);
  // ---- the largest value, and the weight of the row
  uint32_t key = 0;
  for (int i = tid; i < V; i += kRowThreads) key = max(key, order_key(logit<BF16>(row, i)));
  for (int off = 32; off; off >>= 1) key = max(key, static_cast<uint32_t>(__shfl_xor(static_cast<int>(key), off, 64)));
  if (lane == 0) s.wave_count[wave] = key;
  __syncthreads();
  for (int x = 0; x < kWaves; ++x) key = max(key, s.wave_count[x]);
  __syncthreads();
  if (key == kKeyNone) {      // no token is left
    if (tid == 0) {
      a.tokens[r] = -1;
      if (a.logprobs) a.logprobs[r] = NAN;
    }
    return;
  }
  const float top = key_value(key);
  u64 mass = 0;
  uint32_t count = 0;
  for (int i = tid; i < V; i += kRowThreads) {
    const u64 w = weight(logit<BF16>(row, i), top, set.c);
    mass += w;
    count += w != 0;
  }
  mass = wave_sum64(mass);
  count = wave_sum32(count);
  if (lane == 0) s.wave_mass[wave] = mass, s.wave_count[wave] = count;
  __syncthreads();
  mass = 0;
  count = 0;
  for (int x = 0; x < kWaves; ++x) mass += s.wave_mass[x], count += s.wave_count[x];
  __syncthreads();
  // ---- borders: the prefix that all of them keep is the shortest one
  Border b{0u, 0xFFFFFFFFu, mass};
  if (static_cast<uint32_t>(set.k) < count) b = find_border<BF16>(a, row, top, set.c, false, set.k, 0.0, s);
  if (set.p < 1.0) {
    const Border bp = find_border<BF16>(a, row, top, set.c, true, 0u, set.p * static_cast<double>(b.mass), s);
    if (bp.key > b.key || (bp.key == b.key && bp.ties < b.ties)) b = bp;
  }
  // ---- narrow the range that holds the picked token: kWaves contiguous parts at
  // a time, each a wave's, with the equal ones counted ahead of it
  auto kept = [&](float x, uint32_t& tie) -> u64 {     // weight, and whether it equals the border
    const uint32_t k = order_key(x);
    tie = k == b.key;
    if (k < b.key) return 0;
    const u64 w = weight(x, top, set.c);
    return static_cast<double>(w) >= set.least ? w : 0ull;
  };
  const u64 wb = weight(key_value(b.key), top, set.c);
  const u64 wt = b.key != 0 && static_cast<double>(wb) >= set.least ? wb : 0ull;   // weight of a kept equal one
  int lo = 0, hi = V;
  u64 before = 0, target = 0, total = 0;
  uint32_t ties_before = 0;
  bool first = true;
  while (first || hi - lo > 64) {
    const int part = ((hi - lo + kWaves - 1) / kWaves + 63) / 64 * 64;
    const int p0 = min(hi, lo + wave * part), p1 = min(hi, p0 + part);
    u64 m = 0;
    uint32_t n = 0;
    for (int i = p0 + lane; i < p1; i += 64) {
      uint32_t tie;
      const u64 w = kept(logit<BF16>(row, i), tie);
      n += tie;
      m += tie ? 0ull : w;
    }
    m = wave_sum64(m);
    n = wave_sum32(n);
    if (lane == 0) s.wave_mass[wave] = m, s.wave_count[wave] = n;
    __syncthreads();
    // equal ones up to the border's count weigh wt each
    auto tie_mass = [&](uint32_t from, uint32_t more) {
      const uint32_t x = min(from, b.ties), y = b.ties - x < more ? b.ties : x + more;
      return (y - x) * wt;
    };
    if (first) {
      uint32_t t = 0;
      for (int x = 0; x < kWaves; ++x) {
        total += s.wave_mass[x] + tie_mass(t, s.wave_count[x]);
        t += s.wave_count[x];
      }
      target = static_cast<u64>(static_cast<double>(set.u) * static_cast<double>(total));
    }
    u64 run = before;
    uint32_t t = ties_before;
    int at = kWaves - 1;
    for (int x = 0; x < kWaves; ++x) {
      const u64 more = s.wave_mass[x] + tie_mass(t, s.wave_count[x]);
      if (run + more > target) {
        at = x;
        break;
      }
      run += more;
      t += s.wave_count[x];
    }
    before = run;
    ties_before = t;
    const int l0 = lo;
    lo = min(hi, l0 + at * part);
    hi = min(hi, lo + part);
    first = false;
    __syncthreads();
  }
  if (wave == 0) {
    const int i = lo + lane;
    uint32_t tie = 0;
    float x = -INFINITY;
    u64 w = 0;
    if (i < hi) {
      x = logit<BF16>(row, i);
      w = kept(x, tie);
    }
    const u64 ties = __builtin_amdgcn_ballot_w64(tie != 0);
    if (tie && ties_before + __builtin_popcountll(ties & ((1ull << lane) - 1)) >= b.ties) w = 0;
    u64 run = w;
    for (int off = 1; off < 64; off <<= 1) {
      const u64 up = __shfl_up(run, off, 64);
      if (lane >= off) run += up;
    }
    const u64 hit = __builtin_amdgcn_ballot_w64(before + run > target);
    if (hit && lane == static_cast<int>(__builtin_ctzll(hit))) {
      a.tokens[r] = i;
      if (a.logprobs)
        a.logprobs[r] = static_cast<float>((static_cast<double>(x) - static_cast<double>(top)) / set.t -
                                           log(static_cast<double>(total) * 0x1p-43));
    }
  }
}

template <bool BF16>
__global__ __launch_bounds__(kRowThreads) void sample_row_kernel(SampleArgs a) {
  __shared__ RowLds s;
  sample_row<BF16>(a, blockIdx.x, s);
}

// ---------------------------------------------------------------------------
// A row in parts
// ---------------------------------------------------------------------------
constexpr int kPartThreads = 256, kPartWaves = kPartThreads / 64;
constexpr int kMaxParts = 256;                            // parts of a row, a wave each
// Bins: 32 an octave over 20 octaves, then 4 over 25.  A row with top-p and no top-k
// fills the weights of the first ones alone: a border past them is left to sample_row,
// and the rest of the row, most of it, needs no atomics (128 x 152064, T = 0.6: 35.6 us
// with them and 30.6 without, counts of the bins included in both).
constexpr int kFine = 20 * 32, kHist = kFine + 25 * 4;
constexpr int kListed = 2048;                             // tokens that a row lists at most
constexpr int kWaitVmcnt0 = 0x0F70;                       // s_waitcnt vmcnt(0): the wave's memory operations are done
constexpr int kFew = 256;     // kept tokens among which the picked one is found by sorting them by index
constexpr int kGroups = 2048;                             // groups whose largest values a row keeps at most

// What a row's second pass finds: its largest value and which bins hold its borders.
struct Cut {
  uint32_t key;        // of the largest value
  bool none, slow;     // nothing to cut by bins; the row is left to sample_row
  int from, to;        // bins whose tokens are listed; those before are kept
  float keep, end;     // distances at which they begin and end
  uint32_t ahead;      // tokens and weight before `from`
  u64 ahead_mass, all; // weight of the row
};

// What the launches of a row leave each other.
struct alignas(16) RowState {
  u64 mass[kHist];            // weights by bin
  u64 part_mass[kMaxParts], part_kept[kMaxParts];
  u64 list[kListed];          // key << 32 | ~index of the tokens in the borders' bins
  uint32_t count[kHist];
  uint32_t part_top[kMaxParts];
  float part_low[kMaxParts];      // smallest finite values (inf: none)
  uint32_t group_top[kGroups];
  uint32_t listed;
  uint32_t near;              // key that at least top-k tokens reach (Asked::near)
  uint32_t arrived;           // workgroups of the second pass that are done
  Cut cut;
};

// Groups of a part: a power of two, of the part's 256 pairs of a lane and a place in its
// fours.
__host__ __device__ inline int groups_of_part(int parts) {
  int n = 256;
  while (n * parts > kGroups) n >>= 1;
  return n;
}

// The parts of a row: 16-byte groups of logits in equal shares; what lies before the
// first aligned group belongs to the first part, what is left to the last.
template <bool BF16>
struct Parts {
  static constexpr int VEC = BF16 ? 8 : 4;
  const char* row;
  int V, S, lead, groups;
  __device__ Parts(const SampleArgs& a, int r) {
    row = static_cast<const char*>(a.logits) + static_cast<int64_t>(r) * a.stride * (BF16 ? 2 : 4);
    V = a.vocab;
    S = a.parts;
    lead = min(V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (BF16 ? 2 : 4));
    groups = (V - lead) / VEC;
  }
  __device__ int first_group(int s) const { return static_cast<int>(static_cast<int64_t>(s) * groups / S); }
  __device__ int begin(int s) const { return s == 0 ? 0 : lead + first_group(s) * VEC; }
  __device__ int end(int s) const { return s == S - 1 ? V : lead + first_group(s + 1) * VEC; }
  __device__ int holding(int i) const {
    if (i < lead) return 0;
    const int g = (i - lead) / VEC;
    return g >= groups ? S - 1 : static_cast<int>((static_cast<int64_t>(g + 1) * S - 1) / groups);
  }
  // f(first index, four logits as they are, how many of them are there) over part s, by one wave; four 16-byte
  // loads in flight
  // (the caller's lane takes part: its loads are left out otherwise)
  template <class F>
  __device__ void each(int s, F f, bool on = true) const {
    if (!on) return;
    const int lane = threadIdx.x & 63;
    auto edge = [&](int i0, int i1) {      // fewer than VEC tokens
      if (i0 + lane < i1) {
        const float x[4] = {logit<BF16>(row, i0 + lane), -INFINITY, -INFINITY, -INFINITY};
        f(i0 + lane, x, 1);
      }
    };
    if (s == 0) edge(0, lead);
    const int g1 = first_group(s + 1);
    const uint4* p = reinterpret_cast<const uint4*>(row + static_cast<size_t>(lead) * (BF16 ? 2 : 4));
    for (int g = first_group(s) + lane; g < g1; g += 4 * 64) {
      uint4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = p[min(g + u * 64, g1 - 1)];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (g + u * 64 >= g1) break;
        const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
        const int i = lead + (g + u * 64) * VEC;
#pragma unroll
        for (int h = 0; h < VEC / 4; ++h) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e)
            x[e] = __uint_as_float(!BF16 ? w[e] : e & 1 ? w[2 * h + (e >> 1)] & 0xFFFF0000u : w[2 * h + (e >> 1)] << 16);
          f(i + 4 * h, x, 4);
        }
      }
    }
    if (s == S - 1) edge(lead + groups * VEC, V);
  }
};

__device__ inline uint32_t wave_max32(uint32_t v) {
  for (int off = 32; off; off >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), off, 64)));
  return v;
}
// Row and part of a wave.
struct PartOf {
  int r, s;
  __device__ explicit PartOf(const SampleArgs& a) {
    const int per = a.parts / kPartWaves;
    r = blockIdx.x / per;
    s = __builtin_amdgcn_readfirstlane((blockIdx.x % per) * kPartWaves + (threadIdx.x >> 6));
  }
};

template <bool BF16>
__global__ __launch_bounds__(kPartThreads) void sample_max_kernel(SampleArgs a) {
  const PartOf me(a);
  RowState& st = a.state[me.r];
  const int lane = threadIdx.x & 63;
  for (int x = me.s * 64 + lane; x < kHist; x += a.parts * 64) st.mass[x] = 0, st.count[x] = 0;
  if (me.s == 0 && lane == 0) st.listed = 0, st.arrived = 0;
  // (in floats: NaN is neither, -inf is no smallest value; counted at the end)
  float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, least = INFINITY;
  Parts<BF16>(a, me.r).each(me.s, [&](int, const float (&x)[4], int) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      most[e] = x[e] > most[e] ? x[e] : most[e];     // (fmaxf of a signalling NaN is NaN)
      least = fminf(least, x[e] > -INFINITY ? x[e] : INFINITY);
    }
  });
  uint32_t key[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) key[e] = order_key(counted(most[e]));
  for (int off = 32; off; off >>= 1) least = fminf(least, __shfl_xor(least, off, 64));
  const int groups = groups_of_part(a.parts);
  uint32_t* group_top = st.group_top + me.s * groups;
  if (groups == 256) *reinterpret_cast<uint4*>(group_top + 4 * lane) = make_uint4(key[0], key[1], key[2], key[3]);
  key[0] = max(key[0], key[1]);
  key[2] = max(key[2], key[3]);
  if (groups == 128) *reinterpret_cast<uint2*>(group_top + 2 * lane) = make_uint2(key[0], key[2]);
  uint32_t top = max(key[0], key[2]);
  for (int off = 32, n = 64; off; off >>= 1, n >>= 1) {     // n groups: lanes alike in their low bits
    if (n == groups && lane < n) group_top[lane] = top;
    top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), off, 64)));
  }
  if (lane == 0) st.part_top[me.s] = top, st.part_low[me.s] = least;
}

// What the workgroup that finds a row's borders reads of its state, in one round of loads:
// the weight of its parts (every wave) and a few bins to a thread.  Other workgroups of the
// same launch wrote it: loads that no cache of this XCD answers.
template <class T>
__device__ inline T load_shared(const T* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
struct RowView {
  static constexpr int PER = (kHist + kPartThreads - 1) / kPartThreads;
  u64 all;
  u64 m[PER];
  uint32_t n[PER];
  __device__ RowView(const SampleArgs& a, const RowState& st) {
    constexpr int LANE = kMaxParts / 64;
    const int lane = threadIdx.x & 63;
    u64 part[LANE];
#pragma unroll
    for (int u = 0; u < LANE; ++u) part[u] = lane + 64 * u < a.parts ? load_shared(&st.part_mass[lane + 64 * u]) : 0;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int b = threadIdx.x * PER + u;
      m[u] = b < kHist ? load_shared(&st.mass[b]) : 0;
      n[u] = b < kHist ? load_shared(&st.count[b]) : 0;
    }
    all = part[0];
#pragma unroll
    for (int u = 1; u < LANE; ++u) all += part[u];
    all = wave_sum64(all);
  }
};
// Key of a row's largest logit, of its parts' (every wave).
__device__ inline uint32_t row_top(const SampleArgs& a, const RowState& st) {
  const int lane = threadIdx.x & 63;
  uint32_t key = kKeyNone;
#pragma unroll
  for (int u = 0; u < kMaxParts / 64; ++u) key = max(key, lane + 64 * u < a.parts ? st.part_top[lane + 64 * u] : kKeyNone);
  return wave_max32(key);
}
// Distance of a logit from the largest in octaves of weight, and its bin: larger for
// smaller logits (each step is monotonous), kHist where the weight is 0.
__device__ inline float octaves(float x, float top, float c) {
  const float half = 0.5f * top - 0.5f * x;      // (two large values of either sign: no overflow)
  return half == 0.f ? 0.f : half * (2.0f * c);
}
// Bins to an octave of a row: 32, or so many more, a power of two, that the fine bins hold
// all of a flat row (152064 logits of deviation 0.5 at T = 1.7, top-p 0.5: lists of 32 bins
// an octave overflow, 434 us; 49 with 128).  By the range of the row: a single large logit
// keeps them coarse.
__device__ inline float bins_an_octave(const SampleArgs& a, const RowState& st, uint32_t top, float c) {
  const int lane = threadIdx.x & 63;
  float low = INFINITY;
#pragma unroll
  for (int u = 0; u < kMaxParts / 64; ++u) low = fminf(low, lane + 64 * u < a.parts ? st.part_low[lane + 64 * u] : INFINITY);
  for (int off = 32; off; off >>= 1) low = fminf(low, __shfl_xor(low, off, 64));
  const float range = octaves(finite(low), key_value(top), c);
  float f = 32.f;
  while (f < 32.f * 1024.f && range * f < 0.49f * kFine) f *= 2.f;
  return f;
}
__device__ inline int bin_of(float z, float f) {
  return z * f < kFine ? static_cast<int>(z * f) : z < 45.f ? kFine + static_cast<int>((z - 20.f) * 4.f) : kHist;
}

// Distance at which bin b begins (exact: bins are powers of two wide).
__device__ inline float bin_edge(int b, float f) {
  return b < kFine || f > 32.f ? static_cast<float>(b) / f : 20.f + static_cast<float>(b - kFine) * 0.25f;
}

// The largest value of the logits that a lane of part s reads (in sample_max_kernel and in
// every pass after it), or of a few lanes.
__device__ inline float lane_top(const SampleArgs& a, const RowState& st, int s) {
  const int lane = threadIdx.x & 63, groups = groups_of_part(a.parts);
  const uint32_t* top = st.group_top + s * groups;
  uint32_t key;
  if (groups == 256) {
    const uint4 k = *reinterpret_cast<const uint4*>(top + 4 * lane);
    key = max(max(k.x, k.y), max(k.z, k.w));
  } else if (groups == 128) {
    const uint2 k = *reinterpret_cast<const uint2*>(top + 2 * lane);
    key = max(k.x, k.y);
  } else {
    key = top[lane & (groups - 1)];
  }
  return key_value(key);
}

// What a row asks of its passes: nothing but the groups (near: then every kept token is
// listed), weights of its bins (top-p), of its parts (no cut by rank or weight at all),
// counts (top-k).  Near: half the groups' values are reached by 1.4 tokens to a group
// where tokens are spread over the groups at random, so that the list holds them.
struct Asked {
  bool by_k, by_p, least, near;
  __device__ Asked(const SampleArgs& a, const RowSetting& s)
      : by_k(s.k < a.vocab), by_p(s.p < 1.0), least(s.least > 0.0), near(by_k && 2 * s.k <= a.parts * groups_of_part(a.parts)) {}
  __device__ bool weights() const { return !near && (by_p || !(by_k || least)); }
  __device__ bool bins() const { return !near && (by_k || by_p); }
  __device__ bool whole() const { return !(by_k || by_p || least); }
};

// A key that at least k of the groups' largest values reach: the k-th largest one's upper
// 16 bits (bf16 logits: all of it).  By the whole workgroup.
__device__ uint32_t near_key(const SampleArgs& a, const RowState& st, int k) {
  constexpr int PER = kGroups / kPartThreads;
  __shared__ int counts[16][kPartWaves];
  const int tid = threadIdx.x, n = a.parts * groups_of_part(a.parts);
  uint32_t keys[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) keys[u] = tid + u * kPartThreads < n ? st.group_top[tid + u * kPartThreads] : 0u;
  uint32_t found = 0;
#pragma unroll 1
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t at_least = found | 0x10000u << bit;
    int reached = 0;
#pragma unroll
    for (int u = 0; u < PER; ++u) reached += __builtin_popcountll(__builtin_amdgcn_ballot_w64(keys[u] >= at_least));
    if ((tid & 63) == 0) counts[bit][tid >> 6] = reached;
    __syncthreads();
    reached = 0;
#pragma unroll
    for (int x = 0; x < kPartWaves; ++x) reached += counts[bit][x];
    if (reached >= k) found = at_least;
  }
  return found;
}

struct CutLds {
  u64 wave_mass[kPartWaves];
  uint32_t wave_count[kPartWaves];
  int k_bin, p_low, p_high;
  u64 k_before, k_with;
  uint32_t ahead, through;
  u64 ahead_mass;
};
// Found by a whole workgroup, a few bins to a thread, for a row that asks for bins.
__device__ Cut find_cut(const RowView& v, const RowSetting& set, const Asked& ask, float f, CutLds& l) {
  constexpr int PER = RowView::PER;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  Cut cut{};
  cut.all = v.all;
  const u64 (&m)[PER] = v.m;
  const uint32_t (&n)[PER] = v.n;
  u64 sum = 0;
  uint32_t num = 0;
#pragma unroll
  for (int u = 0; u < PER; ++u) sum += m[u], num += n[u];
  u64 im = sum;
  uint32_t in = num;
  for (int off = 1; off < 64; off <<= 1) {
    const u64 um = __shfl_up(im, off, 64);
    const uint32_t un = __shfl_up(in, off, 64);
    if (lane >= off) im += um, in += un;
  }
  if (lane == 63) l.wave_mass[wave] = im, l.wave_count[wave] = in;
  if (tid == 0) l.k_bin = l.p_low = l.p_high = kHist;
  __syncthreads();
  u64 before = im - sum, in_bins = 0;
  uint32_t ahead = in - num, all_count = 0;
  for (int x = 0; x < kPartWaves; ++x) {
    if (x < wave) before += l.wave_mass[x], ahead += l.wave_count[x];
    in_bins += l.wave_mass[x];
    all_count += l.wave_count[x];
  }
  // top-k: the bin with the k-th token; fewer tokens than that have a weight: all of them
  const uint32_t k = static_cast<uint32_t>(set.k);
  const bool past = ask.by_p && in_bins != cut.all;     // tokens past the bins
  const bool by_k = ask.by_k && (k < all_count || past);
  if (by_k && k > all_count) {
    cut.slow = true;
    return cut;
  }
  if (!by_k && !ask.by_p) {
    cut.none = true;
    return cut;
  }
  {
    u64 x = before;
    uint32_t y = ahead;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      if (by_k && y < k && y + n[u] >= k) {
        l.k_bin = tid * PER + u;
        l.k_before = x;
        l.k_with = x + m[u];
      }
      x += m[u];
      y += n[u];
    }
  }
  __syncthreads();
  if (ask.by_p) {
    // what top-k leaves weighs between the bins before its border and those with it
    const double low = set.p * static_cast<double>(by_k ? l.k_before : cut.all);
    const double high = set.p * static_cast<double>(by_k ? l.k_with : cut.all);
    // (the largest logit's weight lies in the first bin)
    u64 x = before;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const bool was_low = x > 0 && static_cast<double>(x) >= low, was_high = x > 0 && static_cast<double>(x) >= high;
      x += m[u];
      if (!was_low && x > 0 && static_cast<double>(x) >= low) l.p_low = tid * PER + u;
      if (!was_high && x > 0 && static_cast<double>(x) >= high) l.p_high = tid * PER + u;
    }
    __syncthreads();
    if (l.p_high == kHist || l.p_low == kHist) {
      cut.slow = true;
      return cut;
    }
  }
  cut.from = ask.by_p ? l.p_low : l.k_bin;
  cut.to = by_k ? l.k_bin : l.p_high;
  {
    u64 x = before;
    uint32_t y = ahead;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const int b = tid * PER + u;
      if (b == cut.from) l.ahead = y, l.ahead_mass = x;
      x += m[u];
      y += n[u];
      if (b == cut.to) l.through = y;
    }
  }
  __syncthreads();
  cut.ahead = l.ahead;
  cut.ahead_mass = l.ahead_mass;
  // the tokens ahead weigh more than 2^43 2^-(where bin `from` begins) each: few of
  // them are listed too
  if (ask.by_p && static_cast<double>(cut.ahead_mass) * exp2f(bin_edge(cut.from, f) - 43.f) < 2.0 * kFew) {
    cut.from = 0;
    cut.ahead = 0;
    cut.ahead_mass = 0;
  }
  cut.keep = bin_edge(cut.from, f);
  cut.end = bin_edge(cut.to + 1, f);
  cut.slow = l.through - cut.ahead > kListed;      // (without top-k: known when they are listed)
  return cut;
}

template <bool BF16>
__global__ __launch_bounds__(kPartThreads) void sample_hist_kernel(SampleArgs a) {
  __shared__ u64 mass[kHist];
  __shared__ uint32_t count[kHist];
  __shared__ CutLds cut_lds;
  __shared__ int last;
  const PartOf me(a);
  const int tid = threadIdx.x, lane = tid & 63;
  RowState& st = a.state[me.r];
  const RowSetting set = row_setting(a, me.r);
  const Asked ask(a, set);
  const int groups = a.parts / kPartWaves;       // workgroups of the row
  const bool lead = blockIdx.x % groups == 0;
  if (!lead && !(ask.weights() || ask.bins())) return;
  const uint32_t key = row_top(a, st);
  if (lead && (!ask.bins() || key == kKeyNone)) {
    const uint32_t near = ask.near ? near_key(a, st, set.k) : 0u;
    if (tid == 0) {
      st.near = near;
      st.cut = Cut{key, true, false, 0, 0, 0.f, 0.f, 0u, 0, 0};
    }
  }
  if (key == kKeyNone || !(ask.weights() || ask.bins())) return;
  if (ask.bins()) {
    for (int x = tid; x < kHist; x += kPartThreads) mass[x] = 0, count[x] = 0;
    __syncthreads();
  }
  const float top = key_value(key), c = static_cast<float>(set.c), f = ask.bins() ? bins_an_octave(a, st, key, c) : 32.f;
  const Parts<BF16> parts(a, me.r);
  if (ask.weights()) {
    u64 sum = 0;
    const bool by_k = ask.by_k;
    const float most = by_k ? 45.f : 20.f;       // (a flat row ends before)
    parts.each(me.s, [&](int, const float (&given)[4], int) {
      const float x[4] = {finite(given[0]), finite(given[1]), finite(given[2]), finite(given[3])};
      u64 w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = weight(x[e], top, set.c);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += w[e];
      if (ask.by_p)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float z = octaves(x[e], top, c);
          if (z < most) {
            const int b = bin_of(z, f);
            atomicAdd(&mass[b], w[e]);
            if (by_k) atomicAdd(&count[b], 1u);
          }
        }
    });
    sum = wave_sum64(sum);
    if (lane == 0) __hip_atomic_store(&st.part_mass[me.s], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  } else {
    parts.each(me.s, [&](int, const float (&x)[4], int) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float z = octaves(finite(x[e]), top, c);
        if (z < 45.f) atomicAdd(&count[bin_of(z, f)], 1u);
      }
    });
  }
  if (ask.bins()) {
    __syncthreads();
    for (int x = tid; x < kHist; x += kPartThreads) {
      if (mass[x]) atomicAdd(&st.mass[x], mass[x]);
      if (count[x]) atomicAdd(&st.count[x], count[x]);
    }
    // the row's last workgroup finds the borders.  What the others leave it they write
    // and it reads by device-wide atomics, past the caches of the XCDs: every wave waits
    // until its own are done, then the workgroup arrives (fences of that scope, which write
    // back and drop those caches, took the pass of 128 rows from 31 us to 230)
    __builtin_amdgcn_s_waitcnt(kWaitVmcnt0);
    __syncthreads();
    if (tid == 0) last = atomicAdd(&st.arrived, 1u) == static_cast<uint32_t>(groups) - 1;
    __syncthreads();
    if (!last) return;
    Cut cut = find_cut(RowView(a, st), set, ask, f, cut_lds);
    cut.key = key;
    if (tid == 0) st.cut = cut;
  }
}

template <bool BF16>
__global__ __launch_bounds__(kPartThreads) void sample_cut_kernel(SampleArgs a) {
  const PartOf me(a);
  const int lane = threadIdx.x & 63;
  RowState& st = a.state[me.r];
  const RowSetting set = row_setting(a, me.r);
  const Asked ask(a, set);
  if (ask.whole()) return;
  const float mine = lane_top(a, st, me.s);     // lanes without a token to list or keep read none
  const Cut cut = st.cut;
  const uint32_t key = cut.key;
  if (key == kKeyNone || cut.slow) return;
  const float top = key_value(key), c = static_cast<float>(set.c);
  // tokens nearer than `keep` are ahead of the listed bins, those from `end` on are
  // out; no token past `far` passes min-p (and none past 45 octaves has a weight): a
  // weight of 128 units and more is rounded by 1/256 of it, 0.0057 octaves, at most;
  // smaller ones by up to all of it
  const float far = ask.least && set.least >= 128.0 ? 43.01f - log2f(static_cast<float>(set.least)) : 45.f;
  const float keep = cut.none ? 64.f : cut.keep, end = cut.none ? far : cut.end;
  auto list = [&](float x, int i) {
    const uint32_t at = atomicAdd(&st.listed, 1u);
    if (at < kListed) st.list[at] = static_cast<u64>(order_key(x + 0.0f)) << 32 | ~static_cast<uint32_t>(i);   // (-0 as 0)
  };
  if (ask.near) {
    const float least = key_value(max(st.near, kKeyNone));
    Parts<BF16>(a, me.r).each(me.s, [&](int i, const float (&given)[4], int n) {
      const float x[4] = {quiet(given[0]), quiet(given[1]), quiet(given[2]), quiet(given[3])};
      if (!(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) >= least)) return;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (x[e] >= least && octaves(x[e], top, c) < 45.f && e < n) list(x[e], i + e);
    }, mine >= least && octaves(mine, top, c) < 45.f);
    return;
  }
  u64 sum = 0;
  Parts<BF16>(a, me.r).each(me.s, [&](int i, const float (&given)[4], int n) {
    const float x[4] = {quiet(given[0]), quiet(given[1]), quiet(given[2]), quiet(given[3])};
    const float nearest = octaves(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), top, c);
    if (!(nearest < end)) return;      // four at once: nearly all of most rows
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float z = octaves(x[e], top, c);
      if (!(z < end) || (z < keep && !(z < far))) continue;
      const u64 w = weight(x[e], top, set.c);
      if (z < keep) {
        sum += static_cast<double>(w) >= set.least ? w : 0ull;
      } else if (w && e < n) {
        list(x[e], i + e);
      }
    }
  }, octaves(mine, top, c) < end);
  sum = wave_sum64(sum);
  if (lane == 0) st.part_kept[me.s] = sum;
}

struct PickLds {
  u64 list[2][kListed];
  u64 mass[kMaxParts];
  u64 wave_mass[kWaves];
  u64 total, k_mass, before;
  int last, part, k_last;
};

// Sorts the n different numbers of l.list[0], largest first, into it: waves sort chunks
// of 64 by counting those ahead of each, and a number's place is the sum of its places in
// all chunks, each found by halving.  l.list[1] holds the chunks in between.
__device__ void sort_listed(PickLds& l, int n) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, chunks = (n + 63) / 64;
  for (int c = wave; c < chunks; c += kWaves) {
    const u64* of = l.list[0] + 64 * c;
    const u64 mine = 64 * c + lane < n ? of[lane] : 0;
    const int there = min(64, n - 64 * c);
    int rank = 0;
#pragma unroll 8
    for (int x = 0; x < there; ++x) rank += of[x] > mine;
    l.list[1][64 * c + (lane < there ? rank : lane)] = mine;
  }
  __syncthreads();
  for (int x = tid; x < n; x += kRowThreads) {
    const u64 mine = l.list[1][x];
    int rank = x & 63;
#pragma unroll 4
    for (int c = 0; c < chunks; ++c) {
      const u64* of = l.list[1] + 64 * c;
      int p = 0;
#pragma unroll
      for (int step = 32; step; step >>= 1) p += of[p + step - 1] > mine ? step : 0;
      p += of[p] > mine;
      rank += c == x >> 6 ? 0 : p;
    }
    l.list[0][rank] = mine;
  }
  __syncthreads();
}

template <bool BF16>
__global__ __launch_bounds__(kRowThreads) void sample_pick_kernel(SampleArgs a) {
  __shared__ union {
    RowLds row;
    PickLds pick;
  } lds;
  PickLds& l = lds.pick;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const RowState& st = a.state[r];
  const RowSetting set = row_setting(a, r);
  const Asked ask(a, set);
  const Cut cut = st.cut;
  const u64 mine = tid < a.parts ? (ask.whole() ? st.part_mass[tid] : st.part_kept[tid]) : 0;
  const uint32_t listed = st.listed;
  const int n = min(listed, static_cast<uint32_t>(kListed));
  const uint32_t key = cut.key;
  if (key == kKeyNone) {      // no token is left
    if (tid == 0) {
      a.tokens[r] = -1;
      if (a.logprobs) a.logprobs[r] = NAN;
    }
    return;
  }
  if (cut.slow || listed > kListed) {
    __syncthreads();
    sample_row<BF16>(a, r, lds.row);
    return;
  }
  const float top = key_value(key);
  const Parts<BF16> parts(a, r);
  auto picked = [&](int i, u64 total) {
    a.tokens[r] = i;
    if (a.logprobs)
      a.logprobs[r] = static_cast<float>((static_cast<double>(logit<BF16>(parts.row, i)) - static_cast<double>(top)) / set.t -
                                         log(static_cast<double>(total) * 0x1p-43));
  };
  if (tid < kMaxParts) l.mass[tid] = ask.near ? 0 : mine;
  u64 border = 0;              // the last kept token of the listed ones, as the list holds it
  // (nothing listed: the k-th token is past all that have a weight, and those are ahead of
  // the border's bin)
  if (n > 0 && (ask.near || !cut.none)) {
    for (int x = tid; x < n; x += kRowThreads) l.list[0][x] = st.list[x];
    __syncthreads();
    sort_listed(l, n);
    const u64* list = l.list[0];
    // ---- running weights: thread t holds PER tokens from PER t on
    constexpr int PER = kListed / kRowThreads;
    const int x0 = PER * tid;
    u64 w[PER], sum = 0;
#pragma unroll
    for (int x = 0; x < PER; ++x) w[x] = x0 + x < n ? weight(key_value(static_cast<uint32_t>(list[x0 + x] >> 32)), top, set.c) : 0;
#pragma unroll
    for (int x = 0; x < PER; ++x) sum += w[x];
    u64 run = sum;
    for (int off = 1; off < 64; off <<= 1) {
      const u64 up = __shfl_up(run, off, 64);
      if (lane >= off) run += up;
    }
    if (lane == 63) l.wave_mass[wave] = run;
    if (tid == 0) l.last = n - 1, l.k_last = n - 1, l.k_mass = cut.all;
    __syncthreads();
    for (int x = 0; x < wave; ++x) run += l.wave_mass[x];
    run += cut.ahead_mass - sum;       // ahead of the thread's tokens
    // listed tokens that top-k keeps (near: those that are not listed have no weight)
    const int64_t left = ask.near ? min(set.k, n) : static_cast<int64_t>(set.k) - cut.ahead;
    if (left >= 1 && left <= n && (left - 1) / PER == tid) {
      u64 through = run;
#pragma unroll
      for (int x = 0; x < PER; ++x)
        if (x0 + x < left) through += w[x];
      l.k_last = static_cast<int>(left) - 1;
      l.k_mass = through;
    }
    __syncthreads();
    if (ask.by_p) {
      const double least = set.p * static_cast<double>(l.k_mass);
      // the first token at which the running weight is enough
      bool before = x0 > 0 && static_cast<double>(run) >= least;
      u64 through = run;
#pragma unroll
      for (int x = 0; x < PER; ++x) {
        through += w[x];
        if (!before && x0 + x < n && static_cast<double>(through) >= least) {
          atomicMin(&l.last, x0 + x);
          before = true;
        }
      }
      __syncthreads();
    }
    const int last = min(l.last, l.k_last);
    border = list[last];
    if (last < kFew && cut.from == 0) {      // every kept token is listed: by index
      __syncthreads();
      const bool mine = tid <= last;
      const u64 as_listed = mine ? list[tid] : 0;
      u64 wk = mine ? weight(key_value(static_cast<uint32_t>(as_listed >> 32)), top, set.c) : 0;
      if (!(static_cast<double>(wk) >= set.least)) wk = 0;
      __syncthreads();
      // 20 bits of index (falling), 44 of weight
      if (mine) l.list[0][tid] = static_cast<u64>(static_cast<uint32_t>(as_listed) & 0xFFFFFu) << 44 | wk;
      __syncthreads();
      sort_listed(l, last + 1);
      const u64 item = mine ? l.list[0][tid] : 0;
      wk = item & ((1ull << 44) - 1);
      u64 run = wk;
      for (int off = 1; off < 64; off <<= 1) {
        const u64 up = __shfl_up(run, off, 64);
        if (lane >= off) run += up;
      }
      if (lane == 63) l.wave_mass[wave] = run;
      __syncthreads();
      u64 total = 0;
      for (int x = 0; x < kFew / 64; ++x) {
        if (x < wave) run += l.wave_mass[x];
        total += l.wave_mass[x];
      }
      const u64 target = static_cast<u64>(static_cast<double>(set.u) * static_cast<double>(total));
      if (mine && run > target && run - wk <= target)      // one thread
        picked(static_cast<int>(~static_cast<uint32_t>(item >> 44) & 0xFFFFFu), total);
      return;
    }
    // ---- kept ones, to their parts
#pragma unroll
    for (int x = 0; x < PER; ++x)
      if (x0 + x <= last && static_cast<double>(w[x]) >= set.least)
        atomicAdd(&l.mass[parts.holding(static_cast<int>(~static_cast<uint32_t>(list[x0 + x])))], w[x]);
  }
  __syncthreads();
  // ---- the part that holds the picked token: lane t has parts 4 t .. 4 t + 3
  if (wave == 0) {
    u64 m[kMaxParts / 64], sum = 0;
#pragma unroll
    for (int u = 0; u < kMaxParts / 64; ++u) sum += m[u] = l.mass[lane * (kMaxParts / 64) + u];
    u64 run = sum;
    for (int off = 1; off < 64; off <<= 1) {
      const u64 up = __shfl_up(run, off, 64);
      if (lane >= off) run += up;
    }
    const u64 total = __shfl(run, 63, 64);
    const u64 target = static_cast<u64>(static_cast<double>(set.u) * static_cast<double>(total));
    u64 at = run - sum;
    if (run > target && at <= target) {     // one lane
#pragma unroll
      for (int u = 0; u < kMaxParts / 64; ++u) {
        if (at + m[u] > target) {
          l.part = lane * (kMaxParts / 64) + u;
          l.total = total;
          l.before = at;
          break;
        }
        at += m[u];
      }
    }
  }
  __syncthreads();
  // ---- its tokens by index, four to a thread at a time
  const u64 total = l.total, target = static_cast<u64>(static_cast<double>(set.u) * static_cast<double>(total));
  u64 before = l.before;
  const int end = parts.end(l.part);
  for (int i0 = parts.begin(l.part); i0 < end; i0 += 4 * kRowThreads) {
    u64 w[4], sum = 0;
    float x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = i0 + 4 * tid + u;
      x[u] = i < end ? logit<BF16>(parts.row, i) : -INFINITY;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const u64 as_listed = static_cast<u64>(order_key(x[u])) << 32 | ~static_cast<uint32_t>(i0 + 4 * tid + u);
      w[u] = weight(x[u], top, set.c);
      if (as_listed < border || !(static_cast<double>(w[u]) >= set.least)) w[u] = 0;
      sum += w[u];
    }
    u64 run = sum;
    for (int off = 1; off < 64; off <<= 1) {
      const u64 up = __shfl_up(run, off, 64);
      if (lane >= off) run += up;
    }
    __syncthreads();
    if (lane == 63) l.wave_mass[wave] = run;
    __syncthreads();
    u64 all = 0;
    run += before;
    for (int y = 0; y < kWaves; ++y) {
      if (y < wave) run += l.wave_mass[y];
      all += l.wave_mass[y];
    }
    if (run > target && run - sum <= target) {     // one thread
      u64 at = run - sum;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (at + w[u] > target) {
          picked(i0 + 4 * tid + u, total);
          break;
        }
        at += w[u];
      }
    }
    before += all;
    if (before > target) break;
  }
}

// Parts of a row, a wave each, four to a workgroup: workgroups of 16384 logits, so that
// rows that ask for little and rows that ask for much even out, more of them where all
// would be fewer than eight a compute unit, no part of fewer than 512 logits.  (All four
// passes of 500 mixed rows with workgroups of 37984, 16384 and 8192 logits: 160, 147 and 149
// us before the bins of flat rows; of 128 rows alike with 9504, 8448 and 4752: 76, 80 and 81.)
int row_parts(int rows, int vocab) {
  const int groups = std::max((2048 + rows - 1) / rows, vocab / 16384);
  return kPartWaves * std::max(1, std::min({kMaxParts / kPartWaves, groups, vocab / (512 * kPartWaves)}));
}

}  // namespace

// Up to here a row is one workgroup's: it takes fewer passes than there are launches.
constexpr int kSmallVocab = 4096;
// Rows of one round of launches (the workspace holds the state of so many).
constexpr int kRowsAtOnce = 1024;

size_t sample_workspace_bytes(const dms_sample_config& c, int rows) {
  return c.vocab <= kSmallVocab ? kAlign : align_up(sizeof(RowState) * std::max(1, std::min(rows, kRowsAtOnce)), kAlign);
}

template <bool BF16>
hipError_t launch_rows(SampleArgs a, hipStream_t st) {
  if (a.vocab <= kSmallVocab) {
    hipLaunchKernelGGL(sample_row_kernel<BF16>, dim3(a.rows), dim3(kRowThreads), 0, st, a);
    return hipGetLastError();
  }
  const int all = a.rows;
  for (int r = 0; r < all; r += kRowsAtOnce) {
    a.rows = std::min(kRowsAtOnce, all - r);
    a.parts = row_parts(a.rows, a.vocab);
    const dim3 grid(a.rows * (a.parts / kPartWaves)), threads(kPartThreads);
    hipLaunchKernelGGL(sample_max_kernel<BF16>, grid, threads, 0, st, a);
    hipLaunchKernelGGL(sample_hist_kernel<BF16>, grid, threads, 0, st, a);
    hipLaunchKernelGGL(sample_cut_kernel<BF16>, grid, threads, 0, st, a);
    hipLaunchKernelGGL(sample_pick_kernel<BF16>, dim3(a.rows), dim3(kRowThreads), 0, st, a);
    a.logits = static_cast<const char*>(a.logits) + static_cast<int64_t>(a.rows) * a.stride * (BF16 ? 2 : 4);
    auto on = [&](auto*& p) { if (p) p += a.rows; };
    on(a.temperature), on(a.top_k), on(a.top_p), on(a.min_p), on(a.u), on(a.tokens), on(a.logprobs);
  }
  return hipGetLastError();
}

hipError_t launch_sample(const dms_sample_config& c, int rows, const void* logits, int64_t stride, const float* temperature,
                         const int32_t* top_k, const float* top_p, const float* min_p, const float* u, int32_t* tokens,
                         float* logprobs, void* ws, hipStream_t st) {
  SampleArgs a{};
  a.logits = logits;
  a.stride = stride;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.u = u;
  a.tokens = tokens;
  a.logprobs = logprobs;
  a.rows = rows;
  a.vocab = c.vocab;
  a.temperature0 = c.temperature;
  a.top_k0 = c.top_k;
  a.top_p0 = c.top_p;
  a.min_p0 = c.min_p;
  a.state = static_cast<RowState*>(ws);
  return c.logits_type == DMS_TYPE_BF16 ? launch_rows<true>(a, st) : launch_rows<false>(a, st);
}

}  // namespace dms
