// One token per row of logits, gfx950: temperature, top-k, top-p and min-p, and
// the token that a given uniform number picks.
//
// The weight of a token is an integer,
//   w = round(2^43 exp((x - max x) / T)),
// formed in float64: sums of a row are exact in 64 bits whatever their order
// (at most 2^20 tokens), so that borders and picks depend on neither the split of a
// row nor the order of atomics.  Tokens of weight 0 are never taken.
#include <math.h>

#include <algorithm>

#include "dms_common.h"
#include "dms_ops.h"

namespace dms {
namespace {

typedef unsigned long long u64;

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

__device__ inline u64 weight(float x, float top, double c) {
  const double e = exp2((static_cast<double>(x) - static_cast<double>(top)) * c);
  // 2^52 and more have no fraction bits: the sum is rounded to an integer, half to even
  const u64 b = static_cast<u64>(__double_as_longlong(fma(e, 0x1p43, 0x1p52)));
  return x == -INFINITY ? 0ull : b & ((1ull << 52) - 1);
}

// ---------------------------------------------------------------------------
// A row by one workgroup: right for every row.  The borders of top-k and top-p
// are found by their keys' digits (11, 11 and 10 bits), from the counts and
// weights of each digit's values.
// ---------------------------------------------------------------------------
constexpr int kRowThreads = 1024, kWaves = kRowThreads / 64, kBins = 2048;

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
    // thread t: the two bins 2047 - 2 t, 2046 - 2 t, in falling order
    const int b0 = kBins - 1 - 2 * tid;
    const uint32_t n0 = s.count[b0], n1 = s.count[b0 - 1];
    const u64 m0 = s.mass[b0], m1 = s.mass[b0 - 1];
    uint32_t n = n0 + n1;
    u64 m = m0 + m1;
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t un = __shfl_up(n, off, 64);
      const u64 um = __shfl_up(m, off, 64);
      if (lane >= off) n += un, m += um;
    }
    if (lane == 63) s.wave_count[wave] = n, s.wave_mass[wave] = m;
    __syncthreads();
    uint32_t en = n - n0 - n1 + above_count;
    u64 em = m - m0 - m1 + above_mass;
    for (int x = 0; x < wave; ++x) en += s.wave_count[x], em += s.wave_mass[x];
    // the first bin whose end reaches the border
    auto reached = [&](uint32_t cn, u64 cm) { return by_mass ? static_cast<double>(cm) >= least : cn >= want; };
    const bool r_before = reached(en, em) && en > 0;
    const bool r0 = reached(en + n0, em + m0) && en + n0 > 0, r1 = reached(en + n0 + n1, em + m0 + m1) && en + n0 + n1 > 0;
    if (!r_before && (r0 || r1)) {
      s.digit = r0 ? b0 : b0 - 1;
      s.above_count = r0 ? en : en + n0;
      s.above_mass = r0 ? em : em + m0;
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
__global__ __launch_bounds__(kRowThreads) void sample_row_kernel(SampleArgs a) {
  __shared__ RowLds s;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.vocab;
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

}  // namespace

size_t sample_workspace_bytes(const dms_sample_config& c, int rows) {
  return kAlign;
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
  if (c.logits_type == DMS_TYPE_BF16) hipLaunchKernelGGL(sample_row_kernel<true>, dim3(rows), dim3(kRowThreads), 0, st, a);
  else hipLaunchKernelGGL(sample_row_kernel<false>, dim3(rows), dim3(kRowThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace dms
