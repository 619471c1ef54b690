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

#include "dms_ops.h"

namespace dms {
namespace {

constexpr int kThreads = 256;
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

// A wave per query row; lanes over the head's elements.
template <int D>
__global__ __launch_bounds__(kThreads) void window_fwd_kernel(WindowArgs a) {
  constexpr int E = D / 64;
  const int Hq = a.H * a.g, lane = threadIdx.x & 63;
  const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + (threadIdx.x >> 6);
  if (row >= static_cast<int64_t>(a.T) * Hq) return;
  const int t = static_cast<int>(row / Hq), hq = static_cast<int>(row % Hq), h = hq / a.g;
  const int2 b = sequence_of(a, t);
  if (b.x > t) return;
  float q[E], o[E] = {}, m = -INFINITY, l = 0.f;
  for (int e = 0; e < E; ++e) q[e] = static_cast<float>(a.q[row * D + E * lane + e]);
  auto key = [&](int j) {
    const size_t kr = (static_cast<size_t>(j) * a.H + h) * D + E * lane;
    float s = 0.f;
    for (int e = 0; e < E; ++e) s += q[e] * static_cast<float>(a.k[kr + e]);
    s = wave_sum(s) * a.scale_log2;
    const float mn = fmaxf(m, s), c = exp2f(m - mn), p = exp2f(s - mn);
    l = l * c + p;
    for (int e = 0; e < E; ++e) o[e] = o[e] * c + p * static_cast<float>(a.v[kr + e]);
    m = mn;
  };
  const int band = max(b.x, t - a.w + 1);
  for (int j = b.x; j < min(band, b.x + a.sinks); ++j) key(j);
  for (int j = band; j <= t; ++j) key(j);
  for (int e = 0; e < E; ++e) a.out[row * D + E * lane + e] = static_cast<__bf16>(o[e] / l);
  if (lane == 0) a.lse_out[static_cast<size_t>(hq) * a.T + t] = (m + log2f(l)) * kLn2;
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
  const dim3 grid(row_blocks(static_cast<int64_t>(a.T) * a.H * a.g));
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
