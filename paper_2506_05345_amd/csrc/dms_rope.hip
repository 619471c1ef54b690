// Rotary positions of queries and keys, gfx950.
//
// Pair i of a token turns by pos[axis(i)] * inv_freq[i]: y1 = x1 cos - x2 sin,
// y2 = x1 sin + x2 cos (the gradient turns back, sin -> -sin).  The angle is
// reduced to a fraction of a turn in float64, where a position of 2^31 still
// leaves 2^-22 of a turn's last bits; sine and cosine are float32.
#include <math.h>

#include <algorithm>

#include "dms_ops.h"

namespace dms {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kThreads = 256;

struct RopeArgs {
  RopeTensors t;
  const int32_t* pos;      // [axes][T]
  const double* inv;       // [rot / 2]
  float* logits;           // nullable, [T][H]
  uint8_t* decisions;      // nullable, [T][H]
  const float* dlogits;    // nullable, [T][H]
  int T, Hq, H, g, d, rot, off, axes;
  int sec[kRopeAxes];      // pairs of each axis (interleaved) or first pair of each axis (sections)
  int interleaved, adjacent, back, borrow;
  float factor, bias;
};

__device__ inline int axis_of(const RopeArgs& a, int i) {
  if (a.interleaved) {
    const int x = i % a.axes;
    return i / a.axes < a.sec[x] ? x : 0;
  }
  int x = 0;
#pragma unroll
  for (int k = 1; k < kRopeAxes; ++k) x = k < a.axes && i >= a.sec[k] ? k : x;
  return x;
}

// (cos, sin) of pair i of token t, times the factor; sin negated on the way back
__device__ inline f32x2 turn(const RopeArgs& a, int t, int i) {
  const int p = a.pos[static_cast<size_t>(axis_of(a, i)) * a.T + t];
  const double x = p * (a.inv[i] * 0.15915494309189533577);   // angle in turns
  const float fr = static_cast<float>(x - rint(x));
  float s, c;
  sincospif(2.0f * fr, &s, &c);
  return f32x2{c * a.factor, (a.back ? -s : s) * a.factor};
}

__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const __bf16* p) { return static_cast<float>(*p); }
__device__ inline void store1(float* p, float x) { *p = x; }
__device__ inline void store1(__bf16* p, float x) { *p = static_cast<__bf16>(x); }

// The borrowed neuron x of (token t, KV head h) is written out and becomes 0.
__device__ inline float borrow_neuron(const RopeArgs& a, int t, int h, float x) {
  const size_t at = static_cast<size_t>(t) * a.H + h;
  if (a.logits) a.logits[at] = x;
  if (a.decisions) a.decisions[at] = x + a.bias > 0.f;
  return 0.f;
}
__device__ inline float neuron_gradient(const RopeArgs& a, int t, int h) {
  return a.dlogits ? a.dlogits[static_cast<size_t>(t) * a.H + h] : 0.f;
}

// Any shape, stride and alignment: a thread per pair or copied element of a head.
template <typename TI, typename TO>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
  const int units = a.rot / 2 + a.d - a.rot;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  const int row = (a.t.q ? a.Hq : 0) + (a.t.k ? a.H : 0);
  if (i >= static_cast<int64_t>(a.T) * row * units) return;
  const int u = static_cast<int>(i % units);
  const int64_t th = i / units;
  const int t = static_cast<int>(th / row);
  int h = static_cast<int>(th % row);
  const bool isq = a.t.q && h < a.Hq;
  if (!isq && a.t.q) h -= a.Hq;
  const TI* x = static_cast<const TI*>(isq ? a.t.q : a.t.k) + t * (isq ? a.t.q_stride : a.t.k_stride) + static_cast<int64_t>(h) * a.d;
  TO* y = static_cast<TO*>(isq ? a.t.q_out : a.t.k_out) + t * (isq ? a.t.q_out_stride : a.t.k_out_stride) + static_cast<int64_t>(h) * a.d;
  const bool first = a.borrow && isq && h % a.g == 0;   // element 0 is the neuron
  if (u >= a.rot / 2) {
    int e = u - a.rot / 2;
    if (e >= a.off) e += a.rot;
    float v = load1(x + e);
    if (first && e == 0) v = a.back ? neuron_gradient(a, t, h / a.g) : borrow_neuron(a, t, h / a.g, v);
    store1(y + e, v);
    return;
  }
  const int e1 = a.off + (a.adjacent ? 2 * u : u), e2 = e1 + (a.adjacent ? 1 : a.rot / 2);
  float x1 = load1(x + e1);
  const float x2 = load1(x + e2);
  if (first && e1 == 0 && !a.back) x1 = borrow_neuron(a, t, h / a.g, x1);
  const f32x2 cs = turn(a, t, u);
  float y1 = x1 * cs[0] - x2 * cs[1];
  const float y2 = x1 * cs[1] + x2 * cs[0];
  if (first && e1 == 0 && a.back) y1 = neuron_gradient(a, t, h / a.g);
  store1(y + e1, y1);
  store1(y + e2, y2);
}

template <typename TI, typename TO>
hipError_t run_rope(const RopeArgs& a, hipStream_t st) {
  const int64_t units = static_cast<int64_t>(a.T) * ((a.t.q ? a.Hq : 0) + (a.t.k ? a.H : 0)) * (a.d - a.rot / 2);
  const int64_t blocks = (units + kThreads - 1) / kThreads;
  hipLaunchKernelGGL((rope_kernel<TI, TO>), dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const dms_rope_config& c, int tokens, const RopeTensors& t, const int32_t* positions,
                       const double* inv_freq, bool back, float* logits_out, uint8_t* decisions_out,
                       const float* dlogits, hipStream_t st) {
  RopeArgs a{};
  a.t = t;
  a.pos = positions;
  a.inv = inv_freq;
  a.logits = logits_out;
  a.decisions = decisions_out;
  a.dlogits = dlogits;
  a.T = tokens;
  a.H = c.num_kv_heads;
  a.g = c.group_size;
  a.Hq = a.H * a.g;
  a.d = c.head_dim;
  a.rot = c.rotary_dim;
  a.off = c.rotary_offset;
  a.axes = c.num_axes;
  a.interleaved = c.axis_order == DMS_ROPE_INTERLEAVED;
  for (int x = 0, sum = 0; x < kRopeAxes && x < c.num_axes; ++x) {
    a.sec[x] = a.interleaved ? c.sections[x] : sum;
    sum += c.sections[x];
  }
  a.adjacent = c.pairing == DMS_ROPE_ADJACENT;
  a.back = back;
  a.borrow = c.borrow;
  a.factor = c.factor > 0.f ? c.factor : 1.f;
  a.bias = c.decision_bias;
  if (c.in_type == DMS_TYPE_BF16)
    return c.out_type == DMS_TYPE_BF16 ? run_rope<__bf16, __bf16>(a, st) : run_rope<__bf16, float>(a, st);
  return c.out_type == DMS_TYPE_BF16 ? run_rope<float, __bf16>(a, st) : run_rope<float, float>(a, st);
}

}  // namespace dms
