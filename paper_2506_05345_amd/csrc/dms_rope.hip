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

// Both kernels rotate with the same operations, so that alignment changes no bits.
__device__ inline f32x2 rotate(float x1, float x2, f32x2 cs) {
  return f32x2{fmaf(x1, cs[0], -(x2 * cs[1])), fmaf(x1, cs[1], x2 * cs[0])};
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

// Any shape, stride and alignment: a thread per pair or copied element of a head, and the next kMaxBlocks blocks
// further on again (a grid holds fewer than 2^32 threads).
constexpr int kMaxBlocks = 65536;

template <typename TI, typename TO>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a) {
  const int units = a.rot / 2 + a.d - a.rot;
  const int row = (a.t.q ? a.Hq : 0) + (a.t.k ? a.H : 0);
  const int64_t total = static_cast<int64_t>(a.T) * row * units;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; i < total;
       i += static_cast<int64_t>(gridDim.x) * kThreads) {
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
      continue;
    }
    const int e1 = a.off + (a.adjacent ? 2 * u : u), e2 = e1 + (a.adjacent ? 1 : a.rot / 2);
    float x1 = load1(x + e1);
    const float x2 = load1(x + e2);
    if (first && e1 == 0 && !a.back) x1 = borrow_neuron(a, t, h / a.g, x1);
    f32x2 r = rotate(x1, x2, turn(a, t, u));
    if (first && e1 == 0 && a.back) r[0] = neuron_gradient(a, t, h / a.g);
    store1(y + e1, r[0]);
    store1(y + e2, r[1]);
  }
}

// ---------------------------------------------------------------------------
// Rows of whole 16-byte pieces.  A wave takes one token: its lanes form the
// token's angles once (a lane each), leave (cos, sin) in LDS and rotate the
// token's heads, 16 elements a lane at a time (8 of each half of the rotated
// part, or 16 that are copied).  The angles cost a wave about as much as two of
// its rounds of rotations, so that tokens of few heads are not split further.
// HBM-bound: 16384 tokens of 8 x 5 heads, d = 128, three axes, bf16 take 80 us
// (403 MB, 5.0 TB/s); their gradients from float32 116 us (605 MB, 5.2 TB/s).
// ---------------------------------------------------------------------------
struct Vec8 {
  float e[8];
};
struct RawF32 {
  f32x4 a, b;
};
__device__ inline RawF32 load8(const float* p) {
  return RawF32{*reinterpret_cast<const f32x4*>(p), *reinterpret_cast<const f32x4*>(p + 4)};
}
__device__ inline u32x4 load8(const __bf16* p) { return *reinterpret_cast<const u32x4*>(p); }
__device__ inline Vec8 widen(const RawF32& r) {
  return Vec8{{r.a[0], r.a[1], r.a[2], r.a[3], r.b[0], r.b[1], r.b[2], r.b[3]}};
}
__device__ inline Vec8 widen(const u32x4& u) {
  Vec8 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v.e[2 * i] = __uint_as_float(u[i] << 16);
    v.e[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
  return v;
}
__device__ inline void store8(float* p, const Vec8& v) {
  *reinterpret_cast<f32x4*>(p) = f32x4{v.e[0], v.e[1], v.e[2], v.e[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{v.e[4], v.e[5], v.e[6], v.e[7]};
}
__device__ inline void store8(__bf16* p, const Vec8& v) {
  u32x4 u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 pr = {v.e[2 * i], v.e[2 * i + 1]};
    u[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, bf16x2));
  }
  *reinterpret_cast<u32x4*>(p) = u;
}

constexpr int kRounds = 4;   // rounds of loads in flight

template <typename TI, typename TO, bool ADJACENT>
__global__ __launch_bounds__(kThreads) void rope_rows_kernel(RopeArgs a, int split, uint32_t per_head_inv) {
  __shared__ __attribute__((aligned(16))) f32x2 turns[kThreads / 64][kMaxRotary / 2];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t w = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + wave;
  const int t = static_cast<int>(w / split), part = static_cast<int>(w % split);
  if (t >= a.T) return;
  const int heads = (a.t.q ? a.Hq : 0) + (a.t.k ? a.H : 0);
  const int per_head = a.d / 16, rotated = a.rot / 16;
  const int rounds = (heads * per_head + 63) / 64;
  const int r0 = rounds * part / split, r1 = rounds * (part + 1) / split;
  const int units = heads * per_head;
  const TI* q = static_cast<const TI*>(a.t.q) + t * a.t.q_stride;
  const TI* k = static_cast<const TI*>(a.t.k) + t * a.t.k_stride;
  TO* qo = static_cast<TO*>(a.t.q_out) + t * a.t.q_out_stride;
  TO* ko = static_cast<TO*>(a.t.k_out) + t * a.t.k_out_stride;
  const int nq = a.t.q ? a.Hq : 0;

  struct Unit {
    int head, e1, e2, pair;   // pair < 0: copied
  };
  auto unit_of = [&](int u) {
    Unit x;
    x.head = __umulhi(u, per_head_inv);   // u / per_head: u * per_head < 2^32
    const int c = u - x.head * per_head;
    if (c < rotated) {
      x.e1 = a.off + 8 * c;
      x.e2 = x.e1 + a.rot / 2;
      x.pair = ADJACENT ? 4 * c : 8 * c;
    } else {
      const int e = 16 * (c - rotated);
      x.e1 = e >= a.off ? e + a.rot : e;
      x.e2 = x.e1 + 8;
      x.pair = -1;
    }
    return x;
  };
  bool ready = false;
  for (int r = r0; r < r1; r += kRounds) {
    decltype(load8(q)) x1[kRounds], x2[kRounds];
#pragma unroll
    for (int n = 0; n < kRounds; ++n) {
      const int u = 64 * (r + n) + lane;
      if (r + n < r1 && u < units) {
        const Unit x = unit_of(u);
        const TI* src = x.head < nq ? q + static_cast<size_t>(x.head) * a.d : k + static_cast<size_t>(x.head - nq) * a.d;
        x1[n] = load8(src + x.e1);
        x2[n] = load8(src + x.e2);
      }
    }
    if (!ready) {   // beside the first loads; a wave reads only what its own lanes wrote
      for (int i = lane; i < a.rot / 2; i += 64) turns[wave][i] = turn(a, t, i);
      __builtin_amdgcn_wave_barrier();
      ready = true;
    }
#pragma unroll
    for (int n = 0; n < kRounds; ++n) {
      const int u = 64 * (r + n) + lane;
      if (r + n < r1 && u < units) {
        const Unit x = unit_of(u);
        TO* dst = x.head < nq ? qo + static_cast<size_t>(x.head) * a.d : ko + static_cast<size_t>(x.head - nq) * a.d;
        const bool first = a.borrow && x.e1 == 0 && x.head < nq && x.head % a.g == 0;   // element 0 is the neuron
        Vec8 y1 = widen(x1[n]), y2 = widen(x2[n]);
        if (first && !a.back) y1.e[0] = borrow_neuron(a, t, x.head / a.g, y1.e[0]);
        if (x.pair >= 0) {
          if (ADJACENT) {
            const f32x2* c1 = &turns[wave][x.pair];
            const f32x2* c2 = c1 + a.rot / 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const f32x2 r1 = rotate(y1.e[2 * i], y1.e[2 * i + 1], c1[i]), r2 = rotate(y2.e[2 * i], y2.e[2 * i + 1], c2[i]);
              y1.e[2 * i] = r1[0];
              y1.e[2 * i + 1] = r1[1];
              y2.e[2 * i] = r2[0];
              y2.e[2 * i + 1] = r2[1];
            }
          } else {
            const f32x2* c = &turns[wave][x.pair];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const f32x2 r1 = rotate(y1.e[i], y2.e[i], c[i]);
              y1.e[i] = r1[0];
              y2.e[i] = r1[1];
            }
          }
        }
        if (first && a.back) y1.e[0] = neuron_gradient(a, t, x.head / a.g);
        store8(dst + x.e1, y1);
        store8(dst + x.e2, y2);
      }
    }
  }
}

template <typename TI, typename TO>
hipError_t run_rope(const RopeArgs& a, hipStream_t st) {
  const int heads = (a.t.q ? a.Hq : 0) + (a.t.k ? a.H : 0);
  auto whole = [](const void* p, int64_t stride, size_t size) {   // rows start on 16-byte pieces
    return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride * size % 16 == 0);
  };
  if (a.d >= 32 && a.d <= 4096 && a.d % 16 == 0 && a.rot % 16 == 0 && a.off % 16 == 0 && whole(a.t.q, a.t.q_stride, sizeof(TI)) &&
      whole(a.t.k, a.t.k_stride, sizeof(TI)) && whole(a.t.q_out, a.t.q_out_stride, sizeof(TO)) &&
      whole(a.t.k_out, a.t.k_out_stride, sizeof(TO))) {
    // tokens too few to fill the chip are split into rounds of their heads, at least one each: 32 tokens of 8 x 5
    // heads take 4.0 us instead of 7.9, 256 of them 5.0 instead of 8.3, 32 of 2 x 6 heads 4.2 instead of 4.9
    const int rounds = (heads * (a.d / 16) + 63) / 64;
    const int split = std::max(1, std::min(rounds, 1024 / a.T));
    const uint32_t inv = static_cast<uint32_t>((uint64_t(1) << 32) / (a.d / 16) + 1);
    const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(a.T) * split + kThreads / 64 - 1) / (kThreads / 64)));
    if (a.adjacent) hipLaunchKernelGGL((rope_rows_kernel<TI, TO, true>), grid, dim3(kThreads), 0, st, a, split, inv);
    else hipLaunchKernelGGL((rope_rows_kernel<TI, TO, false>), grid, dim3(kThreads), 0, st, a, split, inv);
    return hipGetLastError();
  }
  const int64_t units = static_cast<int64_t>(a.T) * heads * (a.d - a.rot / 2);
  const int64_t blocks = std::min<int64_t>(kMaxBlocks, (units + kThreads - 1) / kThreads);
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
