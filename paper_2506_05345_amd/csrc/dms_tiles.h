// Tiles of 32 tokens in LDS as the 32x32x16 bf16 products of the training and
// windowed attention read them, and the small pieces those kernels share.
// gfx950 only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dms {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef short v4i16 __attribute__((ext_vector_type(4)));

#define DMS_LDS __attribute__((address_space(3)))

template <int D>
struct TileOf {
  static constexpr int kRowB = D * 2;       // bytes of one bf16 row
  static constexpr int kUnit = 32 * kRowB;  // one 32-token tile of one tensor
  static constexpr int kKS = D / 16;        // k-steps of a product over the head dimension
  static constexpr int kDB = D / 32;        // 32-dim blocks of a head
};

__device__ inline f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

__device__ inline u32x4 ld16(const void* p) { return *reinterpret_cast<const u32x4*>(p); }

// max / sum over the two lanes of one column (l and l + 32)
__device__ inline float col_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ inline float col_sum(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// The dispatcher deals workgroups to the 8 XCDs round-robin by linear id, and
// each XCD has its own L2.  Map the linear id so that the workgroups one XCD
// receives, in dispatch order, are a contiguous range of logical ids
// (x fastest): the blocks of one (sequence, head) then share an L2 and start
// together.
constexpr int kXcds = 8;
__device__ inline int2 xcd_order() {
  const int nx = gridDim.x;
  const int N = nx * gridDim.y;
  const int id = blockIdx.x + nx * blockIdx.y;
  const int x = id % kXcds, k = id / kXcds;
  const int L = x * (N / kXcds) + min(x, N % kXcds) + k;
  return int2{L % nx, L / nx};
}

// 8 fp32 values -> 4 packed bf16 pairs (round to nearest even)
__device__ inline u32x4 pack_bf16(const float* e) {
  u32x4 u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x2 pr = {e[2 * j], e[2 * j + 1]};
    u[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(pr, bf16x2));
  }
  return u;
}

// ---------------------------------------------------------------------------
// LDS tiles.  A 32-token tile of one head is staged row-major (2 D bytes a
// token, D = 64 or 128) straight from the [tokens, heads, D] input by global ->
// LDS copies, its 16-byte pieces permuted inside each row: piece dg of token t
// lies at t * 2 D + 16 (dg ^ x(t)), x(t) = 4 (t % 4) + (t / 4) % 4 for D = 128
// and 4 ((t / 2) % 2) + (t / 4) % 4 for D = 64, where two tokens share the 256
// bytes of a round over the banks.  Both operand reads then spread over all 64
// banks:
//   rows (a product over dims): lane l of k-step s takes dims 16 s + 8 (l / 32)
//     .. + 7 of token row_token(l % 32) with one 16-byte read;
//   columns (a product over tokens): lane l of (dim block b, half s) takes
//     tokens 16 s + 8 (l / 32) .. + 7 of dim 32 b + l % 32 with two LDS
//     transpose reads (ds_read_b64_tr_b16: in a 16-lane group, lane 4 j + q
//     passes the address of dims 4 q .. of token j and lane i receives dim i).
// Measured with eight waves reading: 4.0 cycles per wave read for both (256
// bytes a cycle for rows), 7.6 or more for the transpose reads of the
// unpermuted or t % 16-permuted rows.  Against tiles re-laid in memory by a
// pass of their own (row part and transposed part) this halves the staged
// bytes of the key-major pass and saves the pass.
// row_token orders the rows of a score MFMA so that accumulator registers
// 8 s .. 8 s + 7 of a lane are tokens 16 s + 8 (l / 32) .. + 7: exactly the B
// operand of half s of the next product.
// ---------------------------------------------------------------------------
__device__ inline int row_token(int r) {
  return 16 * (r >> 4) + 8 * ((r >> 2) & 1) + 4 * ((r >> 3) & 1) + (r & 3);
}

// Per-lane byte offsets; the others follow by an exclusive or (offsets of
// rows are multiples of 256, so it stays inside a row).
struct LaneOffsets {
  uint32_t row;   // row operand of k-step 0; k-step s: ^ 32 s
  uint32_t col;   // column operand of dim block 0, tokens 0-3 of the eight; block b: ^ 64 b,
                  // tokens 4-7: ^ 16, + 1024
  uint32_t src;   // source of copy 0; copy m: ^ copy_flip(m)
};

// Permutation of a row's 16-byte pieces.
template <int D>
__device__ constexpr int piece_flip(int t) {
  return D == 128 ? 4 * (t & 3) + ((t >> 2) & 3) : 4 * ((t >> 1) & 1) + ((t >> 2) & 3);
}
// The same for the rows of copy 0, t < 512 / D.
template <int D>
__device__ constexpr int row_flip(int t) {
  return D == 128 ? 4 * t : 4 * ((t >> 1) & 1) + (t >> 2);
}
// One copy instruction brings kCopyRows rows; its rows' flips differ from copy 0's by copy_flip(m) / 16.
template <int D>
constexpr int kCopyRows = 512 / D;
template <int D>
__device__ constexpr uint32_t copy_flip(int m) {
  return D == 128 ? 16 * (m & 3) : 32 * (m & 1);
}

template <int D>
__device__ inline LaneOffsets lane_offsets(int lane, uint32_t row_stride) {
  constexpr int kRowB = TileOf<D>::kRowB, kPieces = D / 8, kShift = D == 128 ? 4 : 3;
  LaneOffsets o;
  const int hf = lane >> 5;
  const int t = row_token(lane & 31);
  o.row = t * kRowB + 16 * (hf ^ piece_flip<D>(t));
  const int blk = (lane >> 4) & 1, j = (lane & 15) >> 2, q = lane & 3;
  o.col = (8 * hf + j) * kRowB + 16 * ((2 * blk + (q >> 1)) ^ (D == 128 ? 4 * j + 2 * hf : 4 * (j >> 1) + 2 * hf)) + 8 * (q & 1);
  const int tr = lane >> kShift, c = lane & (kPieces - 1);
  o.src = tr * row_stride + 16 * (c ^ row_flip<D>(tr));
  return o;
}

__device__ inline uint32_t lds_addr(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((DMS_LDS const char*)p));
}
// 64 lanes x 16 bytes (4 bytes) from base + off (per lane), or src (per lane), to LDS m0 + 16 (4) lane.  The LDS
// destination goes in M0, written by the same statement from a numbered scalar
// register (not from VCC, so that every M0 write looks alike); nothing else in
// this file reads M0.  The compiler does not count these loads: the kernels wait
// for them (vmcnt) before the barrier that publishes a stage.
__device__ inline void lds_copy16(const void* base, uint32_t off, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(m0), "v"(off), "s"(base) : "memory", "m0", "vcc");
}
__device__ inline void lds_copy16(const void* src, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(m0), "v"(src) : "memory", "m0", "vcc");
}
__device__ inline void lds_copy4(const void* base, uint32_t off, uint32_t m0) {
  asm volatile("s_mov_b32 m0, %0\n\tglobal_load_lds_dword %1, %2" : : "s"(m0), "v"(off), "s"(base) : "memory", "m0", "vcc");
}
__device__ inline void wait_copies() { __builtin_amdgcn_s_waitcnt(0x0F70); }   // vmcnt(0)
// All but the N newest copies (fewer than 64) have landed.
template <int N>
__device__ inline void wait_copies_but() {
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
}

// keeps the compiler from forming what follows from x ahead of a loop and holding it
__device__ inline int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// One wave copies rows t0 .. t0 + 31 of one head (row t at base + t * stride
// bytes) to the LDS tile `dst`, or every second of the copies (PARTS = 2: the
// copies m with m % 2 = part).  Rows from `end` on are copied from 16 zero
// bytes: their weights are 0, and 0 times an Inf or NaN of some token must not
// reach the sums.
template <int D, int PARTS = 1>
__device__ inline void copy_tile(const char* base, int t0, int end, uint32_t stride, const LaneOffsets& o,
                                 int lane, uint32_t dst, const void* zeros, int part = 0) {
  constexpr int kRows = kCopyRows<D>, kPieces = D / 8, kShift = D == 128 ? 4 : 3;
  if (t0 + 32 <= end) {
    const char* src = base + static_cast<size_t>(t0 + (PARTS > 1 ? kRows * part : 0)) * stride;
#pragma unroll
    for (int m = 0; m < 32 / kRows; m += PARTS)
      lds_copy16(src + static_cast<size_t>(kRows * m) * stride, o.src ^ (PARTS > 1 ? copy_flip<D>(m + part) : copy_flip<D>(m)),
                 dst + 1024 * (PARTS > 1 ? m + part : m));
  } else {
    const int ln = fresh(lane);   // formed here, not held ahead of the loop
    const int tr = ln >> kShift, c = ln & (kPieces - 1);
#pragma unroll
    for (int m0 = 0; m0 < 32 / kRows; m0 += PARTS) {
      const int m = PARTS > 1 ? m0 + part : m0;
      const int t = t0 + kRows * m + tr;
      const char* p = base + static_cast<size_t>(t) * stride + 16 * (c ^ (row_flip<D>(tr) + static_cast<int>(copy_flip<D>(m)) / 16));
      lds_copy16(t < end ? p : static_cast<const char*>(zeros), dst + 1024 * m);
    }
  }
}

// Operand reads of the LDS tile at byte address `t` (a multiple of 256).
template <int D>
__device__ inline u32x4 row_operand(uint32_t t, const LaneOffsets& o, int s) {
  return *reinterpret_cast<DMS_LDS const u32x4*>((t + o.row) ^ (32 * s));
}
__device__ inline u32x2 tr_read16(uint32_t p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<DMS_LDS v4i16*>(p)));
}
// column operand of dim block b, token half s
template <int D>
__device__ inline u32x4 col_operand(uint32_t t, const LaneOffsets& o, int b, int s) {
  const u32x2 lo = tr_read16(((t + o.col) ^ (64 * b)) + 16 * s * TileOf<D>::kRowB);
  const u32x2 hi = tr_read16(((t + o.col) ^ (64 * b) ^ 16) + 16 * s * TileOf<D>::kRowB + 4 * TileOf<D>::kRowB);
  return u32x4{lo[0], lo[1], hi[0], hi[1]};
}
// Every operand address of a lane in the tile at LDS byte address 0: passes
// with registers to spare hold them, so that a read is one instruction with
// the tile as its immediate offset (formed per read they were a sixth of the
// forward's VALU instructions).
template <int D>
struct LaneAddresses {
  uint32_t row[TileOf<D>::kKS], col[TileOf<D>::kDB][2];
};
template <int D>
__device__ inline LaneAddresses<D> lane_addresses(uint32_t t, const LaneOffsets& o) {
  LaneAddresses<D> r;
#pragma unroll
  for (int s = 0; s < TileOf<D>::kKS; ++s) r.row[s] = (t + o.row) ^ (32 * s);
#pragma unroll
  for (int b = 0; b < TileOf<D>::kDB; ++b) {
    r.col[b][0] = (t + o.col) ^ (64 * b);
    r.col[b][1] = ((t + o.col) ^ (64 * b) ^ 16) + 4 * TileOf<D>::kRowB;
  }
  return r;
}
template <int D>
__device__ inline u32x4 row_operand(int tile, const LaneAddresses<D>& r, int s) {
  return *reinterpret_cast<DMS_LDS const u32x4*>(r.row[s] + tile);
}
template <int D>
__device__ inline u32x4 col_operand(int tile, const LaneAddresses<D>& r, int b, int s) {
  const u32x2 lo = tr_read16(r.col[b][0] + tile + 16 * s * TileOf<D>::kRowB);
  const u32x2 hi = tr_read16(r.col[b][1] + tile + 16 * s * TileOf<D>::kRowB);
  return u32x4{lo[0], lo[1], hi[0], hi[1]};
}
// keeps the compiler from forming (and holding) every operand address ahead of the loop
__device__ inline void refresh(LaneOffsets& o) { asm volatile("" : "+v"(o.row), "+v"(o.col), "+v"(o.src)); }

// Scheduling order of a stretch of M MFMAs: P LDS reads ahead, then R reads
// beside each (bounds the operands in flight, so that the accumulators and the
// resident operands fit without spills).
template <int P, int M, int R>
__device__ __forceinline__ void paced() {
  __builtin_amdgcn_sched_group_barrier(0x100, P, 0);
#pragma unroll
  for (int i = 0; i < M; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
  }
}

}  // namespace dms
