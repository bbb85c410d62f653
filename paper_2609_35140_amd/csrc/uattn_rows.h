// Shared by the row-wise kernels: 16-byte pieces of bf16 rows, and sums over a
// wave or a workgroup in an order fixed by the thread count alone.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#pragma clang fp contract(off)

namespace uattn {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Two values rounded to bf16 (nearest even) by one instruction.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// Eight bf16 values of a 16-byte piece, and back.
__device__ __forceinline__ void unpack8(const u32x4& w, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    x[2 * j] = bf16_lo(w[j]);
    x[2 * j + 1] = bf16_hi(w[j]);
  }
}
__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] = bf16_pair(x[2 * j], x[2 * j + 1]);
  return w;
}

__device__ __forceinline__ u32x4 load16(const void* p, int64_t piece) {
  return reinterpret_cast<const u32x4*>(p)[piece];
}
__device__ __forceinline__ void store16(void* p, int64_t piece, const u32x4& w) {
  reinterpret_cast<u32x4*>(p)[piece] = w;
}

// The same behind a base that is the wave's: scalar address, 32-bit offset in the lanes.
__device__ __forceinline__ u32x4 load16(const void* base, int64_t uniform, uint32_t piece) {
  return *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(base) + 16 * uniform + 16u * piece);
}
__device__ __forceinline__ void store16(void* base, int64_t uniform, uint32_t piece, const u32x4& w) {
  *reinterpret_cast<u32x4*>(reinterpret_cast<char*>(base) + 16 * uniform + 16u * piece) = w;
}

// A read that passes the caches by, or not.
template <bool kOnce>
__device__ __forceinline__ u32x4 load16_as(const void* base, int64_t uniform, uint32_t piece) {
  const u32x4* from = reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(base) + 16 * uniform + 16u * piece);
  if constexpr (kOnce) return __builtin_nontemporal_load(from);
  return *from;
}
// Outputs past the caches or not.  (The empty asm keeps the two stores apart: merged, they would both be plain.)
__device__ __forceinline__ void store16_as(bool stream, void* base, int64_t uniform, uint32_t piece, const u32x4& w) {
  u32x4* to = reinterpret_cast<u32x4*>(reinterpret_cast<char*>(base) + 16 * uniform + 16u * piece);
  if (stream) {
    asm volatile("" ::: "memory");
    __builtin_nontemporal_store(w, to);
    asm volatile("" ::: "memory");
  } else {
    *to = w;
  }
}
// An output of bf16 rows is streamed from 64 MB on (residual norm, lookup, logits, the logits' two gradients): the caches
// would hand little of it to the operator that reads it next, and lose to it what they hold.  One border for all, where
// they begin to gain; just past it some readers still lose a few percent.  us, cached / streamed, alone and with what
// reads the output next:
//   residual norm    4000 x 4096 (33 MB) 22 / 24, 47 / 49; 8600 x 4096 (70 MB) 47 / 48, 96 / 96; 9815 x 4096 (80 MB)
//                    60 / 54, 120 / 108; 39,855 x 4096 225 / 214, 450 / 428
//   lookup, norm     8000 x 4096 (66 MB) 18.6 / 16.6, 40 / 40; 39,855 x 1024 (82 MB) 20 / 19, 47 / 47; 24,000 x 4096
//                    (197 MB) 54 / 49, 127 / 112
//   logits, log-prob 210 x 151,936 (64 MB) 27 / 26, 41 / 42; 300 (91 MB) 42 / 39, 66 / 69; 1000 (304 MB) 111 / 106,
//                    176 / 161
//   log-prob's gradient   222 x 151,936 (67 MB) 28 / 29; 600 (182 MB) 99 / 86; 1302 x 128,256 160 / 148
//   these four in a row, 151,936 entries: 222 rows 109 / 109, 250 (76 MB) 121 / 126, 300 170 / 168, 1000 466 / 423
inline bool streams(int64_t rows, int64_t width) { return 2 * rows * width >= int64_t{64} << 20; }

// DPP: every lane reads another of its 16; all lanes of the patterns used have a source.
template <int ctrl>
__device__ __forceinline__ float dpp_read(float x) {
  return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), ctrl, 0xF, 0xF, true));
}

// The sum over the wave's 64 lanes in every lane, the same bits in all of them: rotations inside 16
// lanes (after the distances 8 and 4 the sums repeat with period 4, so a swap is an xor), then the
// two lane swaps, whose operands come in the same order in both halves.
__device__ __forceinline__ float wave_sum(float x) {
  x = x + dpp_read<0x128>(x);  // row_ror:8
  x = x + dpp_read<0x124>(x);  // row_ror:4
  x = x + dpp_read<0x4E>(x);   // lane ^ 2
  x = x + dpp_read<0xB1>(x);   // lane ^ 1
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The sum over kWaves values (a power of two up to 16) that lanes l, l + kWaves, ... hold alike, in every lane.
template <int kWaves>
__device__ __forceinline__ float period_sum(float x) {
  if constexpr (kWaves > 8) x = x + dpp_read<0x128>(x);  // row_ror:8
  if constexpr (kWaves > 4) x = x + dpp_read<0x124>(x);  // row_ror:4
  if constexpr (kWaves > 2) x = x + dpp_read<0x4E>(x);   // lane ^ 2
  if constexpr (kWaves > 1) x = x + dpp_read<0xB1>(x);   // lane ^ 1
  return x;
}

// The sum over kWaves waves whose first is `wave0`, in every thread of theirs: wave sums through
// `slots` (one to a wave of the workgroup), every lane reading one of them.  All of the workgroup
// passes the barrier.  Calls in a row take different slots, so that a wave that is ahead does not
// overwrite what another still reads.
template <int kWaves>
__device__ __forceinline__ float waves_sum(float x, float* slots, int wave, int wave0) {
  x = wave_sum(x);
  if constexpr (kWaves == 1) return x;
  const int lane = threadIdx.x & 63;
  if (lane == 0) slots[wave] = x;
  __syncthreads();
  return period_sum<kWaves>(slots[wave0 + (lane & (kWaves - 1))]);
}

}  // namespace uattn
