// The gradient of the token log-probability with respect to the logits:
//
//   dlogits[v] = dlogp * inv_temperature * (1[v = target] - p_v),  p = softmax(logits * inv_temperature)
//
// One workgroup per row.  With k = inv_temperature * log2(e) every thread keeps a
// running maximum m and the sum of exp2((x - m) k); the difference comes first, so
// that logits near the end of bf16's range (a row masked by its lowest value) do not
// overflow.  The target's own exponential is left out of the sum and added last, so
// that 1 - p of the target is the others' sum over the whole one: their difference
// from 1 would leave no digits where the target is nearly certain.  The order of the
// sum depends on the vocabulary alone.
#include <type_traits>

#include "uattn_internal.h"
#include "uattn_rows.h"

namespace uattn {
namespace {

struct LogprobGradParams {
  const uint16_t* logits;
  uint16_t* out;
  const int32_t* targets;
  const float* dlogp;
  int64_t stride, out_stride;
  int32_t vocab;
  bool stream;  // the output past the caches
  float it, k;  // inverse temperature, and times log2(e)
  int32_t first;  // rows of the launches before this one
};

__device__ __forceinline__ float neg_infinity() { return -__builtin_inff(); }
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// A maximum and the sum of exponentials relative to it.
struct MaxSum {
  float m, sum;
};
// What is subtracted from the logits: a maximum of -inf (nothing but masked entries) subtracts nothing.
__device__ __forceinline__ float shift_of(float m) { return m == neg_infinity() ? 0.f : m; }
// A sum relative to `from`, relative to `to` (to >= from).
__device__ __forceinline__ float rebase(float from, float to, float k) { return exp2_of((from - shift_of(to)) * k); }
__device__ __forceinline__ MaxSum combine(MaxSum a, MaxSum b, float k) {
  const float m = fmaxf(a.m, b.m);
  return MaxSum{m, a.sum * rebase(a.m, m, k) + b.sum * rebase(b.m, m, k)};
}

// Bound by memory.  The row stays in registers between its sum and its gradient (kVecs 16-byte pieces to
// a thread, all requested at once): it is read once and written once (4100 rows of 151,936: 490 us, 5.1 TB/s;
// read a second time from the caches it took 1755).  Pieces past kThreads * kVecs are read again.
template <int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads) void logprob_grad_kernel(LogprobGradParams p) {
  constexpr int kWaves = kThreads / 64;
  constexpr u32x4 kNegInf = {0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u};
  __shared__ MaxSum parts[kWaves];
  const int64_t row = p.first + static_cast<int64_t>(blockIdx.x);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint16_t* x = p.logits + row * p.stride;
  uint16_t* out = p.out + row * p.out_stride;
  const int y = p.targets[row], pieces = p.vocab / 8;
  const bool has_tail = tid < p.vocab % 8;  // an entry behind the pieces: the place `tail`
  const int tail = 8 * pieces + (tid & 7);
  const float dlogp = p.dlogp[row];
  if (dlogp == 0.f) {
    for (int v = tid; v < pieces; v += kThreads) store16(out, v, u32x4{0, 0, 0, 0});
    if (has_tail) out[tail] = 0;
    return;
  }
  const bool known = y >= 0 && y < p.vocab;
  const int y_piece = known && y < 8 * pieces ? y >> 3 : -1;

  u32x4 w[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int v0 = 64 * wave + i * kThreads;
    w[i] = kNegInf;
    if (v0 < pieces && v0 + lane < pieces) w[i] = load16(x, 0, v0 + lane);
  }
  MaxSum acc{neg_infinity(), 0.f};
  // adds kN pieces, which begin at v0 + j * kThreads
  auto add = [&](auto n_const, const u32x4* q, int v0) {
    constexpr int kN = decltype(n_const)::value;
    float m = neg_infinity();
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, fmaxf(bf16_lo(q[j][e]), bf16_hi(q[j][e])));
    m = fmaxf(acc.m, m);
    const float shift = shift_of(m);
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      float t[8];
      unpack8(q[j], t);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = exp2_of((t[e] - shift) * p.k);
      const int at = y_piece - (v0 + j * kThreads);
      if (at >= 0 && at < 64) {
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = lane == at && e == (y & 7) ? 0.f : t[e];
      }
      sum = sum + (((t[0] + t[1]) + (t[2] + t[3])) + ((t[4] + t[5]) + (t[6] + t[7])));
    }
    acc.sum = acc.sum * rebase(acc.m, m, p.k) + sum;
    acc.m = m;
  };
  constexpr int kStep = 4;
#pragma unroll
  for (int i = 0; i < kVecs; i += kStep) {
    const int v0 = 64 * wave + i * kThreads;
    if (v0 >= pieces) break;
    if constexpr (kVecs % kStep == 0) {
      add(std::integral_constant<int, kStep>{}, w + i, v0);
    } else {
      if (i + kStep <= kVecs)
        add(std::integral_constant<int, kStep>{}, w + i, v0);
      else
        add(std::integral_constant<int, kVecs % kStep>{}, w + i, v0);
    }
  }
  for (int v0 = 64 * wave + kVecs * kThreads; v0 < pieces; v0 += kThreads) {
    u32x4 q = kNegInf;
    if (v0 + lane < pieces) q = load16(x, 0, v0 + lane);
    add(std::integral_constant<int, 1>{}, &q, v0);
  }
  if (has_tail) {
    const float t = bf16_lo(x[tail]), m = fmaxf(acc.m, t);
    acc.sum = acc.sum * rebase(acc.m, m, p.k) + (tail == y ? 0.f : exp2_of((t - shift_of(m)) * p.k));
    acc.m = m;
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1)
    acc = combine(acc, MaxSum{__shfl_xor(acc.m, off, 64), __shfl_xor(acc.sum, off, 64)}, p.k);
  if constexpr (kWaves > 1) {
    if (lane == 0) parts[wave] = acc;
    __syncthreads();
    acc = parts[0];
#pragma unroll
    for (int u = 1; u < kWaves; ++u) acc = combine(acc, parts[u], p.k);
  }
  const float shift = shift_of(acc.m), g = dlogp * p.it;
  const float of_target = known ? exp2_of((bf16_lo(x[y]) - shift) * p.k) : 0.f;
  const float inv = known ? 1.f / (acc.sum + of_target) : __builtin_nanf("");
  const float scale = -g * inv, at_target = g * (acc.sum * inv);
  auto put = [&](const u32x4& q, int v0) {
    float t[8];
    unpack8(q, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = scale * exp2_of((t[e] - shift) * p.k);
    const int at = y_piece - v0;
    if (at >= 0 && at < 64) {
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] = lane == at && e == (y & 7) ? at_target : t[e];
    }
    if (v0 + lane < pieces) store16_as(p.stream, out, 0, v0 + lane, pack8(t));
  };
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int v0 = 64 * wave + i * kThreads;
    if (v0 >= pieces) break;
    put(w[i], v0);
  }
  for (int v0 = 64 * wave + kVecs * kThreads; v0 < pieces; v0 += kThreads) {
    u32x4 q = kNegInf;
    if (v0 + lane < pieces) q = load16(x, 0, v0 + lane);
    put(q, v0);
  }
  if (has_tail) {
    const float d = tail == y ? at_target : scale * exp2_of((bf16_lo(x[tail]) - shift) * p.k);
    out[tail] = static_cast<uint16_t>(bf16_pair(d, d));
  }
}

}  // namespace

hipError_t launch_logprob_backward(const LogprobBackwardLaunch& a, hipStream_t stream) {
  LogprobGradParams p{};
  p.logits = static_cast<const uint16_t*>(a.logits);
  p.out = static_cast<uint16_t*>(a.dlogits);
  p.targets = a.targets;
  p.dlogp = a.dlogp;
  p.stride = a.row_stride;
  p.out_stride = a.dlogits_stride;
  p.vocab = a.vocab;
  p.stream = streams(a.num_rows, a.vocab);
  p.it = a.inv_temperature;
  p.k = static_cast<float>(static_cast<double>(a.inv_temperature) * 1.4426950408889634);
  auto launch = [&](auto threads_const, auto vecs_const) {
    constexpr int kThreads = decltype(threads_const)::value, kVecs = decltype(vecs_const)::value;
    return launch_parts(a.num_rows, kThreads, [&](int first, unsigned n) {
      p.first = first;
      hipLaunchKernelGGL((logprob_grad_kernel<kThreads, kVecs>), dim3(n), dim3(kThreads), 0, stream, p);
    });
  };
  // Threads and pieces by the vocabulary alone (a row's bits do not depend on the number of rows): four to
  // twenty pieces in flight to a thread, and two rows or more to a CU up to 65,536 entries, so that one is
  // read while the other is written.  us for 600 and for 3000 rows: 32,000 entries 512 x 8 17.5 / 71, 256 x 16
  // 18.9 / 73.5; 50,257 512 x 16 28 / 116, 1024 x 8 35 / 136; 8000 128 x 8 8.6 / 17.6, 256 x 4 8.9 / 18.7.
  // Twenty pieces are what a thread's 128 registers hold (126 used; 21 spill), 163,840 entries of a row: one more
  // or less in registers costs little (4000 rows: 163,840 entries 508 us with 19, 504 with 20; 140,000 469 and 470).
  using std::integral_constant;
  if (a.vocab <= 2048) return launch(integral_constant<int, 64>{}, integral_constant<int, 4>{});
  if (a.vocab <= 8192) return launch(integral_constant<int, 128>{}, integral_constant<int, 8>{});
  if (a.vocab <= 32768) return launch(integral_constant<int, 512>{}, integral_constant<int, 8>{});
  if (a.vocab <= 65536) return launch(integral_constant<int, 512>{}, integral_constant<int, 16>{});
  if (a.vocab <= 131072) return launch(integral_constant<int, 1024>{}, integral_constant<int, 16>{});
  return launch(integral_constant<int, 1024>{}, integral_constant<int, 20>{});
}

}  // namespace uattn
