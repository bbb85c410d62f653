// The gradient of the token log-probability with respect to the logits:
//
//   dlogits[v] = dlogp * inv_temperature * (1[v = target] - p_v),  p = softmax(logits * inv_temperature)
//
// One workgroup per row: the row's maximum and the sum of its exponentials (in an
// order fixed by the vocabulary), then the gradient.  The target's own exponential
// is left out of the sum and added last, so that 1 - p of the target is the
// others' sum over the whole one: their difference from 1 would leave no digits
// where the target is nearly certain.
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
  float it, k;  // inverse temperature, and times log2(e)
  int32_t first;
};

constexpr int kGradThreads = 1024;

__device__ __forceinline__ float logit(const uint16_t* x, int v) { return bf16_lo(x[v]); }

__global__ __launch_bounds__(kGradThreads) void logprob_grad_kernel(LogprobGradParams p) {
  constexpr int kWaves = kGradThreads / 64;
  __shared__ float slots[2][kWaves];
  const int64_t row = p.first + static_cast<int64_t>(blockIdx.x);
  const int tid = threadIdx.x;
  const uint16_t* x = p.logits + row * p.stride;
  uint16_t* out = p.out + row * p.out_stride;
  const int y = p.targets[row];
  const float g = p.dlogp[row] * p.it;
  float m = -__builtin_inff(), sum = 0.f;
  const bool skip = p.dlogp[row] == 0.f, known = y >= 0 && y < p.vocab;
  if (!skip) {
    for (int v = tid; v < p.vocab; v += kGradThreads) m = __builtin_elementwise_maximum(m, logit(x, v));
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) m = __builtin_elementwise_maximum(m, __shfl_xor(m, d, 64));
    if ((tid & 63) == 0) slots[0][tid >> 6] = m;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) m = __builtin_elementwise_maximum(m, slots[0][w]);
    for (int v = tid; v < p.vocab; v += kGradThreads)
      if (v != y) sum = sum + __builtin_amdgcn_exp2f((logit(x, v) - m) * p.k);
    sum = block_sum<kWaves>(sum, slots[1]);
  }
  const float at = !skip && known ? __builtin_amdgcn_exp2f((logit(x, y) - m) * p.k) : 0.f;
  const float inv = known ? 1.f / (sum + at) : __builtin_nanf("");
  for (int v = tid; v < p.vocab; v += kGradThreads) {
    float d = 0.f;
    if (!skip) {
      const float e = __builtin_amdgcn_exp2f((logit(x, v) - m) * p.k);
      d = v == y ? g * (sum * inv) : -g * (e * inv);
    }
    out[v] = static_cast<uint16_t>(bf16_pair(d, d));
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
  p.it = a.inv_temperature;
  p.k = static_cast<float>(static_cast<double>(a.inv_temperature) * 1.4426950408889634);
  return launch_parts(a.num_rows, kGradThreads, [&](int first, unsigned n) {
    p.first = first;
    hipLaunchKernelGGL(logprob_grad_kernel, dim3(n), dim3(kGradThreads), 0, stream, p);
  });
}

}  // namespace uattn
