// The processing of logits between the LM head and the log-probability:
// penalties for repeated tokens, biases and grammar masks, and its gradient.
//
// Of a row with logits z, and the vocabulary entries v of its history:
//   x = z;  in the history: x = x > 0 ? x / repetition : x * repetition
//   x = x - frequency * (times in the response);  in the response: x = x - presence
//   x = x + bias (the last entry of the row's list that names v);  masked: x = -inf
// in fp32, rounded to bf16 once.
//
// A workgroup takes one stretch of kStretch entries of one row: it counts the
// history's tokens that fall into the stretch in LDS (whole numbers, so the order
// of the atomics does not show), then streams the stretch.  Nothing depends on the
// other rows, so a decode step's row and the update's row of the same prefix get
// the same bits.
#include "uattn_internal.h"
#include "uattn_rows.h"

namespace uattn {
namespace {

constexpr int kLogitsThreads = 256;
constexpr int kLogitsVecs = 4;
constexpr int kStretch = kLogitsThreads * kLogitsVecs * 8;
constexpr uint32_t kPrompt = 0x80000000u;  // of a count: the entry occurs in the prompt

struct LogitsParams {
  const uint16_t* in;        // logits, or the processed logits' gradient
  const uint16_t* logits;    // backward: the logits
  uint16_t* out;
  const int32_t* tokens;
  const int32_t* history;    // [rows][3]: begin, start of the response, end in tokens
  const float* penalties;    // [rows][3]: repetition, frequency, presence
  const int32_t* bias_ids;
  const float* bias_values;
  const int32_t* bias_rows;  // [rows][2]: begin, end in bias_ids
  const uint32_t* mask;      // [num_masks][mask_stride]
  const int32_t* mask_rows;  // [rows], or null: row t has mask t
  int64_t in_stride, logits_stride, out_stride, mask_stride;
  int32_t num_rows, vocab, num_tokens, num_bias, num_masks, stretches;
  int32_t first;  // workgroups of the launches before this one
};

__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return min(max(x, lo), hi); }

template <bool kGrad>
__global__ __launch_bounds__(kLogitsThreads) void logits_kernel(LogitsParams p) {
  __shared__ uint32_t table[kStretch];
  const int tid = threadIdx.x;
  const int64_t unit = p.first + static_cast<int64_t>(blockIdx.x);
  const int64_t row = unit / p.stretches;
  const int v0 = static_cast<int>(unit % p.stretches) * kStretch, n = min(kStretch, p.vocab - v0);
  const uint16_t* in = p.in + row * p.in_stride + v0;
  uint16_t* out = p.out + row * p.out_stride + v0;

  float rep = 1.f, freq = 0.f, pres = 0.f;
  int begin = 0, split = 0, end = 0;
  if (p.history != nullptr) {
    begin = clamp_int(p.history[3 * row], 0, p.num_tokens);
    end = clamp_int(p.history[3 * row + 2], begin, p.num_tokens);
    split = clamp_int(p.history[3 * row + 1], begin, end);
    rep = p.penalties[3 * row];
    freq = kGrad ? 0.f : p.penalties[3 * row + 1];
    pres = kGrad ? 0.f : p.penalties[3 * row + 2];
  }
  // the prompt matters to the repetition penalty alone
  if (rep == 1.f) begin = split;
  if (rep == 1.f && freq == 0.f && pres == 0.f) end = begin;
  int bias_begin = 0, bias_end = 0;
  if (!kGrad && p.bias_rows != nullptr) {
    bias_begin = clamp_int(p.bias_rows[2 * row], 0, p.num_bias);
    bias_end = clamp_int(p.bias_rows[2 * row + 1], bias_begin, p.num_bias);
  }
  const uint32_t* mask = nullptr;
  if (p.mask != nullptr) {
    const int64_t m = p.mask_rows != nullptr ? p.mask_rows[row] : row;
    if (m >= 0 && m < p.num_masks) mask = p.mask + m * p.mask_stride;
  }

  float x[kLogitsVecs][8];
#pragma unroll
  for (int i = 0; i < kLogitsVecs; ++i) {
    const int e0 = 8 * (tid + i * kLogitsThreads);
    u32x4 w = {0, 0, 0, 0};
    if (e0 + 8 <= n)
      w = load16(in, e0 / 8);
    else
      for (int e = 0; e < n - e0; ++e) w[e / 2] |= static_cast<uint32_t>(in[e0 + e]) << (16 * (e & 1));
    unpack8(w, x[i]);
  }
  auto clear = [&]() {
    for (int e = tid; e < kStretch; e += kLogitsThreads) table[e] = 0;
    __syncthreads();
  };
  if (begin < end) {
    clear();
    for (int i = begin + tid; i < end; i += kLogitsThreads) {
      const uint32_t v = static_cast<uint32_t>(p.tokens[i]) - v0;
      if (v < static_cast<uint32_t>(n)) {
        if (i < split)
          atomicOr(&table[v], kPrompt);
        else
          atomicAdd(&table[v], 1);
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLogitsVecs; ++i) {
      const int e0 = 8 * (tid + i * kLogitsThreads);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t seen = table[e0 + e];
        if (seen == 0) continue;
        if constexpr (kGrad) {
          const float z = bf16_lo(p.logits[row * p.logits_stride + v0 + e0 + e]);
          x[i][e] = z > 0.f ? x[i][e] / rep : x[i][e] * rep;
        } else {
          const uint32_t count = seen & ~kPrompt;
          float y = x[i][e] > 0.f ? x[i][e] / rep : x[i][e] * rep;
          if (count > 0) y = y - freq * static_cast<float>(count) - pres;
          x[i][e] = y;
        }
      }
    }
  }
  if (!kGrad && bias_begin < bias_end) {
    __syncthreads();
    clear();
    for (int i = bias_begin + tid; i < bias_end; i += kLogitsThreads) {
      const uint32_t v = static_cast<uint32_t>(p.bias_ids[i]) - v0;
      if (v < static_cast<uint32_t>(n)) atomicMax(&table[v], static_cast<uint32_t>(i - bias_begin) + 1);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kLogitsVecs; ++i) {
      const int e0 = 8 * (tid + i * kLogitsThreads);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t at = table[e0 + e];
        if (at != 0) x[i][e] = x[i][e] + p.bias_values[bias_begin + at - 1];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kLogitsVecs; ++i) {
    const int e0 = 8 * (tid + i * kLogitsThreads);
    if (e0 >= n) break;
    if (mask != nullptr) {
      const uint32_t keep = mask[(v0 + e0) / 32] >> ((v0 + e0) & 31);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (!(keep >> e & 1)) x[i][e] = kGrad ? 0.f : -__builtin_inff();
    }
    const u32x4 w = pack8(x[i]);
    if (e0 + 8 <= n)
      store16(out, e0 / 8, w);
    else
      for (int e = 0; e < n - e0; ++e) out[e0 + e] = static_cast<uint16_t>(w[e / 2] >> (16 * (e & 1)));
  }
}

hipError_t launch_logits(const LogitsLaunch& a, bool grad, hipStream_t stream) {
  LogitsParams p{};
  p.in = static_cast<const uint16_t*>(grad ? a.dout : a.logits);
  p.logits = static_cast<const uint16_t*>(a.logits);
  p.out = static_cast<uint16_t*>(a.out);
  p.tokens = a.tokens;
  p.history = a.history;
  p.penalties = a.penalties;
  p.bias_ids = a.bias_ids;
  p.bias_values = a.bias_values;
  p.bias_rows = a.bias_rows;
  p.mask = a.mask;
  p.mask_rows = a.mask_rows;
  p.in_stride = grad ? a.dout_stride : a.logits_stride;
  p.logits_stride = a.logits_stride;
  p.out_stride = a.out_stride;
  p.mask_stride = a.mask_stride;
  p.num_rows = a.num_rows;
  p.vocab = a.vocab;
  p.num_tokens = a.num_tokens;
  p.num_bias = a.num_bias;
  p.num_masks = a.num_masks;
  p.stretches = (a.vocab - 1) / kStretch + 1;
  return launch_parts(static_cast<int64_t>(a.num_rows) * p.stretches, kLogitsThreads, [&](int first, unsigned n) {
    p.first = first;
    if (grad)
      hipLaunchKernelGGL(logits_kernel<true>, dim3(n), dim3(kLogitsThreads), 0, stream, p);
    else
      hipLaunchKernelGGL(logits_kernel<false>, dim3(n), dim3(kLogitsThreads), 0, stream, p);
  });
}

}  // namespace

hipError_t launch_logits_process(const LogitsLaunch& a, hipStream_t stream) { return launch_logits(a, false, stream); }
hipError_t launch_logits_process_backward(const LogitsLaunch& a, hipStream_t stream) {
  return launch_logits(a, true, stream);
}

}  // namespace uattn
