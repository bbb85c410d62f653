// The processing of logits between the LM head and the log-probability:
// penalties for repeated tokens, biases and grammar masks, and its gradient.
//
// Of a row with logits z, and the vocabulary entries v of its history:
//   x = z;  in the history: x = x > 0 ? x / repetition : x * repetition
//   x = x - frequency * (times in the response);  in the response: x = x - presence
//   x = x + bias (the last entry of the row's list that names v);  masked: x = -inf
// in fp32 (the division as a product with 1 / repetition), rounded to bf16 once.
//
// A workgroup takes one stretch of up to 8192 entries (the vocabulary in equal parts,
// sixteen entries to a thread) of some consecutive rows.  It counts the history's
// tokens that fall into the stretch in LDS (whole numbers, so the order of the
// atomics does not show) and streams the stretch.  Rows of an update are
// successive prefixes of a sequence: where a row's history is the one before it and
// some more, only the new tokens are counted, and most of them fall into other
// stretches.  Counts do not depend on how they came about, so a decode step's row and
// the update's row of the same prefix get the same bits.
#include <type_traits>

#include "uattn_internal.h"
#include "uattn_rows.h"

namespace uattn {
namespace {

constexpr int kLogitsThreads = 512;  // at most
constexpr int kLogitsVecs = 2;
constexpr int kThreadEntries = 8 * kLogitsVecs;
constexpr int kMostEntries = kLogitsThreads * kThreadEntries;  // of a stretch
// Rows to a workgroup where there are many: few, as the rows in flight then lie close together (8000 rows of
// 151,936 with 2000 tokens of history: 820 us with 3, 910 with 5, 990 with 16).  Where three rows share a history
// that is long to count (so many tokens to a thread, or more), kParts times as many by the first of as many
// workgroups (3200 rows with 31,000 tokens: 498 us with 3 rows, 408 so; 5000 entries, 30,000 tokens 278 and 222).
// An odd number of parts, as workgroups go to the eight chiplets in turn.
constexpr int kFewRows = 3, kParts = 3, kLongHistory = 24;
constexpr uint32_t kPrompt = 0x80000000u;  // of a count: the entry occurs in the prompt
constexpr int32_t kNoBias = INT32_MIN;     // of the bias table: as a float, -0, which changes no sum

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
  int32_t num_rows, vocab, num_tokens, num_bias, num_masks;
  uint32_t stretches;
  bool stream;    // the output past the caches
  int32_t rows;   // consecutive rows to a workgroup, or `parts` times as many
  int32_t parts;  // 1 or kParts
  int32_t first;  // workgroups of the launches before this one
};

__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return min(max(x, lo), hi); }
__device__ __forceinline__ int lane_int(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
__device__ __forceinline__ float lane_float(float x, int lane) {
  return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane));
}

// kOnce: the input passes the caches by, which serve the logits beside it (backward, us, outputs streamed on both sides: 334 MB
// of gradient 151 -> 148, 304 MB 138 -> 131, 91 MB 54 -> 49, 67 MB 36 -> 37; 32 MB that the caches still hold 18 -> 20).
template <bool kGrad, bool kBias, bool kOnce>
__global__ __launch_bounds__(kLogitsThreads, 6) void logits_kernel(LogitsParams p) {
  // counts, and behind them the biases (in their place where the counts serve one row alone)
  extern __shared__ __align__(16) uint32_t table[];
  int32_t* bias_table = reinterpret_cast<int32_t*>(table) + (p.rows > 1 ? blockDim.x * kThreadEntries : 0);
  const int tid = threadIdx.x, lane = tid & 63, threads = blockDim.x, stretch = threads * kThreadEntries;
  const uint32_t unit = p.first + blockIdx.x, group = unit / p.stretches, part = p.parts > 1 ? group % kParts : 0;
  const int64_t row0 = static_cast<int64_t>(group - part) * p.rows;
  const int v0 = static_cast<int>(unit - group * p.stretches) * stretch, n = min(stretch, p.vocab - v0);
  const int rows = static_cast<int>(min(static_cast<int64_t>(p.rows) * p.parts, p.num_rows - row0));

  // Lane r of every wave keeps row r's arguments; the loops below read them from there.
  int begin = 0, split = 0, end = 0, bias_begin = 0, bias_end = 0, mask_row = -1;
  float rep = 1.f, freq = 0.f, pres = 0.f;
  if (lane < rows) {
    const int64_t row = row0 + lane;
    if (p.history != nullptr) {
      begin = clamp_int(p.history[3 * row], 0, p.num_tokens);
      split = p.history[3 * row + 1];
      end = clamp_int(p.history[3 * row + 2], begin, p.num_tokens);
      rep = p.penalties[3 * row];
      if constexpr (!kGrad) {
        freq = p.penalties[3 * row + 1];
        pres = p.penalties[3 * row + 2];
      }
    }
    if (kBias) {
      bias_begin = clamp_int(p.bias_rows[2 * row], 0, p.num_bias);
      bias_end = clamp_int(p.bias_rows[2 * row + 1], bias_begin, p.num_bias);
    }
    if (p.mask != nullptr) {
      const int64_t m = p.mask_rows != nullptr ? p.mask_rows[row] : row;
      mask_row = m >= 0 && m < p.num_masks ? static_cast<int>(m) : -1;
    }
  }
  // a row's history goes on from the one before: the first of its new tokens; otherwise -1
  int from = -1;
  {
    const int b = __shfl_up(begin, 1, 64), s = __shfl_up(split, 1, 64), e = __shfl_up(end, 1, 64);
    if (lane > 0 && b == begin && s == split && e <= end) from = e;
  }
  const int last_token = lane < rows && from >= 0 && end == from + 1 ? p.tokens[from] : -1;
  const bool one_here = static_cast<uint32_t>(last_token) - v0 < static_cast<uint32_t>(n);
  // the workgroup's rows: its part of the `rows`, or all of them to the first where they share a long history
  const int first_row = part * p.rows;
  int last_row = min(first_row + p.rows, rows);
  if (p.parts > 1 && lane_int(end, 0) - lane_int(begin, 0) > kLongHistory * threads && __ballot(lane > 0 && lane < rows && from < 0) == 0) {
    if (first_row > 0) return;
    last_row = rows;
  }
  const bool active = begin < end && (rep != 1.f || freq != 0.f || pres != 0.f);
  const uint64_t actives = __ballot(active && lane >= first_row && lane < last_row);
  const int bias_before = __shfl_up(bias_begin, 1, 64), bias_until = __shfl_up(bias_end, 1, 64);
  const bool new_bias = lane == first_row || bias_before != bias_begin || bias_until != bias_end;

  // a stretch's last piece, where it is shorter than others: its bounds are the workgroup's, not a thread's
  const int whole = n & ~7, rest = n & 7;
  auto load_rest = [&](const uint16_t* in) {
    u32x4 q = {0, 0, 0, 0};
    for (int e = 0; e < rest; ++e) q[e / 2] |= static_cast<uint32_t>(in[whole + e]) << (16 * (e & 1));
    return q;
  };
  auto load = [&](int r, u32x4 (&w)[kLogitsVecs], uint32_t (&keep)[kLogitsVecs]) {
    const uint16_t* in = p.in + (row0 + r) * p.in_stride + v0;
    const int m = lane_int(mask_row, r);
    const uint8_t* mask = reinterpret_cast<const uint8_t*>(p.mask + m * p.mask_stride) + v0 / 8;
#pragma unroll
    for (int i = 0; i < kLogitsVecs; ++i) {
      const int piece = tid + i * threads, e0 = 8 * piece;
      w[i] = u32x4{0, 0, 0, 0};
      keep[i] = 0xFF;
      if (e0 < whole)
        w[i] = load16_as<kOnce>(in, 0, piece);
      else if (e0 < n)
        w[i] = load_rest(in);
      if (m >= 0 && e0 < n) keep[i] = mask[piece];
    }
  };
  auto count = [&](int lo, int hi, int response) {
    constexpr int kAhead = 4;
    for (int i0 = lo + tid; i0 < hi; i0 += kAhead * threads) {
      int token[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) token[u] = i0 + u * threads < hi ? p.tokens[i0 + u * threads] : -1;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const uint32_t v = static_cast<uint32_t>(token[u]) - v0;
        if (v >= static_cast<uint32_t>(n)) continue;
        if (i0 + u * threads < response)
          atomicOr(&table[v], kPrompt);
        else
          atomicAdd(&table[v], 1);
      }
    }
  };

  // Backward: the logits of the pieces that hold entries of the history, and which of the next row's are here already
  // (those that this row's counts ask for; a row's own new ones are read when its counts are known).
  u32x4 z[kLogitsVecs];
  bool have_z[kLogitsVecs] = {};
  auto load_z = [&](int r, int i) {
    const int piece = tid + i * threads;
    const uint16_t* in = p.logits + (row0 + r) * p.logits_stride + v0;
    return 8 * piece < whole ? load16(in, 0, piece) : load_rest(in);
  };

  u32x4 next[kLogitsVecs];
  uint32_t next_keep[kLogitsVecs];
  load(first_row, next, next_keep);
  for (int r = first_row; r < last_row; ++r) {
    u32x4 w[kLogitsVecs];
    uint32_t keep[kLogitsVecs];
#pragma unroll
    for (int i = 0; i < kLogitsVecs; ++i) {
      w[i] = next[i];
      keep[i] = next_keep[i];
    }
    // a thread's first bias, asked for before the counts
    int first_id = -1;
    if (kBias && lane_int(new_bias, r) != 0) {
      const int i = lane_int(bias_begin, r) + tid;
      if (i < lane_int(bias_end, r)) first_id = p.bias_ids[i];
    }
    if (r + 1 < last_row) load(r + 1, next, next_keep);
    if (actives != 0) {
      const int lo = lane_int(begin, r), hi = lane_int(end, r), response = lane_int(split, r);
      const int at = r > first_row ? lane_int(from, r) : -1;
      if (at < 0) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kThreadEntries / 4; ++e) reinterpret_cast<u32x4*>(table)[e * threads + tid] = u32x4{0, 0, 0, 0};
        __syncthreads();
        count(lo, hi, response);
        __syncthreads();
      } else if (hi - at > 1 || lane_int(one_here, r) != 0) {
        __syncthreads();
        count(at, hi, response);
        __syncthreads();
      }
    }
    auto counts = [&](int i, uint32_t (&seen)[8]) {
      const u32x4* t = reinterpret_cast<const u32x4*>(table) + 2 * (tid + i * threads);
      const u32x4 a = t[0], b = t[1];
      uint32_t any = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        seen[e] = a[e];
        seen[e + 4] = b[e];
        any |= a[e] | b[e];
      }
      return any != 0;
    };
    auto put = [&](int i, float (&x)[8]) {
      uint16_t* out = p.out + (row0 + r) * p.out_stride + v0;
      const bool masked = lane_int(mask_row, r) >= 0;
      const int piece = tid + i * threads, e0 = 8 * piece;
      if (masked) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = keep[i] >> e & 1 ? x[e] : (kGrad ? 0.f : -__builtin_inff());
      }
      const u32x4 o = pack8(x);
      if (e0 < whole)
        store16_as(p.stream, out, 0, piece, o);
      else
        for (int e = 0; e < rest; ++e) out[whole + e] = static_cast<uint16_t>(o[e / 2] >> (16 * (e & 1)));
    };
    if constexpr (kGrad) {
      const float mul = lane_float(rep, r), inv = 1.f / mul;
      uint32_t hits[kLogitsVecs] = {};  // bit e: the piece's entry e is in the history; bit 8 + e: and its logit is above 0
      if (actives >> r & 1) {
#pragma unroll
        for (int i = 0; i < kLogitsVecs; ++i) {
          uint32_t seen[8];
          counts(i, seen);
#pragma unroll
          for (int e = 0; e < 8; ++e) hits[i] |= seen[e] != 0 ? 1u << e : 0;
          if (hits[i] != 0 && !have_z[i]) z[i] = load_z(r, i);
        }
#pragma unroll
        for (int i = 0; i < kLogitsVecs; ++i) {
          if (hits[i] == 0) continue;
          float zs[8];
          unpack8(z[i], zs);
#pragma unroll
          for (int e = 0; e < 8; ++e) hits[i] |= zs[e] > 0.f ? 256u << e : 0;
        }
      }
#pragma unroll
      for (int i = 0; i < kLogitsVecs; ++i) {
        have_z[i] = hits[i] != 0 && r + 1 < last_row;
        if (have_z[i]) z[i] = load_z(r + 1, i);
      }
#pragma unroll
      for (int i = 0; i < kLogitsVecs; ++i) {
        if (8 * (tid + i * threads) >= n) break;
        float x[8];
        unpack8(w[i], x);
        if (hits[i] != 0) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = hits[i] >> e & 1 ? x[e] * (hits[i] >> (8 + e) & 1 ? inv : mul) : x[e];
        }
        put(i, x);
      }
      continue;
    }
    float x[kLogitsVecs][8];
#pragma unroll
    for (int i = 0; i < kLogitsVecs; ++i) unpack8(w[i], x[i]);
    if (actives >> r & 1) {
      const float mul = lane_float(rep, r), inv = 1.f / mul, f = lane_float(freq, r), q = lane_float(pres, r);
#pragma unroll
      for (int i = 0; i < kLogitsVecs; ++i) {
        uint32_t seen[8];
        if (!counts(i, seen)) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t times = seen[e] & ~kPrompt;
          float y = x[i][e] * (x[i][e] > 0.f ? inv : mul);
          y = __builtin_fmaf(-f, static_cast<float>(times), y) - (times != 0 ? q : 0.f);
          x[i][e] = seen[e] == 0 ? x[i][e] : y;
        }
      }
    }
    if (kBias && lane_int(new_bias, r) != 0) {
      const int lo = lane_int(bias_begin, r), hi = lane_int(bias_end, r);
      __syncthreads();
#pragma unroll
      for (int e = 0; e < kThreadEntries / 4; ++e)
        reinterpret_cast<u32x4*>(bias_table)[e * threads + tid] = u32x4{kPrompt, kPrompt, kPrompt, kPrompt};
      __syncthreads();
      // the last entry that names v wins its place
      for (int i = lo + tid; i < hi; i += threads) {
        const uint32_t v = static_cast<uint32_t>(i == lo + tid ? first_id : p.bias_ids[i]) - v0;
        if (v < static_cast<uint32_t>(n)) atomicMax(&bias_table[v], i);
      }
      __syncthreads();
      if (hi - lo <= threads) {
        // an entry to a thread: the winners put their values there, once all have looked
        const uint32_t v = static_cast<uint32_t>(first_id) - v0;
        const bool wins = v < static_cast<uint32_t>(n) && bias_table[v] == lo + tid;
        __syncthreads();
        if (wins) bias_table[v] = __float_as_int(p.bias_values[lo + tid]);
      } else {
        // longer lists: each place takes its winner's value (a value's bits could be another entry's number)
        for (int e = tid; e < stretch; e += threads) {
          const int32_t i = bias_table[e];
          if (i != kNoBias) bias_table[e] = __float_as_int(p.bias_values[i]);
        }
      }
      __syncthreads();
    }
    if (kBias && lane_int(bias_begin, r) < lane_int(bias_end, r)) {
#pragma unroll
      for (int i = 0; i < kLogitsVecs; ++i) {
        const float4* t = reinterpret_cast<const float4*>(bias_table) + 2 * (tid + i * threads);
        const float4 a = t[0], b = t[1];
        const float add[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = x[i][e] + add[e];
      }
    }
#pragma unroll
    for (int i = 0; i < kLogitsVecs; ++i) {
      if (8 * (tid + i * threads) >= n) break;
      put(i, x[i]);
    }
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
  p.stretches = (a.vocab - 1) / kMostEntries + 1;
  const int threads = ((a.vocab - 1) / p.stretches / kThreadEntries / 64 + 1) * 64;  // equal parts, whole waves
  p.stream = streams(a.num_rows, a.vocab);
  // few rows are spread over all CUs, sixteen workgroups to each
  const int64_t share = static_cast<int64_t>(a.num_rows) * p.stretches / (16 * device_cus());
  p.rows = static_cast<int>(share < 1 ? 1 : share > kFewRows ? kFewRows : share);
  p.parts = share < kFewRows ? 1 : kParts;
  const int64_t groups = (static_cast<int64_t>(a.num_rows) + p.rows - 1) / p.rows;
  const size_t lds = sizeof(uint32_t) * threads * kThreadEntries * (a.bias_rows != nullptr && p.rows > 1 ? 2 : 1);
  return launch_parts(groups * p.stretches, threads, [&](int first, unsigned n) {
    p.first = first;
    if (grad && p.stream)
      hipLaunchKernelGGL((logits_kernel<true, false, true>), dim3(n), dim3(threads), lds, stream, p);
    else if (grad)
      hipLaunchKernelGGL((logits_kernel<true, false, false>), dim3(n), dim3(threads), lds, stream, p);
    else if (a.bias_rows != nullptr)
      hipLaunchKernelGGL((logits_kernel<false, true, false>), dim3(n), dim3(threads), lds, stream, p);
    else
      hipLaunchKernelGGL((logits_kernel<false, false, false>), dim3(n), dim3(threads), lds, stream, p);
  });
}

}  // namespace

hipError_t launch_logits_process(const LogitsLaunch& a, hipStream_t stream) { return launch_logits(a, false, stream); }
hipError_t launch_logits_process_backward(const LogitsLaunch& a, hipStream_t stream) {
  return launch_logits(a, true, stream);
}

}  // namespace uattn
