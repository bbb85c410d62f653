// The seam between two blocks of a transformer in one pass, and its gradients:
//
//   u = x * r(x) * w_post      the block output's norm   (u = x without w_post)
//   s = h + scale * gate * u   the residual sum          (h' = bf16(s) is stored)
//   y = s * r(s) * w_pre       the next block's norm     (r(a) = 1 / sqrt(mean a^2 + eps))
//
// A row lives in its workgroup's registers from its loads to its stores.  The
// sums over a row are taken in an order fixed by hidden_dim alone (a thread's
// pieces in order, lanes, waves), so a row's bits do not depend on the batch.
// Squares are summed divided by hidden_dim already: what has to fit fp32 is the
// mean of a row's squares, not their sum.
#include <type_traits>

#include "uattn_internal.h"
#include "uattn_rows.h"

namespace uattn {
namespace {

struct NormParams {
  const void *x, *post, *gate, *residual, *pre;
  void *residual_out, *y;
  int64_t gate_stride;
  float scale, eps, inv_hidden;
  int32_t num_tokens, hidden;
  int32_t first;  // rows of the launches before this one
};

__device__ __forceinline__ float inverse_rms(float mean, float eps) { return 1.0f / __builtin_sqrtf(mean + eps); }

// A row is taken by kRowWaves waves, kVecs pieces to a thread; a workgroup has four waves, or a row's
// where that is more.  Bound by memory.
template <int kRowWaves>
constexpr int kNormWaves = kRowWaves > 4 ? kRowWaves : 4;

// kOnce: the rows pass the caches by, read and written, from the size on from which outputs do (streams(), with what both
// sides take: 80 MB 60 -> 54 us, but 33 MB, which the caches hold, 22 -> 24).
template <int kRowWaves, int kVecs, bool kOnce>
__global__ __launch_bounds__(64 * kNormWaves<kRowWaves>) void residual_norm_kernel(NormParams p) {
  constexpr int kWaves = kNormWaves<kRowWaves>, kRows = kWaves / kRowWaves;
  __shared__ float slots[2][kWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = wave / kRowWaves, wave0 = group * kRowWaves, in_row = (wave - wave0) * 64 + lane;
  const int pieces = p.hidden / 8;
  const int64_t row = p.first + static_cast<int64_t>(blockIdx.x) * kRows + group, base = row * pieces;
  const bool here = row < p.num_tokens;
  auto piece = [&](int i) { return in_row + i * 64 * kRowWaves; };
  const u32x4 zero = {0, 0, 0, 0};
  u32x4 hw[kVecs], xw[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    hw[i] = xw[i] = zero;
    if (!here || piece(i) >= pieces) continue;
    hw[i] = load16_as<kOnce>(p.residual, base, piece(i));
    if (p.x != nullptr) xw[i] = load16_as<kOnce>(p.x, base, piece(i));
  }
  float s[kVecs][8];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) unpack8(hw[i], s[i]);
  if (p.x != nullptr) {
    float r = 1.f;
    if (p.post != nullptr) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        float u[8];
        unpack8(xw[i], u);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(u[e] * p.inv_hidden, u[e], sum);
      }
      r = inverse_rms(waves_sum<kRowWaves>(sum, slots[0], wave, wave0), p.eps);
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      if (!here || piece(i) >= pieces) break;
      float u[8], g[8];
      unpack8(xw[i], u);
      if (p.post != nullptr) {
        unpack8(load16(p.post, 0, piece(i)), g);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = u[e] * r * g[e];
      }
      if (p.gate != nullptr) {
        unpack8(load16(p.gate, row * (p.gate_stride / 8), piece(i)), g);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = u[e] * g[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s[i][e] = __builtin_fmaf(p.scale, u[e], s[i][e]);
      store16_as(kOnce, p.residual_out, base, piece(i), pack8(s[i]));
    }
  }
  if (p.y == nullptr) return;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kVecs; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(s[i][e] * p.inv_hidden, s[i][e], sum);
  const float r = inverse_rms(waves_sum<kRowWaves>(sum, slots[1], wave, wave0), p.eps);
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    if (!here || piece(i) >= pieces) break;
    float g[8];
    unpack8(load16(p.pre, 0, piece(i)), g);
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = s[i][e] * r * g[e];
    store16_as(kOnce, p.y, base, piece(i), pack8(g));
  }
}

// Gradients at the stored h' and x.  With n = h' r(h'), m = x r(x):
//   a = dy w_pre,  ds = dh' + r(h') (a - n mean(a n)),  dw_pre = sum_rows dy n
//   b = scale ds gate,  dgate = scale ds u,  dw_post = sum_rows b m
//   c = b w_post,  dx = r(x) (c - m mean(c m))           (dx = b without w_post)
//
// Bound by memory: five rows read and three written for a token at most.  A workgroup of up to sixteen
// waves, one to a CU, takes as many rows at a time as have room (a wave handles 512 columns of a row,
// or twice 512), and asks for its next rows before it works on these.  mean(a n) is
// r(h') mean(a h'), so the sums of squares and this one meet in one exchange between the waves and
// mean(c m) in a second.  The column sums stay in registers over all rows of the workgroup; the
// workgroup's row groups add theirs through LDS, one set of sums to a workgroup goes to the
// workspace, and a second kernel adds the sets.  Which rows share a set depends on the numbers of
// tokens and columns alone.  Its outputs go through the caches whatever their size (us, so / past them:
// 9815 x 4096 111 / 114, 39,855 x 1024 111 / 112, 39,855 x 4096 389 / 400, 12,000 x 8192 245 / 252, 6000 x 16,384
// 368 / 365, and the same with a reader of both).  Two pieces to a thread take the 128 registers that sixteen
// waves leave and spill 24.
constexpr int kGradWaves = 16, kGradThreads = 64 * kGradWaves;
constexpr int kMaxSets = 256;

struct NormGradParams {
  const void *dy, *dresidual_out, *h, *pre, *x, *post, *gate;
  void *dresidual, *dx, *dgate_rows;
  float* parts;  // [sums][gridDim][hidden]
  int64_t gate_stride;
  float scale, eps, inv_hidden;
  int32_t num_tokens, hidden;
  int32_t row_waves, groups;  // waves to a row, rows to a workgroup at a time
  int32_t pre_at, post_at, gate_at;  // which of the sums each is, or -1
};

// A token's pieces of one thread.
template <int kVecs>
struct GradRow {
  u32x4 dy[kVecs], dr[kVecs], h[kVecs], x[kVecs], gate[kVecs];
};

template <int kVecs, bool kAhead>
__global__ __launch_bounds__(kGradThreads) void residual_norm_grad_kernel(NormGradParams p) {
  __shared__ float4 squares[2][kGradWaves];
  __shared__ float dots[2][kGradWaves];
  // the groups' meeting place; with two pieces to a thread (one group) the place of two of the three column sums, for
  // which the registers have no room
  __shared__ float4 columns[kGradThreads * (kVecs == 1 ? 2 : 4 * kVecs)];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row_waves = p.row_waves, groups = p.groups;
  const int group = wave / row_waves, wave0 = group * row_waves, in_row = (wave - wave0) * 64 + lane;
  const int pieces = p.hidden / 8;
  const int64_t step = static_cast<int64_t>(gridDim.x) * groups;
  const u32x4 zero = {0, 0, 0, 0};
  auto piece = [&](int i) { return in_row + i * 64 * row_waves; };

  // the weights stay in registers where the next rows do, and come from the cache where they are used otherwise
  u32x4 w_pre[kVecs], w_post[kVecs], w_gate[kVecs];
  auto weight = [&](const void* w, int i) { return w != nullptr && piece(i) < pieces ? load16(w, piece(i)) : zero; };
  const void* shared_gate = p.gate_stride == 0 ? p.gate : nullptr;
  if constexpr (kAhead) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      w_pre[i] = weight(p.pre, i);
      w_post[i] = weight(p.post, i);
      w_gate[i] = weight(shared_gate, i);
    }
  }
  auto pre_of = [&](int i) { return kAhead ? w_pre[i] : weight(p.pre, i); };
  auto post_of = [&](int i) { return kAhead ? w_post[i] : weight(p.post, i); };
  float dpre[kVecs][8] = {}, dpost[kVecs][8] = {}, dgate[kVecs][8] = {};
  // the two float4 of piece i of dpost (which = 0) and dgate (1)
  auto held = [&](int which, int i, int half) -> float4& { return columns[((which * kVecs + i) * 2 + half) * kGradThreads + tid]; };
  if constexpr (kVecs > 1) {
#pragma unroll
    for (int u = 0; u < 4 * kVecs; ++u) columns[u * kGradThreads + tid] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  auto add_held = [&](int which, int i, const float(&d)[8]) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      float4 t = held(which, i, half);
      t.x = t.x + d[4 * half];
      t.y = t.y + d[4 * half + 1];
      t.z = t.z + d[4 * half + 2];
      t.w = t.w + d[4 * half + 3];
      held(which, i, half) = t;
    }
  };

  const bool reads_x = p.post != nullptr || p.gate != nullptr;
  // rows behind the last one read as zeros, which add nothing
  auto load = [&](GradRow<kVecs>& d, int64_t row) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = piece(i);
      const bool here = row < p.num_tokens && v < pieces;
      const int64_t at = row * pieces;
      d.dy[i] = d.dr[i] = d.h[i] = d.x[i] = zero;
      d.gate[i] = kAhead ? w_gate[i] : zero;
      if (!here) continue;
      if (p.dresidual_out != nullptr) d.dr[i] = load16(p.dresidual_out, at, v);
      if (p.dy != nullptr) {
        d.h[i] = load16(p.h, at, v);
        d.dy[i] = load16(p.dy, at, v);
      }
      if (reads_x) d.x[i] = load16(p.x, at, v);
      if (p.gate_stride != 0 && p.gate != nullptr) d.gate[i] = load16(p.gate, at, v);
    }
  };

  GradRow<kVecs> next;
  int64_t row = static_cast<int64_t>(blockIdx.x) * groups + group;
  if constexpr (kAhead) load(next, row);
  int side = 0;
  for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * groups; row0 < p.num_tokens; row0 += step, row += step, side ^= 1) {
    if constexpr (!kAhead) load(next, row);
    const GradRow<kVecs> d = next;
    if constexpr (kAhead) load(next, row + step);
    const bool here = row < p.num_tokens;
    float r = 0.f, dot = 0.f, rx = 1.f;
    if (p.dy != nullptr || p.post != nullptr) {
      float hh = 0.f, ah = 0.f, xx = 0.f;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        float h[8], a[8], w[8], x[8];
        unpack8(d.h[i], h);
        unpack8(d.dy[i], a);
        unpack8(pre_of(i), w);
        unpack8(d.x[i], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float t = h[e] * p.inv_hidden;
          hh = __builtin_fmaf(t, h[e], hh);
          ah = __builtin_fmaf(a[e] * w[e], t, ah);
          xx = __builtin_fmaf(x[e] * p.inv_hidden, x[e], xx);
        }
      }
      hh = wave_sum(hh);
      ah = wave_sum(ah);
      xx = wave_sum(xx);
      if (row_waves > 1) {
        if (lane == 0) squares[side][wave] = make_float4(hh, ah, xx, 0.f);
        __syncthreads();
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
        if ((lane & 15) < row_waves) t = squares[side][wave0 + (lane & 15)];
        hh = period_sum<16>(t.x);
        ah = period_sum<16>(t.y);
        xx = period_sum<16>(t.z);
      }
      r = inverse_rms(hh, p.eps);
      dot = r * ah;
      if (p.post != nullptr) rx = inverse_rms(xx, p.eps);
    }
    float ds[kVecs][8];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      unpack8(d.dr[i], ds[i]);
      if (p.dy != nullptr && here) {
        float h[8], dy[8], w[8];
        unpack8(d.h[i], h);
        unpack8(d.dy[i], dy);
        unpack8(pre_of(i), w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float n = h[e] * r;
          dpre[i][e] = __builtin_fmaf(dy[e], n, dpre[i][e]);
          ds[i][e] = __builtin_fmaf(r, __builtin_fmaf(-n, dot, dy[e] * w[e]), ds[i][e]);
        }
      }
      if (here && piece(i) < pieces) store16(p.dresidual, row * pieces, piece(i), pack8(ds[i]));
    }
    if (p.dx == nullptr) continue;
    float cm = 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      float m[8], w[8], g[8];
      unpack8(d.x[i], m);
      unpack8(post_of(i), w);
      unpack8(kAhead || shared_gate == nullptr ? d.gate[i] : weight(shared_gate, i), g);
#pragma unroll
      for (int e = 0; e < 8; ++e) ds[i][e] = p.scale * ds[i][e];
      if (!here) continue;
      if (p.post != nullptr) {
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = m[e] * rx;
      }
      if (p.gate != nullptr) {
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          t[e] = ds[i][e] * (p.post != nullptr ? m[e] * w[e] : m[e]);
          if constexpr (kVecs == 1) dgate[i][e] = dgate[i][e] + t[e];
          ds[i][e] = ds[i][e] * g[e];
        }
        if constexpr (kVecs > 1)
          if (p.gate_at >= 0) add_held(1, i, t);
        if (p.dgate_rows != nullptr && piece(i) < pieces) store16(p.dgate_rows, row * pieces, piece(i), pack8(t));
      }
      if (p.post != nullptr) {
        if constexpr (kVecs > 1) {
          float t[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) t[e] = ds[i][e] * m[e];
          add_held(0, i, t);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (kVecs == 1) dpost[i][e] = __builtin_fmaf(ds[i][e], m[e], dpost[i][e]);
          ds[i][e] = ds[i][e] * w[e];
          cm = __builtin_fmaf(ds[i][e] * p.inv_hidden, m[e], cm);
        }
      }
    }
    if (p.post != nullptr) {
      cm = wave_sum(cm);
      if (row_waves > 1) {
        if (lane == 0) dots[side][wave] = cm;
        __syncthreads();
        cm = period_sum<16>((lane & 15) < row_waves ? dots[side][wave0 + (lane & 15)] : 0.f);
      }
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        float x[8];
        unpack8(d.x[i], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) ds[i][e] = rx * __builtin_fmaf(-(x[e] * rx), cm, ds[i][e]);
      }
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if (here && piece(i) < pieces) store16(p.dx, row * pieces, piece(i), pack8(ds[i]));
  }
  // the row groups' column sums, in the groups' order, by the first of them
  auto put = [&](int at, const float(&d)[8], int v) {
    if (at < 0) return;
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = d[e];
    if (groups > 1) {
      float* meet = reinterpret_cast<float*>(columns);
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) meet[e * kGradThreads + tid] = d[e];
      __syncthreads();
      if (group != 0) return;
      for (int u = 1; u < groups; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = s[e] + meet[e * kGradThreads + u * 64 * row_waves + tid];
    }
    if (v >= pieces) return;
    float4* to = reinterpret_cast<float4*>(p.parts + (static_cast<int64_t>(at) * gridDim.x + blockIdx.x) * p.hidden) + 2 * v;
    to[0] = make_float4(s[0], s[1], s[2], s[3]);
    to[1] = make_float4(s[4], s[5], s[6], s[7]);
  };
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    if constexpr (kVecs > 1) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const float4 a = held(0, i, half), b = held(1, i, half);
        dpost[i][4 * half] = a.x, dpost[i][4 * half + 1] = a.y, dpost[i][4 * half + 2] = a.z, dpost[i][4 * half + 3] = a.w;
        dgate[i][4 * half] = b.x, dgate[i][4 * half + 1] = b.y, dgate[i][4 * half + 2] = b.z, dgate[i][4 * half + 3] = b.w;
      }
    }
    put(p.pre_at, dpre[i], piece(i));
    put(p.post_at, dpost[i], piece(i));
    put(p.gate_at, dgate[i], piece(i));
  }
}

struct FoldParams {
  const float* parts;  // [sums][sets][hidden]
  float* out[3];
  int32_t sets, hidden;
};

// Adds the sets: 64 columns to a workgroup, four to a thread, the sets s, s + 64, ... to the threads
// of slot s, then the slots pairwise.
constexpr int kFoldSlots = 64;
__global__ __launch_bounds__(16 * kFoldSlots) void norm_fold_kernel(FoldParams p) {
  __shared__ float4 slots[kFoldSlots][16];
  const int quad = threadIdx.x & 15, slot = threadIdx.x >> 4, col = blockIdx.x * 64 + 4 * quad;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [](float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); };
  if (col < p.hidden) {
    const float* in = p.parts + static_cast<int64_t>(blockIdx.y) * p.sets * p.hidden + col;
    float4 q[kMaxSets / kFoldSlots];
#pragma unroll
    for (int i = 0; i < kMaxSets / kFoldSlots; ++i) {
      const int set = slot + i * kFoldSlots;
      q[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (set < p.sets) q[i] = *reinterpret_cast<const float4*>(in + static_cast<int64_t>(set) * p.hidden);
    }
#pragma unroll
    for (int i = 0; i < kMaxSets / kFoldSlots; ++i) s = add(s, q[i]);
  }
  for (int half = kFoldSlots / 2; half >= 1; half /= 2) {
    slots[slot][quad] = s;
    __syncthreads();
    if (slot < half) s = add(s, slots[slot + half][quad]);
    __syncthreads();
  }
  if (slot == 0 && col < p.hidden) *reinterpret_cast<float4*>(p.out[blockIdx.y] + col) = s;
}

// Pieces to a thread, and waves to a row.
int grad_vecs(int64_t hidden_dim) { return hidden_dim <= 512 * kGradWaves ? 1 : 2; }
int grad_row_waves(int64_t hidden_dim) {
  const int64_t columns = 512 * grad_vecs(hidden_dim);
  return static_cast<int>((hidden_dim + columns - 1) / columns);
}

int norm_sets(int64_t num_tokens, int64_t hidden_dim) {
  const int groups = kGradWaves / grad_row_waves(hidden_dim);
  const int64_t sets = (num_tokens + groups - 1) / groups;
  return static_cast<int>(sets < kMaxSets ? sets : kMaxSets);
}

}  // namespace

hipError_t launch_residual_norm(const ResidualNormLaunch& a, hipStream_t stream) {
  NormParams p{a.x, a.post_weight, a.gate, a.residual, a.pre_weight, a.residual_out, a.y, a.gate_stride, a.scale, a.eps,
               1.0f / a.hidden_dim, a.num_tokens, a.hidden_dim, 0};
  const bool once = streams(a.num_tokens, a.hidden_dim);
  auto launch = [&](auto row_waves, auto vecs) {
    constexpr int kRowWaves = decltype(row_waves)::value, kVecs = decltype(vecs)::value;
    constexpr int kWaves = kNormWaves<kRowWaves>, kRows = kWaves / kRowWaves;
    return launch_parts((static_cast<int64_t>(a.num_tokens) + kRows - 1) / kRows, 64 * kWaves, [&](int first, unsigned n) {
      p.first = first * kRows;
      if (once)
        hipLaunchKernelGGL((residual_norm_kernel<kRowWaves, kVecs, true>), dim3(n), dim3(64 * kWaves), 0, stream, p);
      else
        hipLaunchKernelGGL((residual_norm_kernel<kRowWaves, kVecs, false>), dim3(n), dim3(64 * kWaves), 0, stream, p);
    });
  };
  using std::integral_constant;
  const integral_constant<int, 1> one;
  const integral_constant<int, 2> two;
  const integral_constant<int, 4> four;
  const integral_constant<int, 8> eight;
  if (a.hidden_dim <= 512) return launch(one, one);
  if (a.hidden_dim <= 1024) return launch(one, two);
  if (a.hidden_dim <= 2048) return launch(one, four);
  if (a.hidden_dim <= 4096) return launch(four, two);
  if (a.hidden_dim <= 8192) return launch(eight, two);
  return launch(eight, four);
}

size_t residual_norm_backward_ws_bytes(int64_t num_tokens, int64_t hidden_dim) {
  return static_cast<size_t>(3) * norm_sets(num_tokens, hidden_dim) * hidden_dim * sizeof(float);
}

hipError_t launch_residual_norm_backward(const ResidualNormBackwardLaunch& a, hipStream_t stream) {
  NormGradParams p{};
  p.dy = a.dy;
  p.dresidual_out = a.dresidual_out;
  p.h = a.residual_out;
  p.pre = a.pre_weight;
  p.x = a.x;
  p.post = a.post_weight;
  p.gate = a.gate;
  p.dresidual = a.dresidual;
  p.dx = a.dx;
  p.dgate_rows = a.gate_stride != 0 ? a.dgate : nullptr;
  p.parts = static_cast<float*>(a.workspace);
  p.gate_stride = a.gate_stride;
  p.scale = a.scale;
  p.eps = a.eps;
  p.inv_hidden = 1.0f / a.hidden_dim;
  p.num_tokens = a.num_tokens;
  p.hidden = a.hidden_dim;
  FoldParams f{};
  f.parts = p.parts;
  f.sets = norm_sets(a.num_tokens, a.hidden_dim);
  f.hidden = a.hidden_dim;
  int sums = 0;
  auto sum_of = [&](float* out) {
    if (out == nullptr) return -1;
    f.out[sums] = out;
    return sums++;
  };
  p.pre_at = sum_of(a.dpre_weight);
  p.post_at = sum_of(a.dpost_weight);
  p.gate_at = sum_of(a.gate_stride == 0 ? static_cast<float*>(a.dgate) : nullptr);
  if (f.sets > 0) {
    p.row_waves = grad_row_waves(a.hidden_dim);
    p.groups = kGradWaves / p.row_waves;
    const dim3 threads(64 * p.row_waves * p.groups);
    if (grad_vecs(a.hidden_dim) == 1)
      hipLaunchKernelGGL((residual_norm_grad_kernel<1, true>), dim3(f.sets), threads, 0, stream, p);
    else
      hipLaunchKernelGGL((residual_norm_grad_kernel<2, false>), dim3(f.sets), threads, 0, stream, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (sums > 0) {
    hipLaunchKernelGGL(norm_fold_kernel, dim3((a.hidden_dim + 63) / 64, sums), dim3(16 * kFoldSlots), 0, stream, f);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace uattn
