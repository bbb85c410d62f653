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
  int32_t hidden;
  int32_t first;  // rows of the launches before this one
};

__device__ __forceinline__ float inverse_rms(float mean, float eps) { return 1.0f / __builtin_sqrtf(mean + eps); }

template <int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads) void residual_norm_kernel(NormParams p) {
  constexpr int kWaves = kThreads / 64;
  __shared__ float slots[2][kWaves];
  const int tid = threadIdx.x, pieces = p.hidden / 8;
  const int64_t row = p.first + static_cast<int64_t>(blockIdx.x), base = row * pieces;
  float s[kVecs][8];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int v = tid + i * kThreads;
    u32x4 w = {0, 0, 0, 0};
    if (v < pieces) w = load16(p.residual, base + v);
    unpack8(w, s[i]);
  }
  if (p.x != nullptr) {
    float u[kVecs][8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kThreads;
      u32x4 w = {0, 0, 0, 0};
      if (v < pieces) w = load16(p.x, base + v);
      unpack8(w, u[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(u[i][e] * p.inv_hidden, u[i][e], sum);
    }
    float r = 1.f;
    if (p.post != nullptr) r = inverse_rms(block_sum<kWaves>(sum, slots[0]), p.eps);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kThreads;
      if (v >= pieces) break;
      float g[8];
      if (p.post != nullptr) {
        unpack8(load16(p.post, v), g);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[i][e] = u[i][e] * r * g[e];
      }
      if (p.gate != nullptr) {
        unpack8(load16(p.gate, row * (p.gate_stride / 8) + v), g);
#pragma unroll
        for (int e = 0; e < 8; ++e) u[i][e] = u[i][e] * g[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s[i][e] = s[i][e] + p.scale * u[i][e];
      store16(p.residual_out, base + v, pack8(s[i]));
    }
  }
  if (p.y == nullptr) return;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < kVecs; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(s[i][e] * p.inv_hidden, s[i][e], sum);
  const float r = inverse_rms(block_sum<kWaves>(sum, slots[1]), p.eps);
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int v = tid + i * kThreads;
    if (v >= pieces) break;
    float g[8];
    unpack8(load16(p.pre, v), g);
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = s[i][e] * r * g[e];
    store16(p.y, base + v, pack8(g));
  }
}

// Gradients at the stored h' and x.  With n = h' r(h'), m = x r(x):
//   a = dy w_pre,  ds = dh' + r(h') (a - n mean(a n)),  dw_pre = sum_rows dy n
//   b = scale ds gate,  dgate = scale ds u,  dw_post = sum_rows b m
//   c = b w_post,  dx = r(x) (c - m mean(c m))           (dx = b without w_post)
// A workgroup takes rows blockIdx, + gridDim, ... and keeps its share of the
// column sums in registers; they go to the workspace, one set to a workgroup, and
// a second kernel adds the sets in order.
struct NormGradParams {
  const void *dy, *dresidual_out, *h, *pre, *x, *post, *gate;
  void *dresidual, *dx, *dgate_rows;
  float* parts;  // [sums][gridDim][hidden]
  int64_t gate_stride;
  float scale, eps, inv_hidden;
  int32_t num_tokens, hidden;
  int32_t pre_at, post_at, gate_at;  // which of the sums each is, or -1
};

template <int kThreads, int kVecs>
__global__ __launch_bounds__(kThreads) void residual_norm_grad_kernel(NormGradParams p) {
  constexpr int kWaves = kThreads / 64;
  __shared__ float slots[4][kWaves];
  const int tid = threadIdx.x, pieces = p.hidden / 8;
  float dpre[kVecs][8] = {}, dpost[kVecs][8] = {}, dgate[kVecs][8] = {};
  for (int64_t row = blockIdx.x; row < p.num_tokens; row += gridDim.x) {
    const int64_t base = row * pieces;
    const u32x4 zero = {0, 0, 0, 0};
    float ds[kVecs][8];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kThreads;
      unpack8(p.dresidual_out != nullptr && v < pieces ? load16(p.dresidual_out, base + v) : zero, ds[i]);
    }
    if (p.dy != nullptr) {
      float n[kVecs][8], a[kVecs][8], sq = 0.f;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int v = tid + i * kThreads;
        unpack8(v < pieces ? load16(p.h, base + v) : zero, n[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sq = __builtin_fmaf(n[i][e] * p.inv_hidden, n[i][e], sq);
      }
      const float r = inverse_rms(block_sum<kWaves>(sq, slots[0]), p.eps);
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int v = tid + i * kThreads;
        float w[8];
        unpack8(v < pieces ? load16(p.dy, base + v) : zero, a[i]);
        unpack8(v < pieces ? load16(p.pre, v) : zero, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          n[i][e] = n[i][e] * r;
          dpre[i][e] = dpre[i][e] + a[i][e] * n[i][e];
          a[i][e] = a[i][e] * w[e];
          dot = dot + a[i][e] * n[i][e];
        }
      }
      dot = block_sum<kWaves>(dot, slots[1]) * p.inv_hidden;
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) ds[i][e] = ds[i][e] + r * (a[i][e] - n[i][e] * dot);
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kThreads;
      if (v < pieces) store16(p.dresidual, base + v, pack8(ds[i]));
    }
    if (p.dx == nullptr) {
      __syncthreads();
      continue;
    }
    float m[kVecs][8], sq = 0.f, r = 1.f;
    if (p.x != nullptr) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i) {
        const int v = tid + i * kThreads;
        unpack8(v < pieces ? load16(p.x, base + v) : zero, m[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sq = __builtin_fmaf(m[i][e] * p.inv_hidden, m[i][e], sq);
      }
      if (p.post != nullptr) r = inverse_rms(block_sum<kWaves>(sq, slots[2]), p.eps);
    }
    float dot = 0.f;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kThreads;
      float w[8], g[8];
      unpack8(p.post != nullptr && v < pieces ? load16(p.post, v) : zero, w);
      unpack8(p.gate != nullptr && v < pieces ? load16(p.gate, row * (p.gate_stride / 8) + v) : zero, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ds[i][e] = p.scale * ds[i][e];
        if (p.post != nullptr) m[i][e] = m[i][e] * r;
        if (p.gate != nullptr) {
          const float u = p.post != nullptr ? m[i][e] * w[e] : m[i][e];
          const float d = ds[i][e] * u;
          dgate[i][e] = dgate[i][e] + d;
          ds[i][e] = ds[i][e] * g[e];
          g[e] = d;
        }
        if (p.post != nullptr) {
          dpost[i][e] = dpost[i][e] + ds[i][e] * m[i][e];
          ds[i][e] = ds[i][e] * w[e];
          dot = dot + ds[i][e] * m[i][e];
        }
      }
      if (p.dgate_rows != nullptr && v < pieces) store16(p.dgate_rows, base + v, pack8(g));
    }
    if (p.post != nullptr) {
      dot = block_sum<kWaves>(dot, slots[3]) * p.inv_hidden;
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) ds[i][e] = r * (ds[i][e] - m[i][e] * dot);
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int v = tid + i * kThreads;
      if (v < pieces) store16(p.dx, base + v, pack8(ds[i]));
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int v = tid + i * kThreads;
    if (v >= pieces) break;
    auto put = [&](int at, const float(&d)[8]) {
      if (at < 0) return;
      float4* to = reinterpret_cast<float4*>(p.parts + (static_cast<int64_t>(at) * gridDim.x + blockIdx.x) * p.hidden) + 2 * v;
      to[0] = make_float4(d[0], d[1], d[2], d[3]);
      to[1] = make_float4(d[4], d[5], d[6], d[7]);
    };
    put(p.pre_at, dpre[i]);
    put(p.post_at, dpost[i]);
    put(p.gate_at, dgate[i]);
  }
}

struct FoldParams {
  const float* parts;  // [sums][sets][hidden]
  float* out[3];
  int32_t sets, hidden;
};

__global__ __launch_bounds__(64) void norm_fold_kernel(FoldParams p) {
  const int col = blockIdx.x * 64 + threadIdx.x;
  if (col >= p.hidden) return;
  const float* in = p.parts + static_cast<int64_t>(blockIdx.y) * p.sets * p.hidden + col;
  float s = 0.f;
  for (int i = 0; i < p.sets; ++i) s = s + in[static_cast<int64_t>(i) * p.hidden];
  p.out[blockIdx.y][col] = s;
}

constexpr int kMaxSets = 256;

int norm_sets(int64_t num_tokens) { return static_cast<int>(num_tokens < kMaxSets ? num_tokens : kMaxSets); }

}  // namespace

hipError_t launch_residual_norm(const ResidualNormLaunch& a, hipStream_t stream) {
  NormParams p{a.x, a.post_weight, a.gate, a.residual, a.pre_weight, a.residual_out, a.y, a.gate_stride, a.scale, a.eps,
               1.0f / a.hidden_dim, a.hidden_dim, 0};
  auto launch = [&](auto vecs) {
    return launch_parts(a.num_tokens, 256, [&](int first, unsigned n) {
      p.first = first;
      hipLaunchKernelGGL((residual_norm_kernel<256, decltype(vecs)::value>), dim3(n), dim3(256), 0, stream, p);
    });
  };
  using std::integral_constant;
  if (a.hidden_dim <= 2048) return launch(integral_constant<int, 1>{});
  if (a.hidden_dim <= 4096) return launch(integral_constant<int, 2>{});
  if (a.hidden_dim <= 8192) return launch(integral_constant<int, 4>{});
  return launch(integral_constant<int, 8>{});
}

size_t residual_norm_backward_ws_bytes(int64_t num_tokens, int64_t hidden_dim) {
  return static_cast<size_t>(3) * norm_sets(num_tokens) * hidden_dim * sizeof(float);
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
  f.sets = norm_sets(a.num_tokens);
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
    auto launch = [&](auto threads, auto vecs) {
      hipLaunchKernelGGL((residual_norm_grad_kernel<decltype(threads)::value, decltype(vecs)::value>), dim3(f.sets),
                         dim3(decltype(threads)::value), 0, stream, p);
    };
    using std::integral_constant;
    if (a.hidden_dim <= 2048)
      launch(integral_constant<int, 256>{}, integral_constant<int, 1>{});
    else if (a.hidden_dim <= 4096)
      launch(integral_constant<int, 512>{}, integral_constant<int, 1>{});
    else if (a.hidden_dim <= 8192)
      launch(integral_constant<int, 1024>{}, integral_constant<int, 1>{});
    else
      launch(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (sums > 0) {
    hipLaunchKernelGGL(norm_fold_kernel, dim3((a.hidden_dim + 63) / 64, sums), dim3(64), 0, stream, f);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace uattn
