// Embedding lookup, and the gradient of its table by sorted tokens.
//
// Lookup: out[t] = bf16(scale * table[ids[t]]), a wave to a token's row.
//
// Gradient: grad[v] = scale * (sum of dout[t] over the tokens t with ids[t] = v).
// The tokens are sorted by id, stably (a radix sort of 9 bits a pass), so that an
// entry's tokens stand together and in ascending order.  An entry's run is cut
// into pieces of kPiece tokens counted from the run's own first one; a wave sums
// one piece over 512 columns, in order, in fp32; runs of one piece are written at
// once, the pieces of longer ones meet in the workspace and are added in order.
// So a row's sum depends on its own tokens' rows alone: no atomic touches a
// value, and the same tokens give the same bits in any batch.
#include <type_traits>

#include "uattn_internal.h"
#include "uattn_rows.h"

namespace uattn {
namespace {

// ---------------------------------------------------------------------------
// Lookup
// ---------------------------------------------------------------------------
struct EmbeddingParams {
  const int32_t* ids;
  const void* table;
  void* out;
  int64_t table_stride, out_stride;
  float scale;
  int32_t num_tokens, vocab, hidden;
  int32_t first;  // tokens of the launches before this one
};

constexpr int kEmbedWaves = 4;

__global__ __launch_bounds__(kEmbedWaves * 64) void embedding_kernel(EmbeddingParams p) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t t = p.first + static_cast<int64_t>(blockIdx.x) * kEmbedWaves + wave;
  if (t >= p.num_tokens) return;
  const int32_t id = p.ids[t];
  const int pieces = p.hidden / 8;
  const bool known = id >= 0 && id < p.vocab;
  const int64_t from = known ? id * (p.table_stride / 8) : 0, to = t * (p.out_stride / 8);
  const uint32_t fill = id < 0 ? 0u : 0x7FC07FC0u;  // padding, or an id outside the table
  for (int v = lane; v < pieces; v += 64) {
    u32x4 w = {fill, fill, fill, fill};
    if (known) {
      float x[8];
      unpack8(load16(p.table, from + v), x);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] * p.scale;
      w = pack8(x);
    }
    store16(p.out, to + v, w);
  }
}

// ---------------------------------------------------------------------------
// Sorting
// ---------------------------------------------------------------------------
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;
constexpr int kSortThreads = 256, kSortWaves = kSortThreads / 64;
constexpr int kSortTile = 4096, kWaveTile = kSortTile / kSortWaves;

// Ids outside [0, vocab) have no row: they sort behind all others.
__device__ __forceinline__ uint32_t sort_key(int32_t id, int32_t vocab) {
  return static_cast<uint32_t>(id >= 0 && id < vocab ? id : vocab);
}

struct SortParams {
  const int32_t* ids;            // the first pass reads these, the others keys_in and order_in
  const uint32_t* keys_in;
  const int32_t* order_in;
  uint32_t* keys_out;
  int32_t* order_out;
  int32_t* hist;                 // [tiles][kBins]
  int32_t* counts;               // of the lists built after the sort: cleared by the first pass
  int32_t num_tokens, vocab, tiles, shift;
};

template <bool kFirst>
__device__ __forceinline__ uint32_t key_at(const SortParams& p, int i) {
  return kFirst ? sort_key(p.ids[i], p.vocab) : p.keys_in[i];
}

// How often each digit occurs in a tile.
template <bool kFirst>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortParams p) {
  __shared__ int32_t count[kBins];
  const int tid = threadIdx.x;
  if (kFirst && blockIdx.x == 0 && tid < 2) p.counts[tid] = 0;
  for (int b = tid; b < kBins; b += kSortThreads) count[b] = 0;
  __syncthreads();
  const int begin = blockIdx.x * kSortTile;
  for (int i = begin + tid; i < min(begin + kSortTile, p.num_tokens); i += kSortThreads)
    atomicAdd(&count[key_at<kFirst>(p, i) >> p.shift & (kBins - 1)], 1);
  __syncthreads();
  for (int b = tid; b < kBins; b += kSortThreads) p.hist[static_cast<int64_t>(blockIdx.x) * kBins + b] = count[b];
}

// The lanes of the wave whose digit is this lane's.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool valid) {
  uint64_t same = __ballot(valid);
#pragma unroll
  for (int b = 0; b < kDigitBits; ++b) {
    const uint64_t set = __ballot(digit >> b & 1);
    same &= digit >> b & 1 ? set : ~set;
  }
  return same;
}

// Moves a tile's tokens behind the smaller digits of all tiles and the equal ones of the tiles before.
template <bool kFirst>
__global__ __launch_bounds__(kSortThreads) void sort_move_kernel(SortParams p) {
  __shared__ int32_t next[kSortWaves][kBins];  // where a wave's next token of a digit goes
  __shared__ int32_t scan[2][kBins];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int begin = blockIdx.x * kSortTile + wave * kWaveTile, end = min(begin + kWaveTile, p.num_tokens);
  for (int b = tid; b < kSortWaves * kBins; b += kSortThreads) next[0][b] = 0;
  __syncthreads();
  for (int i = begin + lane; i < end; i += 64)
    atomicAdd(&next[wave][key_at<kFirst>(p, i) >> p.shift & (kBins - 1)], 1);
  // of each digit: all its tokens, and those in the tiles before this one
  int32_t before[kBins / kSortThreads];
#pragma unroll
  for (int u = 0; u < kBins / kSortThreads; ++u) {
    const int b = tid + u * kSortThreads;
    int32_t all = 0, earlier = 0;
    for (int t = 0; t < p.tiles; ++t) {
      const int32_t n = p.hist[static_cast<int64_t>(t) * kBins + b];
      all += n;
      if (t < static_cast<int>(blockIdx.x)) earlier += n;
    }
    scan[0][b] = all;
    before[u] = earlier - all;
  }
  __syncthreads();
  int from = 0;
  for (int d = 1; d < kBins; d *= 2, from ^= 1) {
    for (int b = tid; b < kBins; b += kSortThreads) scan[from ^ 1][b] = scan[from][b] + (b >= d ? scan[from][b - d] : 0);
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < kBins / kSortThreads; ++u) {
    const int b = tid + u * kSortThreads;
    int32_t at = scan[from][b] + before[u];
    for (int w = 0; w < kSortWaves; ++w) {
      const int32_t n = next[w][b];
      next[w][b] = at;
      at += n;
    }
  }
  __syncthreads();
  for (int i0 = begin; i0 < end; i0 += 64) {
    const int i = i0 + lane;
    const bool valid = i < end;
    const uint32_t key = valid ? key_at<kFirst>(p, i) : 0;
    const uint32_t digit = key >> p.shift & (kBins - 1);
    const uint64_t same = same_digit(digit, valid);
    const int rank = __popcll(same & ((uint64_t{1} << lane) - 1));
    int at = 0;
    if (valid && rank == 0) at = atomicAdd(&next[wave][digit], __popcll(same));
    at = __shfl(at, same != 0 ? __ffsll(static_cast<unsigned long long>(same)) - 1 : 0, 64) + rank;
    if (valid) {
      p.keys_out[at] = key;
      p.order_out[at] = kFirst ? i : p.order_in[i];
    }
  }
}

// ---------------------------------------------------------------------------
// Sums
// ---------------------------------------------------------------------------
constexpr int kPiece = 64;                 // tokens a wave sums
constexpr int kPieceOfLong = 1 << 30;      // the run goes on: the sum is a part

struct GradParams {
  const uint32_t* keys;   // sorted
  const int32_t* order;
  const void* dout;
  void* grad;
  int32_t* counts;        // pieces, long runs
  int2* pieces;           // first sorted position, tokens (| kPieceOfLong)
  int32_t* longs;         // first sorted position
  float* parts;           // [2 * ceil(T / kPiece)][hidden]
  int64_t dout_stride, grad_stride;
  float scale;
  int32_t num_tokens, vocab, hidden;
};

// The first sorted position in [lo, hi) whose key is above `key - !after`: the run's start or its end.
__device__ __forceinline__ int run_bound(const uint32_t* keys, int lo, int hi, uint32_t key, bool after) {
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (keys[mid] < key || (after && keys[mid] == key))
      lo = mid + 1;
    else
      hi = mid;
  }
  return lo;
}

// Of the pieces of runs longer than one: at most one first piece, and at most one later one, starts in
// any kPiece positions (the run between two first ones is longer, and a later piece starts that far
// behind its predecessor), so the two places of a stretch are never shared.
__device__ __forceinline__ int64_t part_of(int position, bool first) { return 2 * (position / kPiece) + (first ? 0 : 1); }

// Lists the pieces: every sorted position that is a multiple of kPiece behind its run's start begins one.
__global__ __launch_bounds__(256) void list_pieces_kernel(GradParams p) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= p.num_tokens) return;
  const uint32_t key = p.keys[i];
  if (key >= static_cast<uint32_t>(p.vocab)) return;
  const bool first = i == 0 || p.keys[i - 1] != key;
  if (!first) {
    if (i < kPiece || p.keys[i - kPiece] != key) return;
    if ((i - run_bound(p.keys, 0, i, key, false)) % kPiece != 0) return;
  }
  const int most = min(i + kPiece, p.num_tokens);
  const int n = run_bound(p.keys, i, most, key, true) - i;
  const bool goes_on = i + n < p.num_tokens && p.keys[i + n] == key;
  const bool is_long = !first || goes_on;
  p.pieces[atomicAdd(&p.counts[0], 1)] = make_int2(i, is_long ? n | kPieceOfLong : n);
  if (first && goes_on) p.longs[atomicAdd(&p.counts[1], 1)] = i;
}

// Eight sums to a row of the gradient, as it is typed.
template <bool kFp32, bool kAdd>
__device__ __forceinline__ void write_row(const GradParams& p, uint32_t row, int col, const float (&s)[8]) {
  float v[8];
  const int64_t at = row * p.grad_stride + col;
  if constexpr (kFp32) {
    float4* to = reinterpret_cast<float4*>(static_cast<float*>(p.grad) + at);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
    if constexpr (kAdd) a = to[0], b = to[1];
    const float old[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = kAdd ? old[e] + s[e] * p.scale : s[e] * p.scale;
    to[0] = make_float4(v[0], v[1], v[2], v[3]);
    to[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    if constexpr (kAdd) unpack8(load16(p.grad, at / 8), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = kAdd ? v[e] + s[e] * p.scale : s[e] * p.scale;
    store16(p.grad, at / 8, pack8(v));
  }
}

template <bool kFp32, bool kAdd>
__global__ __launch_bounds__(256) void sum_pieces_kernel(GradParams p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int blocks = (p.hidden + 511) / 512;
  const int64_t units = static_cast<int64_t>(p.counts[0]) * blocks;
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * 4 + wave; u < units; u += static_cast<int64_t>(gridDim.x) * 4) {
    const int2 piece = p.pieces[u / blocks];
    const int col = static_cast<int>(u % blocks) * 512 + 8 * lane;
    const int n = piece.y & (kPieceOfLong - 1);
    const int mine = lane < n ? p.order[piece.x + lane] : 0;
    float s[8] = {};
    for (int j = 0; j < n; ++j) {
      const int64_t t = __builtin_amdgcn_readlane(mine, j);
      if (col < p.hidden) {
        float x[8];
        unpack8(load16(p.dout, t * (p.dout_stride / 8) + col / 8), x);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = s[e] + x[e];
      }
    }
    if (col >= p.hidden) continue;
    const uint32_t row = p.keys[piece.x];
    if (piece.y & kPieceOfLong) {
      const bool first = piece.x == 0 || p.keys[piece.x - 1] != row;
      float4* to = reinterpret_cast<float4*>(p.parts + part_of(piece.x, first) * p.hidden + col);
      to[0] = make_float4(s[0], s[1], s[2], s[3]);
      to[1] = make_float4(s[4], s[5], s[6], s[7]);
    } else {
      write_row<kFp32, kAdd>(p, row, col, s);
    }
  }
}

template <bool kFp32, bool kAdd>
__global__ __launch_bounds__(64) void join_pieces_kernel(GradParams p) {
  const int blocks = (p.hidden + 511) / 512;
  const int64_t units = static_cast<int64_t>(p.counts[1]) * blocks;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int begin = p.longs[u / blocks];
    const int col = static_cast<int>(u % blocks) * 512 + 8 * threadIdx.x;
    const uint32_t row = p.keys[begin];
    const int end = run_bound(p.keys, begin, p.num_tokens, row, true);
    if (col >= p.hidden) continue;
    float s[8] = {};
    for (int i = begin; i < end; i += kPiece) {
      const float4* in = reinterpret_cast<const float4*>(p.parts + part_of(i, i == begin) * p.hidden + col);
      const float4 a = in[0], b = in[1];
      const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = s[e] + x[e];
    }
    write_row<kFp32, kAdd>(p, row, col, s);
  }
}

// Zeros in `pieces` 16-byte pieces of every row.
__global__ __launch_bounds__(256) void zero_rows_kernel(void* grad, int64_t row_pieces, int pieces, int32_t rows) {
  const u32x4 zero = {0, 0, 0, 0};
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int v = threadIdx.x; v < pieces; v += 256) store16(grad, r * row_pieces + v, zero);
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// The workspace's parts, in order.
struct GradSpace {
  size_t keys, order, hist, counts, pieces, longs, parts, total;
  GradSpace(int64_t tokens, int64_t hidden) {
    const int64_t tiles = (tokens + kSortTile - 1) / kSortTile, stretches = (tokens + kPiece - 1) / kPiece;
    keys = 0;
    order = keys + 2 * round256(4 * tokens);
    hist = order + 2 * round256(4 * tokens);
    counts = hist + round256(4 * kBins * tiles);
    pieces = counts + 256;
    longs = pieces + round256(8 * tokens);
    parts = longs + round256(4 * stretches);
    total = parts + round256(2 * stretches * hidden * 4);
  }
};

}  // namespace

hipError_t launch_embedding(const EmbeddingLaunch& a, hipStream_t stream) {
  EmbeddingParams p{a.ids, a.table, a.out, a.table_stride, a.out_stride, a.scale, a.num_tokens, a.vocab, a.hidden_dim, 0};
  return launch_parts((static_cast<int64_t>(a.num_tokens) + kEmbedWaves - 1) / kEmbedWaves, kEmbedWaves * 64,
                      [&](int first, unsigned n) {
                        p.first = first * kEmbedWaves;
                        hipLaunchKernelGGL(embedding_kernel, dim3(n), dim3(kEmbedWaves * 64), 0, stream, p);
                      });
}

size_t embedding_backward_ws_bytes(int64_t num_tokens, int64_t hidden_dim) {
  return GradSpace(num_tokens, hidden_dim).total;
}

hipError_t launch_embedding_backward(const EmbeddingBackwardLaunch& a, hipStream_t stream) {
  const int cus = device_cus();
  const int size = a.grad_fp32 ? 4 : 2;
  if (!a.accumulate) {
    hipLaunchKernelGGL(zero_rows_kernel, dim3(a.vocab < 16 * cus ? a.vocab : 16 * cus), dim3(256), 0, stream, a.grad,
                       a.grad_stride * size / 16, a.hidden_dim * size / 16, a.vocab);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (a.num_tokens == 0) return hipSuccess;
  const GradSpace at(a.num_tokens, a.hidden_dim);
  char* ws = static_cast<char*>(a.workspace);
  const size_t list = round256(4 * static_cast<size_t>(a.num_tokens));
  SortParams s{};
  s.ids = a.ids;
  s.hist = reinterpret_cast<int32_t*>(ws + at.hist);
  s.counts = reinterpret_cast<int32_t*>(ws + at.counts);
  s.num_tokens = a.num_tokens;
  s.vocab = a.vocab;
  s.tiles = (a.num_tokens - 1) / kSortTile + 1;
  int bits = 1;
  while (bits < 31 && (a.vocab >> bits) != 0) ++bits;
  int side = 0;
  for (s.shift = 0; s.shift < bits; s.shift += kDigitBits, side ^= 1) {
    s.keys_in = reinterpret_cast<const uint32_t*>(ws + at.keys + (side ^ 1) * list);
    s.order_in = reinterpret_cast<const int32_t*>(ws + at.order + (side ^ 1) * list);
    s.keys_out = reinterpret_cast<uint32_t*>(ws + at.keys + side * list);
    s.order_out = reinterpret_cast<int32_t*>(ws + at.order + side * list);
    if (s.shift == 0) {
      hipLaunchKernelGGL(sort_count_kernel<true>, dim3(s.tiles), dim3(kSortThreads), 0, stream, s);
      hipLaunchKernelGGL(sort_move_kernel<true>, dim3(s.tiles), dim3(kSortThreads), 0, stream, s);
    } else {
      hipLaunchKernelGGL(sort_count_kernel<false>, dim3(s.tiles), dim3(kSortThreads), 0, stream, s);
      hipLaunchKernelGGL(sort_move_kernel<false>, dim3(s.tiles), dim3(kSortThreads), 0, stream, s);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  GradParams p{};
  p.keys = s.keys_out;
  p.order = s.order_out;
  p.dout = a.dout;
  p.grad = a.grad;
  p.counts = s.counts;
  p.pieces = reinterpret_cast<int2*>(ws + at.pieces);
  p.longs = reinterpret_cast<int32_t*>(ws + at.longs);
  p.parts = reinterpret_cast<float*>(ws + at.parts);
  p.dout_stride = a.dout_stride;
  p.grad_stride = a.grad_stride;
  p.scale = a.scale;
  p.num_tokens = a.num_tokens;
  p.vocab = a.vocab;
  p.hidden = a.hidden_dim;
  hipLaunchKernelGGL(list_pieces_kernel, dim3((a.num_tokens - 1) / 256 + 1), dim3(256), 0, stream, p);
  auto launch = [&](auto fp32, auto add) {
    constexpr bool kFp32 = decltype(fp32)::value, kAdd = decltype(add)::value;
    hipLaunchKernelGGL((sum_pieces_kernel<kFp32, kAdd>), dim3(8 * cus), dim3(256), 0, stream, p);
    hipLaunchKernelGGL((join_pieces_kernel<kFp32, kAdd>), dim3(8 * cus), dim3(64), 0, stream, p);
  };
  if (a.grad_fp32 && a.accumulate)
    launch(std::true_type{}, std::true_type{});
  else if (a.grad_fp32)
    launch(std::true_type{}, std::false_type{});
  else if (a.accumulate)
    launch(std::false_type{}, std::true_type{});
  else
    launch(std::false_type{}, std::false_type{});
  return hipGetLastError();
}

}  // namespace uattn
