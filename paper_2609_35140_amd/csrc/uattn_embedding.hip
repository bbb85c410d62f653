// Embedding lookup, and the gradient of its table by sorted tokens.
//
// Lookup: out[t] = bf16(scale * table[ids[t]]), a wave to a token's row.
//
// Gradient: grad[v] = scale * (sum of dout[t] over the tokens t with ids[t] = v).
// The tokens are sorted by id, stably (a radix sort of up to 9 bits a pass), so that an
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
  // eight pieces of a lane in flight
  constexpr int kAhead = 8;
  for (int v0 = lane; v0 < pieces; v0 += 64 * kAhead) {
    u32x4 w[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      w[u] = u32x4{fill, fill, fill, fill};
      if (known && v0 + 64 * u < pieces) w[u] = load16(p.table, from, v0 + 64 * u);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (v0 + 64 * u >= pieces) break;
      if (known) {
        float x[8];
        unpack8(w[u], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = x[e] * p.scale;
        w[u] = pack8(x);
      }
      store16(p.out, to, v0 + 64 * u, w[u]);
    }
  }
}

// ---------------------------------------------------------------------------
// Sorting, and zeros for the rows without a token beside it
// ---------------------------------------------------------------------------
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;  // of a pass of the sort, at most
constexpr int kPiece = 32;                 // tokens a wave sums
constexpr int kPieceOfLong = 1 << 30;      // of a piece's length: the run is longer than a piece
// Up to kSmall tokens one workgroup sorts them in LDS (a launch instead of five); it takes about as
// long as five small launches there, and runs beside the zeros where these are asked for.
constexpr int kSmall = 16384, kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64;
constexpr int kSmallRounds = kSmall / kSmallThreads;
constexpr int kTileThreads = 512, kTileWaves = kTileThreads / 64;
constexpr int kTile = 2048, kTileRounds = kTile / kTileThreads;

// The zeros of a launch: rows [begin, end) of the gradient that no id names, 16-byte pieces.
struct ZeroParams {
  void* grad;
  const int32_t* ids;
  int64_t row_pieces;  // from row to row
  int32_t pieces;      // of a row
  int32_t num_tokens, begin, end;
  int32_t sorters;     // workgroups of the launch that sort; the others write zeros
};

// By a workgroup of kThreads threads, the `part`-th of `parts`: it marks the rows of its share that have
// a token and clears the others.
template <int kThreads>
__device__ __forceinline__ void zero_rows(const ZeroParams& z, int part, int parts, uint32_t* marks) {
  constexpr int kRows = 4096;  // marked at a time
  const int64_t rows = z.end - z.begin;
  const int64_t first = z.begin + rows * part / parts, last = z.begin + rows * (part + 1) / parts;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t r0 = first; r0 < last; r0 += kRows) {
    const uint32_t n = static_cast<uint32_t>(last - r0 < kRows ? last - r0 : kRows);
    for (int i = threadIdx.x; i < kRows / 32; i += kThreads) marks[i] = 0;
    __syncthreads();
    constexpr int kAhead = 8;
    for (int64_t i0 = threadIdx.x; i0 < z.num_tokens; i0 += kAhead * kThreads) {
      int32_t id[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) id[u] = i0 + u * kThreads < z.num_tokens ? z.ids[i0 + u * kThreads] : -1;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const uint32_t r = static_cast<uint32_t>(id[u]) - static_cast<uint32_t>(r0);
        if (r < n) atomicOr(&marks[r / 32], 1u << (r & 31));
      }
    }
    __syncthreads();
    for (uint32_t r = wave; r < n; r += kThreads / 64) {
      if (marks[r / 32] >> (r & 31) & 1) continue;
      for (int v = lane; v < z.pieces; v += 64) store16(z.grad, (r0 + r) * z.row_pieces, v, u32x4{0, 0, 0, 0});
    }
    __syncthreads();
  }
}

// Ids outside [0, vocab) have no row: they sort behind all others.
__device__ __forceinline__ uint32_t sort_key(int32_t id, int32_t vocab) {
  return static_cast<uint32_t>(id >= 0 && id < vocab ? id : vocab);
}

// The lanes of the wave whose digit is this lane's.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool valid, int bits) {
  uint64_t same = __ballot(valid);
#pragma unroll
  for (int b = 0; b < kDigitBits; ++b) {
    if (b >= bits) break;
    const uint64_t set = __ballot(digit >> b & 1);
    same &= digit >> b & 1 ? set : ~set;
  }
  return same;
}

// How many of the wave's tokens of this digit came before, in rounds of 64: `seen` counts them.
__device__ __forceinline__ int rank_in_wave(int32_t* seen, uint32_t digit, bool valid, int bits, int lane) {
  const uint64_t same = same_digit(digit, valid, bits);
  const int rank = __popcll(same & ((uint64_t{1} << lane) - 1));
  int at = 0;
  if (valid && rank == 0) at = atomicAdd(&seen[digit], __popcll(same));
  return __shfl(at, same != 0 ? __ffsll(static_cast<unsigned long long>(same)) - 1 : 0, 64) + rank;
}

// Exclusive sums of kBins values held one to a thread by the first kBins threads of the workgroup; all
// of it passes the barrier.
__device__ __forceinline__ int32_t scan_bins(int32_t x, int32_t* wave_totals) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t s = x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int32_t y = __shfl_up(s, d, 64);
    if (lane >= d) s += y;
  }
  if (lane == 63 && wave < kBins / 64) wave_totals[wave] = s;
  __syncthreads();
  int32_t before = 0;
#pragma unroll
  for (int w = 0; w < kBins / 64; ++w)
    if (w < wave) before += wave_totals[w];
  return before + s - x;
}

// The first position in [lo, hi) whose key is above `key - !after`: the run's start or its end.
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

// Whether sorted position i begins a piece (a multiple of kPiece behind its run's start), its length
// with kPieceOfLong, and whether it is the first of a run of several.
struct PieceAt {
  int length;  // 0: no piece begins here
  bool first_of_long;
};
__device__ __forceinline__ PieceAt piece_at(const uint32_t* keys, int num_tokens, int32_t vocab, int i) {
  const uint32_t key = keys[i];
  if (key >= static_cast<uint32_t>(vocab)) return {0, false};
  const bool first = i == 0 || keys[i - 1] != key;
  if (!first) {
    if (i < kPiece || keys[i - kPiece] != key) return {0, false};
    if ((i - run_bound(keys, 0, i, key, false)) % kPiece != 0) return {0, false};
  }
  const int n = run_bound(keys, i, min(i + kPiece, num_tokens), key, true) - i;
  const bool goes_on = i + n < num_tokens && keys[i + n] == key;
  return {!first || goes_on ? n | kPieceOfLong : n, first && goes_on};
}

struct SortParams {
  const int32_t* ids;            // the first pass reads these, the others keys_in and order_in
  const uint32_t* keys_in;
  const int32_t* order_in;
  uint32_t* keys_out;
  int32_t* order_out;
  int32_t* hist;                 // [tiles][kBins]
  int32_t* counts;               // pieces, runs of several
  int2* pieces;                  // first sorted position, tokens (| kPieceOfLong)
  int32_t* longs;                // first sorted position
  int32_t num_tokens, vocab, tiles, shift, bits;  // of the digit
  int32_t passes;
  ZeroParams zero;
};

// All passes and the list of pieces for up to kSmall tokens, by workgroup 0.  A wave's tokens are
// consecutive, 64 to a round; in a pass each gets its place among the wave's of its digit, the counts
// of (digit, wave) are summed, and the tokens move.
__global__ __launch_bounds__(kSmallThreads) void sort_small_kernel(SortParams p) {
  __shared__ uint32_t keys[kSmall];
  __shared__ uint16_t order[kSmall];
  __shared__ int32_t seen[kSmallWaves][kBins];
  __shared__ int32_t base[kBins], wave_totals[kBins / 64], counts[2];
  if (static_cast<int>(blockIdx.x) >= p.zero.sorters) {
    zero_rows<kSmallThreads>(p.zero, blockIdx.x - p.zero.sorters, gridDim.x - p.zero.sorters, keys);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rounds = (p.num_tokens + kSmallThreads - 1) / kSmallThreads, begin = wave * rounds * 64 + lane;
  uint32_t key[kSmallRounds];
  int32_t from[kSmallRounds], at[kSmallRounds];
#pragma unroll
  for (int r = 0; r < kSmallRounds; ++r) {
    from[r] = begin + r * 64;
    key[r] = r < rounds && from[r] < p.num_tokens ? sort_key(p.ids[from[r]], p.vocab) : 0;
  }
  if (tid < 2) counts[tid] = 0;
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.bits;
    const uint32_t low = (1u << p.bits) - 1;
    for (int i = tid; i < kSmallWaves * kBins; i += kSmallThreads) seen[0][i] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r)
      if (r < rounds) at[r] = rank_in_wave(seen[wave], key[r] >> shift & low, begin + r * 64 < p.num_tokens, p.bits, lane);
    __syncthreads();
    int32_t all = 0;
    if (tid < kBins)
      for (int w = 0; w < kSmallWaves; ++w) {
        const int32_t n = seen[w][tid];
        seen[w][tid] = all;
        all += n;
      }
    const int32_t before = scan_bins(all, wave_totals);
    if (tid < kBins) base[tid] = before;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r) {
      if (r >= rounds || begin + r * 64 >= p.num_tokens) continue;
      const uint32_t digit = key[r] >> shift & low;
      const int to = base[digit] + seen[wave][digit] + at[r];
      keys[to] = key[r];
      order[to] = static_cast<uint16_t>(from[r]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSmallRounds; ++r) {
      const int i = begin + r * 64;
      if (r >= rounds || i >= p.num_tokens) continue;
      key[r] = keys[i];
      from[r] = order[i];
    }
  }
  for (int i = tid; i < p.num_tokens; i += kSmallThreads) {
    p.keys_out[i] = keys[i];
    p.order_out[i] = order[i];
    const PieceAt piece = piece_at(keys, p.num_tokens, p.vocab, i);
    if (piece.length != 0) p.pieces[atomicAdd(&counts[0], 1)] = make_int2(i, piece.length);
    if (piece.first_of_long) p.longs[atomicAdd(&counts[1], 1)] = i;
  }
  __syncthreads();
  if (tid < 2) p.counts[tid] = counts[tid];
}

template <bool kFirst>
__device__ __forceinline__ uint32_t key_at(const SortParams& p, int i) {
  return kFirst ? sort_key(p.ids[i], p.vocab) : p.keys_in[i];
}

// How often each digit occurs in a tile.
template <bool kFirst>
__global__ __launch_bounds__(kTileThreads) void sort_count_kernel(SortParams p) {
  __shared__ int32_t count[kBins];
  if (static_cast<int>(blockIdx.x) >= p.zero.sorters) {
    zero_rows<kTileThreads>(p.zero, blockIdx.x - p.zero.sorters, gridDim.x - p.zero.sorters, reinterpret_cast<uint32_t*>(count));
    return;
  }
  const int tid = threadIdx.x;
  if (kFirst && blockIdx.x == 0 && tid < 2) p.counts[tid] = 0;
  count[tid] = 0;
  __syncthreads();
  const int begin = blockIdx.x * kTile;
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const int i = begin + r * kTileThreads + tid;
    if (i < p.num_tokens) atomicAdd(&count[key_at<kFirst>(p, i) >> p.shift & ((1u << p.bits) - 1)], 1);
  }
  __syncthreads();
  p.hist[static_cast<int64_t>(blockIdx.x) * kBins + tid] = count[tid];
}

// Moves a tile's tokens behind the smaller digits of all tiles and the equal ones of the tiles before.
template <bool kFirst>
__global__ __launch_bounds__(kTileThreads) void sort_move_kernel(SortParams p) {
  __shared__ int32_t seen[kTileWaves][kBins];
  __shared__ int32_t wave_totals[kBins / 64];
  if (static_cast<int>(blockIdx.x) >= p.zero.sorters) {
    zero_rows<kTileThreads>(p.zero, blockIdx.x - p.zero.sorters, gridDim.x - p.zero.sorters, reinterpret_cast<uint32_t*>(seen));
    return;
  }
  static_assert(kTileThreads == kBins, "a thread to a digit");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int begin = blockIdx.x * kTile + wave * kTileRounds * 64 + lane;
  const uint32_t low = (1u << p.bits) - 1;
  uint32_t key[kTileRounds];
  int32_t from[kTileRounds], at[kTileRounds];
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    const int i = begin + r * 64;
    key[r] = 0;
    from[r] = i;
    if (i >= p.num_tokens) continue;
    key[r] = key_at<kFirst>(p, i);
    if (!kFirst) from[r] = p.order_in[i];
  }
  for (int w = 0; w < kTileWaves; ++w) seen[w][tid] = 0;
  // of this thread's digit: all its tokens, and those in the tiles before this one
  int32_t all = 0, earlier = 0;
  constexpr int kAhead = 8;
  for (int t0 = 0; t0 < p.tiles; t0 += kAhead) {
    int32_t n[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) n[u] = t0 + u < p.tiles ? p.hist[static_cast<int64_t>(t0 + u) * kBins + tid] : 0;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      all += n[u];
      if (t0 + u < static_cast<int>(blockIdx.x)) earlier += n[u];
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r)
    at[r] = rank_in_wave(seen[wave], key[r] >> p.shift & low, begin + r * 64 < p.num_tokens, p.bits, lane);
  int32_t place = scan_bins(all, wave_totals) + earlier;
  for (int w = 0; w < kTileWaves; ++w) {
    const int32_t n = seen[w][tid];
    seen[w][tid] = place;
    place += n;
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < kTileRounds; ++r) {
    if (begin + r * 64 >= p.num_tokens) continue;
    const int to = seen[wave][key[r] >> p.shift & low] + at[r];
    p.keys_out[to] = key[r];
    p.order_out[to] = from[r];
  }
}

// Lists the pieces of sorted tokens.
__global__ __launch_bounds__(kTileThreads) void list_pieces_kernel(SortParams p) {
  __shared__ uint32_t marks[4096 / 32];
  if (static_cast<int>(blockIdx.x) >= p.zero.sorters) {
    zero_rows<kTileThreads>(p.zero, blockIdx.x - p.zero.sorters, gridDim.x - p.zero.sorters, marks);
    return;
  }
  const int i = blockIdx.x * kTileThreads + threadIdx.x;
  if (i >= p.num_tokens) return;
  const PieceAt piece = piece_at(p.keys_out, p.num_tokens, p.vocab, i);
  if (piece.length != 0) p.pieces[atomicAdd(&p.counts[0], 1)] = make_int2(i, piece.length);
  if (piece.first_of_long) p.longs[atomicAdd(&p.counts[1], 1)] = i;
}

// ---------------------------------------------------------------------------
// Sums
// ---------------------------------------------------------------------------
struct GradParams {
  const uint32_t* keys;   // sorted
  const int32_t* order;
  const void* dout;
  void* grad;
  const int32_t* counts;  // pieces, runs of several
  const int2* pieces;     // first sorted position, tokens (| kPieceOfLong)
  const int32_t* longs;   // first sorted position
  float* parts;           // [2 * ceil(T / kPiece)][hidden]
  int64_t dout_stride, grad_stride;
  float scale;
  int32_t num_tokens, vocab, hidden;
};

// Of the pieces of runs longer than one: at most one first piece, and at most one later one, starts in
// any kPiece positions (the run between two first ones is longer, and a later piece starts that far
// behind its predecessor), so the two places of a stretch are never shared.
__device__ __forceinline__ int64_t part_of(int position, bool first) { return 2 * static_cast<int64_t>(position / kPiece) + (first ? 0 : 1); }

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

// A wave to a piece and 512 columns, eight of the piece's rows in flight, added in order.
template <bool kFp32, bool kAdd>
__global__ __launch_bounds__(256) void sum_pieces_kernel(GradParams p) {
  constexpr int kAhead = 8;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int blocks = (p.hidden + 511) / 512;
  const int64_t units = static_cast<int64_t>(p.counts[0]) * blocks;
  for (int64_t u = static_cast<int64_t>(blockIdx.x) * 4 + wave; u < units; u += static_cast<int64_t>(gridDim.x) * 4) {
    const int2 piece = p.pieces[u / blocks];
    const int col = static_cast<int>(u % blocks) * 512 + 8 * lane;
    const int n = __builtin_amdgcn_readfirstlane(piece.y & (kPieceOfLong - 1));
    const int mine = lane < n ? p.order[piece.x + lane] : 0;
    const bool here = col < p.hidden;
    float s[8] = {};
    for (int j0 = 0; j0 < n; j0 += kAhead) {
      u32x4 w[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        w[j] = u32x4{0, 0, 0, 0};
        if (j0 + j >= n) continue;
        const int64_t t = __builtin_amdgcn_readlane(mine, j0 + j);
        if (here) w[j] = load16(p.dout, t * (p.dout_stride / 8), col / 8);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (j0 + j >= n) break;
        float x[8];
        unpack8(w[j], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = s[e] + x[e];
      }
    }
    if (!here) continue;
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

// Adds the pieces of runs of several, in order.
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
    constexpr int kAhead = 4;
    float s[8] = {};
    for (int i0 = begin; i0 < end; i0 += kAhead * kPiece) {
      float4 q[kAhead][2];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int i = i0 + j * kPiece;
        q[j][0] = q[j][1] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i >= end) continue;
        const float4* in = reinterpret_cast<const float4*>(p.parts + part_of(i, i == begin) * p.hidden + col);
        q[j][0] = in[0];
        q[j][1] = in[1];
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (i0 + j * kPiece >= end) break;
        const float x[8] = {q[j][0].x, q[j][0].y, q[j][0].z, q[j][0].w, q[j][1].x, q[j][1].y, q[j][1].z, q[j][1].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = s[e] + x[e];
      }
    }
    write_row<kFp32, kAdd>(p, row, col, s);
  }
}

// Zeros alone, for no tokens.
__global__ __launch_bounds__(kTileThreads) void zero_rows_kernel(ZeroParams z) {
  __shared__ uint32_t marks[4096 / 32];
  zero_rows<kTileThreads>(z, blockIdx.x, gridDim.x, marks);
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// The workspace's parts, in order.
struct GradSpace {
  size_t keys, order, hist, counts, pieces, longs, parts, total;
  GradSpace(int64_t tokens, int64_t hidden) {
    const int64_t tiles = (tokens + kTile - 1) / kTile, stretches = (tokens + kPiece - 1) / kPiece;
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
  ZeroParams z{};
  z.grad = a.grad;
  z.ids = a.ids;
  z.row_pieces = a.grad_stride * size / 16;
  z.pieces = a.hidden_dim * size / 16;
  z.num_tokens = a.num_tokens;
  // workgroups that write zeros beside `sorters` that sort, `threads` each: all CUs' threads
  auto zeroers = [&](int threads) {
    const int64_t rows = z.end - z.begin, most = static_cast<int64_t>(cus) * 2048 / threads;
    return static_cast<unsigned>(rows < most ? rows : most);
  };
  if (a.num_tokens == 0) {
    z.end = a.vocab;
    hipLaunchKernelGGL(zero_rows_kernel, dim3(zeroers(kTileThreads)), dim3(kTileThreads), 0, stream, z);
    return hipGetLastError();
  }
  const GradSpace at(a.num_tokens, a.hidden_dim);
  char* ws = static_cast<char*>(a.workspace);
  const size_t list = round256(4 * static_cast<size_t>(a.num_tokens));
  SortParams s{};
  s.ids = a.ids;
  s.hist = reinterpret_cast<int32_t*>(ws + at.hist);
  s.counts = reinterpret_cast<int32_t*>(ws + at.counts);
  s.pieces = reinterpret_cast<int2*>(ws + at.pieces);
  s.longs = reinterpret_cast<int32_t*>(ws + at.longs);
  s.num_tokens = a.num_tokens;
  s.vocab = a.vocab;
  s.tiles = (a.num_tokens - 1) / kTile + 1;
  int bits = 1;  // of a key, vocab the largest
  while (bits < 31 && (a.vocab >> bits) != 0) ++bits;
  s.passes = (bits + kDigitBits - 1) / kDigitBits;
  s.bits = (bits + s.passes - 1) / s.passes;
  // the rows to clear are shared out over the launches of the sort
  const int launches = a.num_tokens <= kSmall ? 1 : 2 * s.passes + 1;
  int done = 0;
  auto launch = [&](auto kernel, int sorters, int threads) {
    unsigned grid = sorters;
    s.zero = z;
    s.zero.sorters = sorters;
    if (!a.accumulate) {
      z.begin = static_cast<int32_t>(static_cast<int64_t>(a.vocab) * done / launches);
      z.end = static_cast<int32_t>(static_cast<int64_t>(a.vocab) * (done + 1) / launches);
      s.zero.begin = z.begin;
      s.zero.end = z.end;
      grid += zeroers(threads);
    }
    ++done;
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), 0, stream, s);
    return hipGetLastError();
  };
  auto buffers = [&](int side) {
    s.keys_in = reinterpret_cast<const uint32_t*>(ws + at.keys + (side ^ 1) * list);
    s.order_in = reinterpret_cast<const int32_t*>(ws + at.order + (side ^ 1) * list);
    s.keys_out = reinterpret_cast<uint32_t*>(ws + at.keys + side * list);
    s.order_out = reinterpret_cast<int32_t*>(ws + at.order + side * list);
  };
  hipError_t e = hipSuccess;
  if (a.num_tokens <= kSmall) {
    buffers(0);
    e = launch(sort_small_kernel, 1, kSmallThreads);
  } else {
    for (int pass = 0; pass < s.passes && e == hipSuccess; ++pass) {
      buffers(pass & 1);
      s.shift = pass * s.bits;
      e = pass == 0 ? launch(sort_count_kernel<true>, s.tiles, kTileThreads) : launch(sort_count_kernel<false>, s.tiles, kTileThreads);
      if (e == hipSuccess)
        e = pass == 0 ? launch(sort_move_kernel<true>, s.tiles, kTileThreads) : launch(sort_move_kernel<false>, s.tiles, kTileThreads);
    }
    if (e == hipSuccess) e = launch(list_pieces_kernel, (a.num_tokens - 1) / kTileThreads + 1, kTileThreads);
  }
  if (e != hipSuccess) return e;
  GradParams p{};
  p.keys = s.keys_out;
  p.order = s.order_out;
  p.dout = a.dout;
  p.grad = a.grad;
  p.counts = s.counts;
  p.pieces = s.pieces;
  p.longs = s.longs;
  p.parts = reinterpret_cast<float*>(ws + at.parts);
  p.dout_stride = a.dout_stride;
  p.grad_stride = a.grad_stride;
  p.scale = a.scale;
  p.num_tokens = a.num_tokens;
  p.vocab = a.vocab;
  p.hidden = a.hidden_dim;
  const int64_t units = static_cast<int64_t>(a.num_tokens) * ((a.hidden_dim + 511) / 512);
  const int64_t sum_grid = (units + 3) / 4 < 8 * cus ? (units + 3) / 4 : 8 * cus;
  const int64_t join_grid = units / kPiece + 1 < 16 * cus ? units / kPiece + 1 : 16 * cus;
  auto sums = [&](auto fp32, auto add) {
    constexpr bool kFp32 = decltype(fp32)::value, kAdd = decltype(add)::value;
    hipLaunchKernelGGL((sum_pieces_kernel<kFp32, kAdd>), dim3(sum_grid), dim3(256), 0, stream, p);
    if (a.num_tokens > kPiece)
      hipLaunchKernelGGL((join_pieces_kernel<kFp32, kAdd>), dim3(join_grid), dim3(64), 0, stream, p);
  };
  if (a.grad_fp32 && a.accumulate)
    sums(std::true_type{}, std::true_type{});
  else if (a.grad_fp32)
    sums(std::true_type{}, std::false_type{});
  else if (a.accumulate)
    sums(std::false_type{}, std::true_type{});
  else
    sums(std::false_type{}, std::false_type{});
  return hipGetLastError();
}

}  // namespace uattn
