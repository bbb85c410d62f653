// Embedding lookup, and the gradient of its table by sorted tokens.
//
// Lookup: out[t] = bf16(scale * table[ids[t]]), a wave to a token's row.
//
// Gradient: grad[v] = scale * (sum of dout[t] over the tokens t with ids[t] = v).
// The tokens are sorted by id, stably, so that an entry's tokens stand together and in
// ascending order.  An entry's run is cut
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
  bool stream;    // the output past the caches
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
      store16_as(p.stream, p.out, to, v0 + 64 * u, w[u]);
    }
  }
}

// ---------------------------------------------------------------------------
// Sorting, and zeros for the table beside it
// ---------------------------------------------------------------------------
constexpr int kDigitBits = 9, kBins = 1 << kDigitBits;  // of a pass of a radix sort, at most
constexpr int kPiece = 32;                 // tokens a wave sums
// Up to kSmall tokens are sorted in one launch, by kBuckets workgroups in LDS: the b-th takes the ids
// v with v % kBuckets = b, so that frequent neighbours are spread.  (16,000 tokens: 62 us by one workgroup,
// 18 by 64; the launches for more tokens take about 35, whatever their number up to 65,536.)
constexpr int kSmall = 16384, kSmallThreads = 1024, kSmallWaves = kSmallThreads / 64, kBuckets = 64;
constexpr int kSmallRounds = kSmall / kSmallThreads;
constexpr int kTileThreads = 512, kTileWaves = kTileThreads / 64;
constexpr int kTile = 2048, kTileRounds = kTile / kTileThreads;

// The zeros of a launch: rows [begin, end) of the gradient, 16-byte pieces.  Rows that have tokens are
// cleared too: to find the others, every workgroup would read all ids, which costs about as much.
struct ZeroParams {
  void* grad;
  int64_t row_pieces;  // from row to row
  int32_t pieces;      // of a row
  int32_t begin, end;
  int32_t sorters;     // workgroups of the launch that sort; the others write zeros
};

// By a workgroup of kThreads threads, the `part`-th of `parts`, a wave to a row.
template <int kThreads>
__device__ __forceinline__ void zero_rows(const ZeroParams& z, int part, int parts) {
  constexpr int kWaves = kThreads / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  for (int64_t r = z.begin + static_cast<int64_t>(part) * kWaves + wave; r < z.end; r += static_cast<int64_t>(parts) * kWaves)
    for (int v = lane; v < z.pieces; v += 64) store16(z.grad, r * z.row_pieces, v, u32x4{0, 0, 0, 0});
}

// Ids outside [0, vocab) have no row: they sort behind all others.
__device__ __forceinline__ uint32_t sort_key(int32_t id, int32_t vocab) {
  return static_cast<uint32_t>(id >= 0 && id < vocab ? id : vocab);
}

// The lanes of the wave whose digit is this lane's.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool valid, int bits) {
  uint64_t same = __ballot(valid);
  for (int b = 0; b < bits; ++b) {
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

// The first of the `n` ascending keys that is not below `key`, by a wave: 64 probes a step.
__device__ __forceinline__ int wave_lower_bound(const uint32_t* keys, int n, uint32_t key) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 0) {
    const int step = (n + 63) / 64, at = lane * step;
    const int below = __popcll(__ballot(at < n && keys[lo + at] < key));
    if (below == 0) return lo;
    lo += (below - 1) * step + 1;
    n = min(step - 1, n - (below - 1) * step - 1);
  }
  return lo;
}

// A piece: what one wave sums over 512 columns.
struct Piece {
  int32_t at;      // its first sorted position
  int32_t tokens;  // up to kPiece, with the marks below
  uint32_t row;    // of the gradient
  int32_t token;   // the first
};
constexpr int kOfLong = 1 << 30;   // its run is longer than a piece: the sum is a part
constexpr int kFirst = 1 << 29;    // ... the run's first
struct LongRun {
  int32_t begin, end;  // sorted positions
  uint32_t row;
};

// Lists the pieces that begin at the wave's 64 sorted positions i0 + lane of `n`, whose keys ascend up to
// `limit` (keys from there on have no row): every position a multiple of kPiece behind its run's start.
// order(i) and row(key) name position i's token and a key's row; sorted positions count from `base` on in the lists.
// pieces and longs are counted in counts[0] and counts[1].
template <class Order, class Row>
__device__ __forceinline__ void list_pieces(const uint32_t* keys, int n, uint32_t limit, int i0, int base, const Order& order,
                                            const Row& row, int32_t* counts, Piece* pieces, LongRun* longs) {
  const int lane = threadIdx.x & 63, i = i0 + lane;
  // the starts of runs at the positions from i0 on: 64, and 32 behind them (positions from n on count as starts)
  const uint32_t key = i < n ? keys[i] : limit;
  const bool start = i >= n || i == 0 || keys[i - 1] != key;
  const uint64_t starts = __ballot(start);
  const int j = i0 + 64 + lane;
  const uint64_t behind = __ballot(lane < kPiece + 1 && (j >= n || keys[j - 1] != keys[j]));
  // the run of the positions before the wave's first start
  int before = i0;
  if ((starts & 1) == 0) {
    const uint32_t first = __builtin_amdgcn_readfirstlane(key);
    before = wave_lower_bound(keys, i0, first);
  }
  const uint64_t until = starts & (~uint64_t{0} >> (63 - lane));  // starts at this lane or before
  const int begin = until != 0 ? i0 + 63 - __clzll(static_cast<long long>(until)) : before;
  if (i >= n || key >= limit || (i - begin) % kPiece != 0) return;
  // positions to the next start, up to kPiece + 1
  const uint64_t later = lane == 63 ? behind : (starts >> (lane + 1)) | (behind << (63 - lane));
  const int run = later != 0 ? __ffsll(static_cast<unsigned long long>(later)) : kPiece + 1;
  const bool goes_on = run > kPiece, is_first = i == begin;
  int tokens = goes_on ? kPiece : run;
  if (goes_on || !is_first) tokens |= kOfLong | (is_first ? kFirst : 0);
  pieces[atomicAdd(&counts[0], 1)] = Piece{base + i, tokens, row(key), order(i)};
  // the run's last piece names the run
  if (!goes_on && !is_first) longs[atomicAdd(&counts[1], 1)] = LongRun{base + begin, base + i + run, row(key)};
}

// The lists have a part to a bucket (all in the first where there are none): its pieces begin at the
// bucket's first sorted position, its long runs at a kPiece-th of it (they are longer than kPiece).
struct ListHeads {
  int32_t pieces[kBuckets], longs[kBuckets], base[kBuckets];
};

// The lists' parts as a wave reads them: lane b keeps the b-th's.
struct ListParts {
  int32_t until, count, base;
  __device__ __forceinline__ ListParts(const int32_t* counts, const int32_t* bases, int divide) {
    const int lane = threadIdx.x & 63;
    static_assert(kBuckets == 64, "a lane to a part");
    count = counts[lane];
    base = bases[lane] / divide;
    until = count;
#pragma unroll
    for (int d = 1; d < kBuckets; d *= 2) {
      const int32_t y = __shfl_up(until, d, 64);
      if (lane >= d) until += y;
    }
  }
  __device__ __forceinline__ int total() const { return __builtin_amdgcn_readlane(until, kBuckets - 1); }
  // where the k-th entry of all stands
  __device__ __forceinline__ int at(int k) const {
    const int b = __popcll(__ballot(until <= k));
    return k - __builtin_amdgcn_readlane(until, b) + __builtin_amdgcn_readlane(count, b) + __builtin_amdgcn_readlane(base, b);
  }
};

// Walks (entry, block of 512 columns) pairs, entries outside, `step` pairs at a time, without divisions.
struct PairWalk {
  int32_t entry, block, blocks, entry_step, block_step;
  __device__ __forceinline__ PairWalk(int32_t first, int32_t step, int32_t columns) {
    blocks = (columns + 511) / 512;
    entry = first / blocks;
    block = first % blocks;
    entry_step = step / blocks;
    block_step = step % blocks;
  }
  __device__ __forceinline__ void go_on() {
    entry += entry_step;
    block += block_step;
    if (block >= blocks) {
      block -= blocks;
      ++entry;
    }
  }
};

struct SortParams {
  const int32_t* ids;            // the first pass reads these, the others keys_in and order_in
  const uint32_t* keys_in;
  const int32_t* order_in;
  uint32_t* keys_out;
  int32_t* order_out;
  int32_t* hist;                 // [tiles + 1][kBins]; of many tiles, summed: before the tile, and of all behind the last
  ListHeads* heads;
  Piece* pieces;
  LongRun* longs;
  int32_t num_tokens, vocab, tiles, shift, bits;  // of the digit
  int32_t passes;
  ZeroParams zero;
};

// A bucket of up to kSmall tokens, sorted and listed.  A wave's tokens are consecutive, 64 to a round; in
// a pass each gets its place among the wave's of its digit, the counts of (digit, wave) are summed, and
// the tokens move.
__global__ __launch_bounds__(kSmallThreads) void sort_small_kernel(SortParams p) {
  extern __shared__ __align__(16) uint32_t keys[];  // [num_tokens] and as many 16-bit orders
  __shared__ int32_t seen[kSmallWaves][kBins];
  __shared__ int32_t first_of[kBins], wave_totals[kBins / 64], mine_of[kSmallWaves], before_of[kSmallWaves], counts[2];
  if (static_cast<int>(blockIdx.x) >= p.zero.sorters) {
    zero_rows<kSmallThreads>(p.zero, blockIdx.x - p.zero.sorters, gridDim.x - p.zero.sorters);
    return;
  }
  uint16_t* order = reinterpret_cast<uint16_t*>(keys + p.num_tokens);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint64_t below = (uint64_t{1} << lane) - 1;  // the lanes before this one
  int rounds = (p.num_tokens + kSmallThreads - 1) / kSmallThreads, begin = wave * rounds * 64 + lane;
  uint32_t key[kSmallRounds];
  int32_t from[kSmallRounds], at[kSmallRounds];
  // the bucket's tokens, in order, and the number of tokens in the buckets before it
  int mine = 0, before = 0;
#pragma unroll
  for (int r = 0; r < kSmallRounds; ++r) {
    key[r] = p.vocab;
    if (r < rounds && begin + r * 64 < p.num_tokens) key[r] = sort_key(p.ids[begin + r * 64], p.vocab);
  }
  for (int r = 0; r < rounds; ++r) {
    const bool valid = key[r] < static_cast<uint32_t>(p.vocab);
    mine += __popcll(__ballot(valid && key[r] % kBuckets == blockIdx.x));
    before += __popcll(__ballot(valid && key[r] % kBuckets < blockIdx.x));
  }
  if (lane == 0) {
    mine_of[wave] = mine;
    before_of[wave] = before;
  }
  if (tid < 2) counts[tid] = 0;
  __syncthreads();
  int n = 0, base = 0, to = 0;
#pragma unroll
  for (int w = 0; w < kSmallWaves; ++w) {
    if (w == wave) to = n;
    n += mine_of[w];
    base += before_of[w];
  }
  for (int r = 0; r < rounds; ++r) {
    const bool here = key[r] < static_cast<uint32_t>(p.vocab) && key[r] % kBuckets == blockIdx.x;
    const uint64_t all = __ballot(here);
    if (here) {
      keys[to + __popcll(all & below)] = key[r] / kBuckets;
      order[to + __popcll(all & below)] = static_cast<uint16_t>(begin + r * 64);
    }
    to += __popcll(all);
  }
  rounds = (n + kSmallThreads - 1) / kSmallThreads;
  begin = wave * rounds * 64 + lane;
  for (int pass = 0; pass < p.passes; ++pass) {
    const int shift = pass * p.bits, bins = 1 << p.bits;
    const uint32_t low = bins - 1;
    for (int i = tid; i < kSmallWaves * kBins; i += kSmallThreads) seen[0][i] = 0;
    __syncthreads();
    for (int r = 0; r < rounds; ++r) {
      const int i = begin + r * 64;
      key[r] = i < n ? keys[i] : 0;
      from[r] = i < n ? order[i] : 0;
      at[r] = rank_in_wave(seen[wave], key[r] >> shift & low, i < n, p.bits, lane);
    }
    __syncthreads();
    int32_t all = 0;
    if (tid < bins)
      for (int w = 0; w < kSmallWaves; ++w) {
        const int32_t c = seen[w][tid];
        seen[w][tid] = all;
        all += c;
      }
    const int32_t smaller = scan_bins(all, wave_totals);
    if (tid < kBins) first_of[tid] = smaller;
    __syncthreads();
    for (int r = 0; r < rounds; ++r) {
      if (begin + r * 64 >= n) break;
      const uint32_t digit = key[r] >> shift & low;
      const int place = first_of[digit] + seen[wave][digit] + at[r];
      keys[place] = key[r];
      order[place] = static_cast<uint16_t>(from[r]);
    }
    __syncthreads();
  }
  for (int i = tid; i < n; i += kSmallThreads) p.order_out[base + i] = order[i];
  for (int i0 = wave * 64; i0 < n; i0 += kSmallThreads)
    list_pieces(
        keys, n, ~0u, i0, base, [&](int i) { return static_cast<int32_t>(order[i]); },
        [&](uint32_t k) { return k * kBuckets + blockIdx.x; }, counts, p.pieces + base, p.longs + base / kPiece);
  __syncthreads();
  if (tid == 0) {
    p.heads->pieces[blockIdx.x] = counts[0];
    p.heads->longs[blockIdx.x] = counts[1];
    p.heads->base[blockIdx.x] = base;
  }
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
    zero_rows<kTileThreads>(p.zero, blockIdx.x - p.zero.sorters, gridDim.x - p.zero.sorters);
    return;
  }
  const int tid = threadIdx.x;
  if (kFirst && blockIdx.x == 0 && tid < static_cast<int>(sizeof(ListHeads) / 4)) reinterpret_cast<int32_t*>(p.heads)[tid] = 0;
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

// Up to kManyTiles every workgroup sums the digits' counts of all tiles for itself; past them, where that
// grows with the square of the tiles, a launch does it for all: each digit's counts become those of the tiles
// before.  (256 tiles of 2048 tokens: a pass takes 30 us so, and 18 + 12 with the launch.)
constexpr int kManyTiles = 256;

__global__ __launch_bounds__(64) void sum_tiles_kernel(int32_t* hist, int32_t tiles) {
  int32_t* at = hist + blockIdx.x * 64 + threadIdx.x;
  constexpr int kAhead = 16;
  int32_t sum = 0;
  for (int32_t t0 = 0; t0 < tiles; t0 += kAhead) {
    int32_t n[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) n[u] = t0 + u < tiles ? at[static_cast<int64_t>(t0 + u) * kBins] : 0;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (t0 + u < tiles) at[static_cast<int64_t>(t0 + u) * kBins] = sum;
      sum += n[u];
    }
  }
  at[static_cast<int64_t>(tiles) * kBins] = sum;
}

// Moves a tile's tokens behind the smaller digits of all tiles and the equal ones of the tiles before.
template <bool kFirst>
__global__ __launch_bounds__(kTileThreads) void sort_move_kernel(SortParams p) {
  __shared__ int32_t seen[kTileWaves][kBins];
  __shared__ int32_t wave_totals[kBins / 64];
  if (static_cast<int>(blockIdx.x) >= p.zero.sorters) {
    zero_rows<kTileThreads>(p.zero, blockIdx.x - p.zero.sorters, gridDim.x - p.zero.sorters);
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
  if (p.tiles > kManyTiles) {
    earlier = p.hist[static_cast<int64_t>(blockIdx.x) * kBins + tid];
    all = p.hist[static_cast<int64_t>(p.tiles) * kBins + tid];
  } else {
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

// Lists the pieces of sorted tokens, a wave to 64 of them; the lists follow no order (their places come
// from counters).
__global__ __launch_bounds__(kTileThreads) void list_pieces_kernel(SortParams p) {
  if (static_cast<int>(blockIdx.x) >= p.zero.sorters) {
    zero_rows<kTileThreads>(p.zero, blockIdx.x - p.zero.sorters, gridDim.x - p.zero.sorters);
    return;
  }
  __shared__ int32_t counts[2], places[2];
  __shared__ Piece pieces[kTileThreads];
  __shared__ LongRun longs[kTileThreads / kPiece + 1];
  const int tid = threadIdx.x;
  if (tid < 2) counts[tid] = 0;
  __syncthreads();
  const int i0 = blockIdx.x * kTileThreads + __builtin_amdgcn_readfirstlane(tid >> 6) * 64;
  if (i0 < p.num_tokens)
    list_pieces(
        p.keys_out, p.num_tokens, p.vocab, i0, 0, [&](int i) { return p.order_out[i]; }, [](uint32_t k) { return k; },
        counts, pieces, longs);
  __syncthreads();
  if (tid == 0) places[0] = atomicAdd(&p.heads->pieces[0], counts[0]);
  if (tid == 1) places[1] = atomicAdd(&p.heads->longs[0], counts[1]);
  __syncthreads();
  if (tid < counts[0]) p.pieces[places[0] + tid] = pieces[tid];
  if (tid < counts[1]) p.longs[places[1] + tid] = longs[tid];
}

// ---------------------------------------------------------------------------
// Sums
// ---------------------------------------------------------------------------
struct GradParams {
  const int32_t* order;
  const void* dout;
  void* grad;
  const ListHeads* heads;
  const Piece* pieces;
  const LongRun* longs;
  float* parts;           // [2 * ceil(T / kPiece)][hidden]
  int64_t dout_stride, grad_stride;
  float scale;
  int32_t num_tokens, hidden;
};

// Of the pieces of long runs at most one first and at most one later one starts in any kPiece positions
// (the run between two first ones is longer, and a later piece starts that far behind its predecessor),
// so the two places of a stretch are never shared.
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

// A wave to a piece and 512 columns, eight of the piece's rows in flight, added in order; the next piece's
// record comes meanwhile.  Pieces differ in length, so a CU gets 32 workgroups one after another, not all
// of its work at once (16,384 tokens, 32,000 x 4096 bf16: 92 us with 8 to a CU, 87.6 with 32, 88.4 with 128).
// kOnce: the tokens' rows pass the caches by, which then take the sums (us for dout of 33 MB and a table of 131 57 -> 42, of
// 131 and 262 103 -> 87; where the caches hold both, of 51 and 16 57 -> 61, of 4-16 and 65 21 -> 22.5; added to a table, of
// which the sums' rows alone are touched, 134 MB 61 -> 67, 537 MB 285 -> 256).
template <bool kFp32, bool kAdd, bool kOnce>
__global__ __launch_bounds__(256, 6) void sum_pieces_kernel(GradParams p) {
  constexpr int kAhead = 8;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const ListParts parts(p.heads->pieces, p.heads->base, 1);
  const int total = parts.total();
  PairWalk walk(blockIdx.x * 4 + wave, gridDim.x * 4, p.hidden);
  Piece next{};
  if (walk.entry < total) next = p.pieces[parts.at(walk.entry)];
  while (walk.entry < total) {
    const Piece piece = next;
    const int col = walk.block * 512 + 8 * lane;
    walk.go_on();
    if (walk.entry < total) next = p.pieces[parts.at(walk.entry)];
    const int n = __builtin_amdgcn_readfirstlane(piece.tokens & (2 * kPiece - 1));
    int mine = piece.token;
    if (lane > 0 && lane < n) mine = p.order[piece.at + lane];
    const bool here = col < p.hidden;
    float s[8] = {};
    for (int j0 = 0; j0 < n; j0 += kAhead) {
      u32x4 w[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        w[j] = u32x4{0, 0, 0, 0};
        if (j0 + j >= n) continue;
        const int64_t t = __builtin_amdgcn_readlane(mine, j0 + j);
        if (here) w[j] = load16_as<kOnce>(p.dout, t * (p.dout_stride / 8), col / 8);
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
    if (piece.tokens & kOfLong) {
      float4* to = reinterpret_cast<float4*>(p.parts + part_of(piece.at, (piece.tokens & kFirst) != 0) * p.hidden + col);
      to[0] = make_float4(s[0], s[1], s[2], s[3]);
      to[1] = make_float4(s[4], s[5], s[6], s[7]);
    } else {
      write_row<kFp32, kAdd>(p, piece.row, col, s);
    }
  }
}

// Adds the pieces of long runs: a workgroup to a run and 512 columns, the pieces in kJoinWaves equal parts,
// each part by a wave in order, then the parts in order.
constexpr int kJoinWaves = 8;
template <bool kFp32, bool kAdd>
__global__ __launch_bounds__(64 * kJoinWaves) void join_pieces_kernel(GradParams p) {
  constexpr int kAhead = 8;
  __shared__ float sums[kJoinWaves][8][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const ListParts parts(p.heads->longs, p.heads->base, kPiece);
  const int total = parts.total();
  for (PairWalk walk(blockIdx.x, gridDim.x, p.hidden); walk.entry < total; walk.go_on()) {
    const LongRun run = p.longs[parts.at(walk.entry)];
    const int col = walk.block * 512 + 8 * lane;
    const bool here = col < p.hidden;
    const int pieces = (run.end - run.begin + kPiece - 1) / kPiece, share = (pieces + kJoinWaves - 1) / kJoinWaves;
    const int last = min((wave + 1) * share, pieces);
    float s[8] = {};
    for (int k0 = wave * share; k0 < last; k0 += kAhead) {
      float4 q[kAhead][2];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        q[j][0] = q[j][1] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k0 + j >= last || !here) continue;
        const float4* in = reinterpret_cast<const float4*>(p.parts + part_of(run.begin + (k0 + j) * kPiece, k0 + j == 0) * p.hidden + col);
        q[j][0] = in[0];
        q[j][1] = in[1];
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        if (k0 + j >= last) break;
        const float x[8] = {q[j][0].x, q[j][0].y, q[j][0].z, q[j][0].w, q[j][1].x, q[j][1].y, q[j][1].z, q[j][1].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = s[e] + x[e];
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[wave][e][lane] = s[e];
    __syncthreads();
    if (wave == 0 && here) {
      for (int w = 1; w * share < pieces; ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = s[e] + sums[w][e][lane];
      write_row<kFp32, kAdd>(p, run.row, col, s);
    }
    __syncthreads();
  }
}

// Zeros alone, for no tokens.
__global__ __launch_bounds__(kTileThreads) void zero_rows_kernel(ZeroParams z) {
  zero_rows<kTileThreads>(z, blockIdx.x, gridDim.x);
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// The workspace's parts, in order.
struct GradSpace {
  size_t keys, order, hist, heads, pieces, longs, parts, total;
  GradSpace(int64_t tokens, int64_t hidden) {
    const int64_t tiles = (tokens + kTile - 1) / kTile, stretches = (tokens + kPiece - 1) / kPiece;
    keys = 0;
    order = keys + 2 * round256(4 * tokens);
    hist = order + 2 * round256(4 * tokens);
    heads = hist + round256(4 * kBins * (tiles + 1));
    pieces = heads + round256(sizeof(ListHeads));
    longs = pieces + round256(sizeof(Piece) * tokens);
    parts = longs + round256(sizeof(LongRun) * stretches);
    total = parts + round256(2 * stretches * hidden * 4);
  }
};

}  // namespace

hipError_t launch_embedding(const EmbeddingLaunch& a, hipStream_t stream) {
  EmbeddingParams p{a.ids, a.table, a.out, a.table_stride, a.out_stride, a.scale, a.num_tokens, a.vocab, a.hidden_dim,
                    streams(a.num_tokens, a.hidden_dim), 0};
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
  z.row_pieces = a.grad_stride * size / 16;
  z.pieces = static_cast<int32_t>(static_cast<int64_t>(a.hidden_dim) * size / 16);
  // workgroups of `threads` that write zeros: a row to a wave, in the order they start, so that neighbours are
  // written together (151,936 x 4096 fp32: 32 us less a call than with two to a CU that walk the table)
  auto zeroers = [&](int threads) {
    const int64_t waves = threads / 64, blocks = (z.end - z.begin + waves - 1) / waves;
    const int64_t most = static_cast<int64_t>(cus) * 131072 / threads;
    return static_cast<unsigned>(blocks < most ? blocks : most);
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
  s.heads = reinterpret_cast<ListHeads*>(ws + at.heads);
  s.pieces = reinterpret_cast<Piece*>(ws + at.pieces);
  s.longs = reinterpret_cast<LongRun*>(ws + at.longs);
  s.num_tokens = a.num_tokens;
  s.vocab = a.vocab;
  s.tiles = (a.num_tokens - 1) / kTile + 1;
  const bool small = a.num_tokens <= kSmall;
  const int32_t largest = small ? (a.vocab - 1) / kBuckets : a.vocab;  // of the keys
  int bits = 1;
  while (bits < 31 && (largest >> bits) != 0) ++bits;
  s.passes = (bits + kDigitBits - 1) / kDigitBits;
  s.bits = (bits + s.passes - 1) / s.passes;
  // the rows to clear are shared out over the launches of the sort
  const int launches = small ? 1 : 2 * s.passes + 1;
  int done = 0;
  auto launch = [&](auto kernel, int sorters, int threads, size_t lds) {
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
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(threads), lds, stream, s);
    return hipGetLastError();
  };
  auto buffers = [&](int side) {
    s.keys_in = reinterpret_cast<const uint32_t*>(ws + at.keys + (side ^ 1) * list);
    s.order_in = reinterpret_cast<const int32_t*>(ws + at.order + (side ^ 1) * list);
    s.keys_out = reinterpret_cast<uint32_t*>(ws + at.keys + side * list);
    s.order_out = reinterpret_cast<int32_t*>(ws + at.order + side * list);
  };
  hipError_t e = hipSuccess;
  if (small) {
    buffers(0);
    e = launch(sort_small_kernel, kBuckets, kSmallThreads, static_cast<size_t>(a.num_tokens) * 6);
  } else {
    for (int pass = 0; pass < s.passes && e == hipSuccess; ++pass) {
      buffers(pass & 1);
      s.shift = pass * s.bits;
      e = pass == 0 ? launch(sort_count_kernel<true>, s.tiles, kTileThreads, 0) : launch(sort_count_kernel<false>, s.tiles, kTileThreads, 0);
      if (e == hipSuccess && s.tiles > kManyTiles) {
        hipLaunchKernelGGL(sum_tiles_kernel, dim3(kBins / 64), dim3(64), 0, stream, s.hist, s.tiles);
        e = hipGetLastError();
      }
      if (e == hipSuccess)
        e = pass == 0 ? launch(sort_move_kernel<true>, s.tiles, kTileThreads, 0) : launch(sort_move_kernel<false>, s.tiles, kTileThreads, 0);
    }
    if (e == hipSuccess) e = launch(list_pieces_kernel, (a.num_tokens - 1) / kTileThreads + 1, kTileThreads, 0);
  }
  if (e != hipSuccess) return e;
  GradParams p{};
  p.order = s.order_out;
  p.dout = a.dout;
  p.grad = a.grad;
  p.heads = s.heads;
  p.pieces = s.pieces;
  p.longs = s.longs;
  p.parts = reinterpret_cast<float*>(ws + at.parts);
  p.dout_stride = a.dout_stride;
  p.grad_stride = a.grad_stride;
  p.scale = a.scale;
  p.num_tokens = a.num_tokens;
  p.hidden = a.hidden_dim;
  const int64_t units = static_cast<int64_t>(a.num_tokens) * ((a.hidden_dim + 511) / 512);
  const int64_t sum_grid = (units + 3) / 4 < 32 * cus ? (units + 3) / 4 : 32 * cus;
  const int64_t join_grid = units / kPiece + 1 < 4 * cus ? units / kPiece + 1 : 4 * cus;
  const int64_t read = 2 * static_cast<int64_t>(a.num_tokens) * a.hidden_dim, table = static_cast<int64_t>(a.vocab) * a.hidden_dim * size;
  const bool once = a.accumulate ? read >= int64_t{256} << 20 : read >= int64_t{24} << 20 && read + table >= int64_t{128} << 20;
  auto sums = [&](auto fp32, auto add) {
    constexpr bool kFp32 = decltype(fp32)::value, kAdd = decltype(add)::value;
    if (once)
      hipLaunchKernelGGL((sum_pieces_kernel<kFp32, kAdd, true>), dim3(sum_grid), dim3(256), 0, stream, p);
    else
      hipLaunchKernelGGL((sum_pieces_kernel<kFp32, kAdd, false>), dim3(sum_grid), dim3(256), 0, stream, p);
    if (a.num_tokens > kPiece)
      hipLaunchKernelGGL((join_pieces_kernel<kFp32, kAdd>), dim3(join_grid), dim3(64 * kJoinWaves), 0, stream, p);
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
