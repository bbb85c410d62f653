// Token-wise decode against a cache held in 8 or 4 bits (uattn_mx.h).
//
// The values that the codes stand for are bf16 numbers, and what is done with them is
// what uattn_decode does with a bf16 cache, operation for operation and in the same
// order (uattn_numerics.h): the same products, tiles of 64 keys, chunks of 256,
// references, weights and fold.  So a row has the bits of uattn_decode over a bf16
// cache of the same values, and of uattn_prefill over those rows.
//
// A wave computes a chunk by itself, the G query heads of the kv head in the MFMA
// columns, its four tiles one after another: with a quarter (4 bits) to a half of the
// bytes of a bf16 cache there is as much less time for everything else, so a chunk
// has no barrier and its waves share nothing.
//
//   K  a lane (row r = lane % 16 of a 16-key block, group g = lane / 16) loads a quarter
//      of a row; the score product's operand wants of every 32-wide step the g-th eight
//      elements, which a transposition of the words between the lane groups gives
//      (permlane swaps), still as codes; the conversion's result is the operand;
//   V  a lane loads a quarter of a row, converts it and writes it to LDS as the rows that
//      the transposing read of the P V product expects, 32 keys at a time (a wave's own
//      8 KB, in order: no barrier).
//
// The weights are rounded to bf16 for the P V product and its normaliser, as uattn_decode
// does (2^-8 of each; without this the two would have other bits): rows are off by 0.0022
// of their size against 64 bits, 0.0017 with weights in 32 bits.
//
// What bounds it: memory.  8 x 32K keys, 64/8 heads, 4 bits (285 MB of codes and scales)
// take 65 us.  Timing copies: without the merge's launch 57, without partials at all 51,
// without the conversion of V too 47, loads alone 44 (6.5 TB/s).  In 8 bits (554 MB) 113,
// 105, 89, 88 and 88.  The partials (34 MB) are what costs: mixed into a read stream they
// take several times their share of the bytes, in whatever order, width or policy they are
// stored (as [chunk][head][d] in whole lines: no change; past the caches: no change;
// device-coherent: 1-3% less, kept).  So where many (entry, kv head) pairs are there, a
// workgroup keeps a pair to itself and nothing is stored (Split, below).  Codes are read
// past the caches where there are more than these hold (71 -> 65 us; a step of 64 MB that
// the caches hold 25 -> 29).  Of earlier forms of this kernel, a walk of persistent waves,
// the next item's codes on their way while one is computed, was 7% slower than one wave an
// item, and three waves to a SIMD, for whose registers the next tile's codes come later, 1%.
#include <type_traits>

#include "uattn_internal.h"
#include "uattn_mx.h"
#include "uattn_tile_io.h"

namespace uattn {
namespace {

struct DecodeMxParams {
  const __bf16* q;
  const uint8_t* kc;
  const uint8_t* ks;
  const uint8_t* vc;
  const uint8_t* vs;
  const int32_t* bt;
  const int32_t* seqlens;
  __bf16* out;
  float* lse;
  float* ws_acc;  // [batch][Hq][nslot][D]
  float* ws_ml;   // [batch][Hq][nslot][2]
  int batch, hq, hkv, group, maxp, page_size, page_shift, num_pages, max_seqlen, nchunk_max, nslot;
  int stride;     // kChunks, kWalk: waves of an (entry, kv head)
  int first;      // workgroups of the launches before this one
  float c;
};

// Buffer access with a wave-uniform base and size: loads past `bytes` return zero
// without touching memory.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_rsrc(const void* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), static_cast<short>(0), bytes, 0x00020000);
}

// A row's codes and a lane's quarter of them.
template <int D, int Bits>
struct MxRow {
  static constexpr int kBytes = D * Bits / 8;
  static constexpr int kLaneBytes = kBytes / 4;
  static constexpr int kWords = kLaneBytes / 4;
  static constexpr int kOctWords = Bits / 4;         // words of eight elements
  static constexpr int kOcts = kWords / kOctWords;   // D / 32
  static constexpr int kScales = D / kMxBlock;       // scale bytes of a row
  // the quarter is loaded in runs of up to 16 bytes, lanes side by side, so that every
  // load covers whole sectors of memory
  static constexpr int kRunBytes = kLaneBytes < 16 ? kLaneBytes : 16;
  static constexpr int kRuns = kLaneBytes / kRunBytes;
};

// One tile's codes in this lane: its quarter rows of the four 16-key blocks and their scales.
template <int D, int KB, int VB>
struct TileCodes {
  uint32_t k[kKeyBlocks][MxRow<D, KB>::kWords];
  uint32_t v[kKeyBlocks][MxRow<D, VB>::kWords];
  uint32_t ks[kKeyBlocks];  // all scale bytes of row lane % 16
  uint32_t vs[kKeyBlocks][MxRow<D, VB>::kRuns];  // the scale bytes of this lane's runs of V
};

template <int kPolicy, int Words>
__device__ __forceinline__ void load_words(uint32_t (&w)[Words], __amdgpu_buffer_rsrc_t r, int off, int step) {
  if constexpr (Words == 2) {
    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, kPolicy));
    w[0] = x[0];
    w[1] = x[1];
  } else {
#pragma unroll
    for (int i = 0; i < Words / 4; ++i) {
      const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off + step * i, 0, kPolicy));
#pragma unroll
      for (int j = 0; j < 4; ++j) w[4 * i + j] = x[j];
    }
  }
}

__device__ __forceinline__ void swap16(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}
__device__ __forceinline__ void swap32(uint32_t& a, uint32_t& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

// The words of a lane's octets -> those that step j of the score product wants of lane
// group g, octet 4 * j + g.  A lane holds octets 4 * g .. 4 * g + 3 of its row (D = 128
// in 4 bits) or, a run of two at a time, 2 * g and 2 * g + 1 of eight.
template <class R, int Words>
__device__ __forceinline__ void to_steps(uint32_t (&w)[Words]) {
  static_assert(Words == R::kWords, "a lane's quarter");
  constexpr int O = R::kOctWords;
#pragma unroll
  for (int x = 0; x < O; ++x) {
    if constexpr (R::kOcts == 4 && O == 1) {
      swap16(w[0], w[1]);
      swap16(w[2], w[3]);
      swap32(w[0], w[2]);
      swap32(w[1], w[3]);
    } else {
#pragma unroll
      for (int i = 0; i < R::kOcts; i += 2) {
        swap16(w[i * O + x], w[(i + 1) * O + x]);
        swap32(w[i * O + x], w[(i + 1) * O + x]);
      }
    }
  }
}

// Waits until matrix results may be read.  The compiler does so ahead of every read, but
// looks past a branch in between along one of its ways only: with the mask's branch after
// the score products, tiles that were not the last read sums of which a part was missing
// (ROCm 7.2.0).  So the products are followed by the wait states here, before the branch.
template <int NB>
__device__ __forceinline__ void settle(f32x4 (&s)[NB][kKeyBlocks]) {
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
    asm volatile("s_nop 7" : "+v"(s[nb][0]), "+v"(s[nb][1]), "+v"(s[nb][2]), "+v"(s[nb][3]));
}

// Who takes what (launch() chooses):
//   kChunks  a workgroup is one wave and takes one chunk of an (entry, kv head); fp32
//            partials go to the workspace for decode_mx_merge_kernel (entries of one chunk
//            are finished)
//   kWalk    the same, but a wave takes every stride-th chunk
//   kFused   a workgroup takes all chunks, at most kTeamWaves, of an (entry, kv head), one
//            to a wave, and folds them in LDS behind one barrier
//   kTeam    a workgroup takes all chunks of an (entry, kv head), its waves in turn; a
//            wave adds its chunk to one state in LDS when the chunks before are in it
enum class Split { kChunks, kWalk, kFused, kTeam };
constexpr int kTeamWaves = 8;  // of a kFused workgroup, at most
constexpr int kTurnWaves = 4;  // of a kTeam workgroup: two to a CU
constexpr int64_t kMostWaves = 32768;  // of one wave each, where (entry, kv head) pairs alone are not more

// kLoad: cache policy of the loads of codes (0, or kStreamed).
constexpr int kStreamed = 2;   // the nt bit of the buffer instructions' cache-policy operand
constexpr int kCoherent = 16;  // the sc1 bit: stores to the device-coherent level

// Two blocks of heads at d = 128 take all registers of a SIMD; in 4 bits half of them
// will do, with the queries in LDS and the next tile's codes in this tile's registers.
// 10 x 1500-12000 keys, 136/8 heads 28.5 -> 25.5 us, 16 x 4000-8000, 128/4 30.2 -> 26.6;
// with 8 bits on either side registers spill (keys 32.1 -> 34.2, values 32.4 -> 36.4).
template <int D, int NB, int KB, int VB>
constexpr bool kHalfSimd = NB == 2 && D == 128 && KB + VB == 8;

template <int D, int NB, int KB, int VB, Split kSplit, int kLoad>
__global__ __launch_bounds__(64 * (kSplit == Split::kFused ? kTeamWaves : kSplit == Split::kTeam ? kTurnWaves : 1),
                             (kHalfSimd<D, NB, KB, VB> ? 2 : 1)) void decode_mx_kernel(
    DecodeMxParams p, const int32_t* __restrict__ seqlens, const int32_t* __restrict__ block_table) {
  using TL = TileLayout<D>;
  using RK = MxRow<D, KB>;
  using RV = MxRow<D, VB>;
  constexpr int KS = D / 32;   // K steps of the score product
  constexpr int NDB = D / 16;  // d blocks of the output
  constexpr int kPieces = D / 4;  // 16-byte pieces of a head's partial
  constexpr bool kFused = kSplit == Split::kFused, kTeam = kSplit == Split::kTeam, kChunks = !kFused && !kTeam;
  constexpr int kWaves = kFused ? kTeamWaves : kTeam ? kTurnWaves : 1;
  // The next tile's codes have registers of their own where there are enough.  kTeam, 256
  // entries, 32/8 heads of 128: 4000 keys, keys in 4 bits, values in 8 277 us with, 253
  // without; 8 bits 354 and 331; keys in 8, values in 4 268 and 278.  Of 64, 500-8000 keys,
  // 8 bits: 183 and 196.
  constexpr bool kQueriesInLds = kHalfSimd<D, NB, KB, VB>;
  constexpr bool kTwo = !kQueriesInLds && !(kTeam && D == 128 && VB == 8);
  // per wave: 32 keys' values on their way to the products; then (kFused) its partial
  // [NB][16][D] fp32.  Rows of partials and of the state below: 16-byte pieces,
  // XOR-swizzled by the head.
  static_assert(32 * sizeof(__bf16) == kQCols * sizeof(float), "a partial of 16 heads takes 32 keys' room");
  __shared__ __attribute__((aligned(1024))) __bf16 room[kWaves][(kFused ? NB : 1) * 32 * D];
  __shared__ bf16x8 queries[kQueriesInLds ? NB * kQCols * KS * 4 : 1];  // rows' pieces swizzled by the head
  __shared__ float2 ml[kFused ? kWaves : 1][NB * kQCols];
  // kTeam: the fold so far and how many chunks it holds
  __shared__ __attribute__((aligned(16))) f32x4 state[kTeam ? NB * kQCols * kPieces : 1];
  __shared__ float2 state_ml[kTeam ? NB * kQCols : 1];
  __shared__ int turn;

  const int wave = kWaves > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  __bf16* const vrows = room[wave];
  const int lane = threadIdx.x & 63;
  const int g = lane >> 4, col = lane & 15;
  // kv heads side by side: their pages' parts lie side by side
  const int u = p.first + blockIdx.x;
  const int kvh = u % p.hkv;
  int chunk = wave, b = u / p.hkv;
  if constexpr (kChunks) {
    chunk = b % p.stride;
    b /= p.stride;
  }
  const int n = min(seqlens[b], p.max_seqlen);
  if (kChunks ? chunk * kChunkKeys >= n : n < 1) return;
  if constexpr (kTeam) {
    if (threadIdx.x == 0) turn = 0;
    __syncthreads();
  }
  const int nch = (n + kChunkKeys - 1) / kChunkKeys;
  const int last_tile = (n - 1) / kTileKeys;
  const int head0 = kvh * p.group;

  // the pages of a chunk's sixteen 16-key blocks, one to a lane
  auto load_pages = [&](int ch) {
    const int pos = ch * kChunkKeys + 16 * col;
    return block_table[static_cast<int64_t>(b) * p.maxp + min(pos >> p.page_shift, p.maxp - 1)];
  };
  int pages = load_pages(chunk);

  // query operands: column col of block nb, d = 32 * step + 8 * g .. + 7
  bf16x8 qf[NB][KS];
  {
    const auto rq = buffer_rsrc(p.q + (static_cast<int64_t>(b) * p.hq + head0) * D, p.group * D * 2);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int st = 0; st < KS; ++st)
        qf[nb][st] = __builtin_bit_cast(
            bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rq, (nb * kQCols + col) * D * 2 + 16 * g + 64 * st, 0, 0));
  }

  if constexpr (kQueriesInLds) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int st = 0; st < KS; ++st) queries[(nb * kQCols + col) * (4 * KS) + ((4 * st + g) ^ col)] = qf[nb][st];
  }
  auto query = [&](int nb, int st) __attribute__((always_inline)) {
    if constexpr (kQueriesInLds)
      return queries[(nb * kQCols + col) * (4 * KS) + ((4 * st + g) ^ col)];
    else
      return qf[nb][st];
  };

  // Codes of 16-key block kb of tile t of chunk ch.  Blocks past the context, on a page
  // outside the pool or past the table read as zeros (codes 0, scale byte 0) without
  // touching memory.
  const int k_off = col * RK::kBytes + g * RK::kRunBytes;
  // V: run i of a lane is that of row kRunRows * i + v_row, the v_part-th of the row
  constexpr int kRunRows = 64 * RV::kRunBytes / RV::kBytes, kRowRuns = 64 / kRunRows;
  constexpr int kRunOcts = RV::kOcts / RV::kRuns;
  const int v_row = lane / kRowRuns, v_part = lane % kRowRuns;
  const int v_off = lane * RV::kRunBytes;
  const int vs_off = v_row * RV::kScales + v_part * RV::kScales / kRowRuns;
  struct Place {
    int64_t row;  // the block's first row in the pools
    int rows;     // its keys inside the context
  };
  auto place = [&](int ch, int its_pages, int t, int kb) -> Place {
    const int page = __builtin_amdgcn_readlane(its_pages, 4 * t + kb);
    const int pos = ch * kChunkKeys + t * kTileKeys + 16 * kb;
    const bool ok = page >= 0 && page < p.num_pages && pos < n;
    return {ok ? (((static_cast<int64_t>(page) * p.hkv + kvh) << p.page_shift) + (pos & (p.page_size - 1))) : 0,
            ok ? min(n - pos, 16) : 0};
  };
  TileCodes<D, KB, VB> codes[kTwo ? 2 : 1];
  auto load_k = [&](TileCodes<D, KB, VB>& x, const Place& at, int kb) __attribute__((always_inline)) {
    load_words<kLoad>(x.k[kb], buffer_rsrc(p.kc + at.row * RK::kBytes, at.rows * RK::kBytes), k_off, 4 * RK::kRunBytes);
    const auto r = buffer_rsrc(p.ks + at.row * RK::kScales, at.rows * RK::kScales);
    if constexpr (D == 128)
      x.ks[kb] = __builtin_amdgcn_raw_buffer_load_b32(r, 4 * col, 0, 0);
    else
      x.ks[kb] = static_cast<uint16_t>(__builtin_amdgcn_raw_buffer_load_b16(r, 2 * col, 0, 0));
  };
  auto load_v = [&](TileCodes<D, KB, VB>& x, const Place& at, int kb) __attribute__((always_inline)) {
    load_words<kLoad>(x.v[kb], buffer_rsrc(p.vc + at.row * RV::kBytes, at.rows * RV::kBytes), v_off, 64 * RV::kRunBytes);
    const auto r = buffer_rsrc(p.vs + at.row * RV::kScales, at.rows * RV::kScales);
#pragma unroll
    for (int i = 0; i < RV::kRuns; ++i)
      x.vs[kb][i] = static_cast<uint8_t>(__builtin_amdgcn_raw_buffer_load_b8(r, vs_off + i * kRunRows * RV::kScales, 0, 0));
  };
  auto load_tile = [&](TileCodes<D, KB, VB>& x, int ch, int its_pages, int t) __attribute__((always_inline)) {
#pragma unroll
    for (int kb = 0; kb < kKeyBlocks; ++kb) {
      const Place at = place(ch, its_pages, t, kb);
      load_k(x, at, kb);
      load_v(x, at, kb);
    }
  };

  f32x4 acc[NB][NDB], lsum[NB];
  float m[NB];
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = static_cast<__bf16>(1.0f);

  // Tile t of chunk ch; the tile after it is t_next of ch_next, on next_pages.
  auto tile_step = [&](int ch, int t, int ch_next, int t_next, int next_pages) __attribute__((always_inline)) {
    const int tile = ch * kTilesPerChunk + t;
    TileCodes<D, KB, VB>& x = codes[kTwo ? t & 1 : 0];
    if constexpr (kTwo) {
      if (kTeam || t_next > 0) load_tile(codes[t_next & 1], ch_next, next_pages, t_next);
      __builtin_amdgcn_sched_barrier(0);
    }
    f32x4 s[NB][kKeyBlocks];
#pragma unroll
    for (int kb = 0; kb < kKeyBlocks; ++kb) {
      to_steps<RK>(x.k[kb]);
      bf16x8 a[KS];
      a[0] = mx_decode8<KB>(&x.k[kb][0], mx_scale_of<0>(x.ks[kb]));
      a[1] = mx_decode8<KB>(&x.k[kb][RK::kOctWords], mx_scale_of<1>(x.ks[kb]));
      if constexpr (KS == 4) {
        a[2] = mx_decode8<KB>(&x.k[kb][2 * RK::kOctWords], mx_scale_of<2>(x.ks[kb]));
        a[3] = mx_decode8<KB>(&x.k[kb][3 * RK::kOctWords], mx_scale_of<3>(x.ks[kb]));
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < KS; ++st) r = mfma16(a[st], query(nb, st), r);
        s[nb][kb] = r;
      }
    }
    settle(s);
    if constexpr (!kTwo) {
      // the registers of these keys take the next tile's
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kb = 0; kb < kKeyBlocks; ++kb)
        if (kTeam || t_next > 0) load_k(x, place(ch_next, next_pages, t_next, kb), kb);
      __builtin_amdgcn_sched_barrier(0);
    }
    float alpha[NB];
    bf16x8 pb[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (tile == last_tile) mask_scores(s[nb], tile * kTileKeys, n - 1, lane);
      alpha[nb] = softmax_tile(s[nb], m[nb], p.c);
      pack_p(s[nb], pb[nb]);
    }
    rescale_acc<NB, NDB>(acc, lsum, alpha);
#pragma unroll
    for (int st = 0; st < 2; ++st) {
      // 32 keys' values into LDS
#pragma unroll
      for (int kh = 0; kh < 2; ++kh) {
        const int kb = 2 * st + kh;
#pragma unroll
        for (int i = 0; i < RV::kRuns; ++i) {
          const int row = 16 * kh + kRunRows * i + v_row;
          const float scale = mx_scale(x.vs[kb][i]);
#pragma unroll
          for (int o = 0; o < kRunOcts; ++o) {
            const int piece = (v_part * kRunOcts + o) ^ TL::v_swz(row);
            *reinterpret_cast<bf16x8*>(vrows + row * D + 8 * piece) =
                mx_decode8<VB>(&x.v[kb][(i * kRunOcts + o) * RV::kOctWords], scale);
          }
        }
      }
      if constexpr (!kTwo) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 2 * st; kb < 2 * st + 2; ++kb)
          if (kTeam || t_next > 0) load_v(x, place(ch_next, next_pages, t_next, kb), kb);
        __builtin_amdgcn_sched_barrier(0);
      }
      // acc <- acc + V^T P^T and lsum <- lsum + 1^T P^T over them: step st of pv_tile
      const int src = lane & 15, key = 4 * g + (src >> 2), sub = src & 3;
      const __bf16* vrow = vrows + key * D + 4 * (sub & 1);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) lsum[nb] = mfma16(ones, pb[nb][st], lsum[nb]);
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        const int piece = (2 * db + (sub >> 1)) ^ TL::v_swz(key);
        const s16x4 w[2] = {lds_read_tr16(vrow + 8 * piece), lds_read_tr16(vrow + 16 * D + 8 * piece)};
        bf16x8 a;
        __builtin_memcpy(&a, w, sizeof(bf16x8));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[nb][db] = mfma16(a, pb[nb][st], acc[nb][db]);
      }
    }
  };
  // The chunk's tiles in order, the next tile's codes on their way (kTeam: then those of
  // the wave's next chunk); (m, lsum, acc) is its partial.
  auto chunk_step = [&](int ch, int ch_next, int next_pages) __attribute__((always_inline)) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      m[nb] = neg_inf();
      lsum[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int db = 0; db < NDB; ++db) acc[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int t = 0; t < kTilesPerChunk; ++t) {
      if (ch * kTilesPerChunk + t > last_tile) break;
      if (t + 1 < kTilesPerChunk)
        tile_step(ch, t, ch, t + 1, pages);
      else
        tile_step(ch, t, ch_next, 0, next_pages);
    }
  };

  // The outputs of the columns' heads from (M, L, acc).
  auto finish = [&](int nb, float M, float L) __attribute__((always_inline)) {
    const int gi = kQCols * nb + col;
    if (gi >= p.group) return;
    const int64_t orow = static_cast<int64_t>(b) * p.hq + head0 + gi;
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      bf16x4 w;
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = finalize_val(acc[nb][db][j], L);
      *reinterpret_cast<bf16x4*>(p.out + orow * D + 16 * db + 4 * g) = w;
    }
    if (p.lse != nullptr && g == 0) p.lse[orow] = finalize_lse(M, L, p.c);
  };

  if constexpr (kTeam) {
    load_tile(codes[0], chunk, pages, 0);
#pragma unroll 1
    for (; chunk < nch; chunk += kWaves) {
      const int next_pages = load_pages(chunk + kWaves);  // past the last chunk no key is read through them
      chunk_step(chunk, chunk + kWaves, next_pages);
      pages = next_pages;
      // the chunks before this one are this workgroup's other waves', each on its way or done
      while (__builtin_amdgcn_readfirstlane(__hip_atomic_load(&turn, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP)) != chunk)
        __builtin_amdgcn_s_sleep(1);
      asm volatile("" ::: "memory");
      const bool last = chunk + 1 == nch;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int gi = kQCols * nb + col;
        float M = m[nb], L = lsum[nb][0];
        if (chunk > 0) {
          const float2 z = state_ml[gi];
          const FoldScale f = fold_scale(z.x, m[nb], p.c);
          M = f.m_new;
          L = fold_val(f, z.y, L);
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            const f32x4 y = state[gi * kPieces + ((4 * db + g) ^ col)];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[nb][db][j] = fold_val(f, y[j], acc[nb][db][j]);
          }
        }
        if (last) {
          finish(nb, M, L);
        } else {
#pragma unroll
          for (int db = 0; db < NDB; ++db) state[gi * kPieces + ((4 * db + g) ^ col)] = acc[nb][db];
          if (g == 0) state_ml[gi] = float2{M, L};
        }
      }
      // (a wave's LDS accesses are done in order: whoever sees the turn sees the state)
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (lane == 0) __hip_atomic_store(&turn, chunk + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
    return;
  }

  auto only = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) finish(nb, m[nb], lsum[nb][0]);
  };
  if constexpr (kChunks) {
    const int64_t row = static_cast<int64_t>(b) * p.hq + head0;
#pragma unroll 1
    for (;;) {
      load_tile(codes[0], chunk, pages, 0);
      chunk_step(chunk, chunk, pages);
      if (nch == 1) return only();
      // heads past the group's fall outside the resource and store nothing
      const auto racc = buffer_rsrc(p.ws_acc + row * p.nslot * D, p.group * p.nslot * D * 4);
      int head = col;
      // (the addresses of these stores are formed anew: kept over the walk they cost a register too many)
      if constexpr (kSplit == Split::kWalk && kQueriesInLds) asm volatile("" : "+v"(head));
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const int gi = kQCols * nb + head;
        const int off = ((gi * p.nslot + chunk) * D + 4 * g) * 4;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[nb][db]), racc, off + 64 * db, 0, kCoherent);
        if (g == 0 && gi < p.group)
          *reinterpret_cast<float2*>(p.ws_ml + ((row + gi) * p.nslot + chunk) * 2) = float2{m[nb], lsum[nb][0]};
      }
      chunk += p.stride;
      if (kSplit == Split::kChunks || chunk >= nch) return;
      pages = load_pages(chunk);
    }
  }
  if (chunk < nch) {
    load_tile(codes[0], chunk, pages, 0);
    chunk_step(chunk, chunk, pages);
  }
  if (nch == 1) {
    if (chunk == 0) only();
    return;
  }
  if constexpr (kFused) {
    if (chunk < nch) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        f32x4* rows = reinterpret_cast<f32x4*>(vrows) + nb * kQCols * kPieces;
#pragma unroll
        for (int db = 0; db < NDB; ++db) rows[col * kPieces + ((4 * db + g) ^ col)] = acc[nb][db];
        if (g == 0) ml[wave][nb * kQCols + col] = float2{m[nb], lsum[nb][0]};
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.group * kPieces; i += blockDim.x) {
      const int gi = i / kPieces, piece = i % kPieces;
      const int at = gi * kPieces + (piece ^ (gi % kQCols));
      f32x4 A = reinterpret_cast<const f32x4*>(room[0])[at];
      float M = ml[0][gi].x, L = ml[0][gi].y;
      for (int k = 1; k < nch; ++k) {
        const f32x4 y = reinterpret_cast<const f32x4*>(room[k])[at];
        const float2 z = ml[k][gi];
        const FoldScale f = fold_scale(M, z.x, p.c);
        L = fold_val(f, L, z.y);
#pragma unroll
        for (int j = 0; j < 4; ++j) A[j] = fold_val(f, A[j], y[j]);
        M = f.m_new;
      }
      const int64_t orow = static_cast<int64_t>(b) * p.hq + head0 + gi;
      bf16x4 o;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = finalize_val(A[j], L);
      *reinterpret_cast<bf16x4*>(p.out + orow * D + 4 * piece) = o;
      if (p.lse != nullptr && piece == 0) p.lse[orow] = finalize_lse(M, L, p.c);
    }
  }
}

// Folds the partials of one (entry, q head) row in chunk order; a wave takes 64 of a
// row's d, one to a lane.  Lane i forms the fold scales of chunk i of a group of 64:
// the running maximum before a chunk is a scan of the chunks' maxima (the maximum is
// exact and associative, so the scan has the bits of the chain), and fold_scale gets
// the arguments of the chain.  Then the sum goes chunk by chunk, with a chunk's scales
// from its lane, while kAhead chunks' partials are on their way.
template <int D>
__global__ __launch_bounds__(64) void decode_mx_merge_kernel(DecodeMxParams p) {
  constexpr int kAhead = 32;
  const int lane = threadIdx.x;
  const int id = p.first + blockIdx.x;
  const int row = id / (D / 64), d = 64 * (id % (D / 64)) + lane;
  const int n = min(p.seqlens[row / p.hq], p.max_seqlen);
  const int nch = (n + kChunkKeys - 1) / kChunkKeys;
  if (nch < 2) return;  // the item wrote it (or the entry has no keys)
  const int64_t slot = static_cast<int64_t>(row) * p.nslot;
  const auto racc = buffer_rsrc(p.ws_acc + slot * D, nch * D * 4);
  const auto rml = buffer_rsrc(p.ws_ml + slot * 2, nch * 8);
  float x[2][kAhead];
  // (the whole offset where the resource's bounds are checked: chunks past the last read 0)
  auto load = [&](int k0, float (&y)[kAhead]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      y[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(racc, ((k0 + i) * D + d) * 4, 0, 0));
  };
  float M = 0.f, L = 0.f, A = 0.f;
  load(0, x[0]);
  for (int k0 = 0; k0 < nch; k0 += 64) {
    const u32x2 ml = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rml, (k0 + lane) * 8, 0, 0));
    const float m = k0 + lane < nch ? __uint_as_float(ml[0]) : neg_inf();
    const float l = __uint_as_float(ml[1]);
    load(k0 + kAhead, x[1]);
    float run = m;
#pragma unroll
    for (int sh = 1; sh < 64; sh <<= 1) {
      const float o = __shfl_up(run, sh, 64);
      if (lane >= sh) run = vmax(run, o);
    }
    if (k0 > 0) run = vmax(M, run);
    float before = __shfl_up(run, 1, 64);
    if (lane == 0) before = M;
    const FoldScale f = fold_scale(before, m, p.c);
    const float bl = f.b * l;
    auto fold = [&](int first, const float (&y)[kAhead]) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int k = first + i;
        if (k0 + k < nch) {
          FoldScale s;
          s.a = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f.a), k));
          s.b = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f.b), k));
          if (k == 0 && k0 == 0) {
            L = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(l), 0));
            A = y[0];
          } else {
            L = __builtin_fmaf(s.a, L, __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(bl), k)));
            A = fold_val(s, A, y[i]);
          }
        }
      }
    };
    fold(0, x[0]);
    if (k0 + kAhead < nch) {
      if (k0 + 64 < nch) load(k0 + 64, x[0]);
      fold(kAhead, x[1]);
    }
    M = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(run), 63));
  }
  p.out[static_cast<int64_t>(row) * D + d] = finalize_val(A, L);
  if (p.lse != nullptr && d == 0) p.lse[row] = finalize_lse(M, L, p.c);
}

template <int D, int NB, int KB, int VB>
hipError_t launch(DecodeMxParams p, int num_cus, hipStream_t stream) {
  const int64_t pairs = static_cast<int64_t>(p.batch) * p.hkv;
  auto run = [&](auto kernel, int64_t workgroups, int waves) {
    return launch_parts(workgroups, 64 * waves, [&](int first, unsigned n) {
      p.first = first;
      hipLaunchKernelGGL(kernel, dim3(n), dim3(64 * waves), 0, stream, p, p.seqlens, p.bt);
    });
  };
  // Two blocks of heads at d = 128 go by chunks alone.  Eight waves that fold in LDS have too
  // few registers in 8 bits; in 4 they were no faster (16 entries of 300-2000 keys, 128/4
  // heads 18.0 us by chunks, 19.0 folded).  A workgroup to a pair is not built there, though
  // it fits (337 registers in 8 bits, 15 of them spilled in 4) and gains with many pairs: 256
  // x 4000 keys, 136/8 heads 351 -> 286 us in 4 bits, 555 -> 491 in 8.
  if constexpr (NB == 1 || D == 64) {
    // Up to kTeamWaves chunks: one launch, nothing through memory.  A step of 700 keys,
    // 32/8 heads, 8 bits 11.0 us with a merge, 9.3 so; 64 entries of 300-2000 keys 44.3 and
    // 41.6.
    if (p.nchunk_max > 1 && decode_mx_in_lds(p.nchunk_max, p.group, D))
      return run(decode_mx_kernel<D, NB, KB, VB, Split::kFused, 0>, pairs, p.nchunk_max);
    // Many pairs: a workgroup to a pair.  256 entries of 4000 keys, 32/8 heads, 8 bits 430
    // us with partials and their merge, 332 so; of 500-8000 keys in 4 bits 228, 217.  With
    // 512 pairs the longest are too long for their workgroups (64 of 1280-16384, keys in 8
    // bits, values in 4: 201, 209; of one length, which a launch does not know, 189, 150).
    if (p.nchunk_max > kTeamWaves && pairs >= 4 * static_cast<int64_t>(num_cus))
      return run(decode_mx_kernel<D, NB, KB, VB, Split::kTeam, kStreamed>, pairs, kTurnWaves);
  }
  // Codes go past the caches where the call may read more than half of what the last of
  // them holds (256 MB): 8 x 32K keys 71 -> 65 us, 64 of 4000-8000, d = 64, 4 bits 56 -> 53; 10
  // of 1500-12000, 136/8 heads (64 MB, bound 104) 25 -> 29.
  const int64_t bytes = pairs * p.max_seqlen * (MxRow<D, KB>::kBytes + MxRow<D, VB>::kBytes + 2 * MxRow<D, KB>::kScales);
  // A wave to each chunk up to 32768 waves, as those without keys cost too: 64 entries of
  // 500-1000 keys, 32/8 heads, 4 bits under a bound of 128K keys 68 us so, 26 with a walk
  // (with one of 4096 waves 20, but 64 of 1280-16384 keys then 229, not 195).  The walk's
  // bound says nothing of the lengths; it reads past the caches: 64 of 2000-4000 keys (209
  // MB) 55 us, 59 through them; 64 of 500-1000 in 8 bits (101 MB, which they hold) 36 and 31.
  const int64_t most = pairs < kMostWaves ? kMostWaves / pairs : 1;
  p.stride = p.nchunk_max < most ? p.nchunk_max : static_cast<int>(most);
  const hipError_t e = p.stride < p.nchunk_max ? run(decode_mx_kernel<D, NB, KB, VB, Split::kWalk, kStreamed>, pairs * p.stride, 1)
                       : bytes > (int64_t{128} << 20)
                           ? run(decode_mx_kernel<D, NB, KB, VB, Split::kChunks, kStreamed>, pairs * p.stride, 1)
                           : run(decode_mx_kernel<D, NB, KB, VB, Split::kChunks, 0>, pairs * p.stride, 1);
  if (e != hipSuccess || p.nchunk_max == 1) return e;
  return launch_parts(static_cast<int64_t>(p.batch) * p.hq * (D / 64), 64, [&](int first, unsigned n) {
    p.first = first;
    hipLaunchKernelGGL(decode_mx_merge_kernel<D>, dim3(n), dim3(64), 0, stream, p);
  });
}

}  // namespace

bool decode_mx_in_lds(int64_t nchunk, int64_t group, int64_t head_dim) {
  return nchunk <= kTeamWaves && (group <= kQCols || head_dim == 64);
}

hipError_t launch_decode_mx(const DecodeLaunch& a, const MxCache& cache, hipStream_t stream) {
  DecodeMxParams p;
  p.q = static_cast<const __bf16*>(a.q);
  p.kc = static_cast<const uint8_t*>(cache.k_codes);
  p.ks = static_cast<const uint8_t*>(cache.k_scales);
  p.vc = static_cast<const uint8_t*>(cache.v_codes);
  p.vs = static_cast<const uint8_t*>(cache.v_scales);
  p.bt = a.block_table;
  p.seqlens = a.seqlens;
  p.out = static_cast<__bf16*>(a.out);
  p.lse = a.lse;
  p.ws_acc = a.ws_acc;
  p.ws_ml = a.ws_ml;
  p.batch = a.batch;
  p.hq = a.num_q_heads;
  p.hkv = a.num_kv_heads;
  p.group = a.num_q_heads / a.num_kv_heads;
  p.maxp = a.max_pages_per_seq;
  p.page_size = a.page_size;
  p.page_shift = __builtin_ctz(static_cast<unsigned>(a.page_size));
  p.num_pages = a.num_pages;
  p.max_seqlen = a.max_seqlen;
  p.nchunk_max = a.nchunk_max;
  p.nslot = static_cast<int>(decode_slots(a.nchunk_max));
  p.first = p.stride = 0;
  p.c = a.c;
  using std::integral_constant;
  auto pick = [&](auto d, auto nb, auto kb, auto vb) {
    return launch<decltype(d)::value, decltype(nb)::value, decltype(kb)::value, decltype(vb)::value>(p, a.num_cus, stream);
  };
  auto pick_v = [&](auto d, auto nb, auto kb) {
    return cache.v_bits == 8 ? pick(d, nb, kb, integral_constant<int, 8>{}) : pick(d, nb, kb, integral_constant<int, 4>{});
  };
  auto pick_k = [&](auto d, auto nb) {
    return cache.k_bits == 8 ? pick_v(d, nb, integral_constant<int, 8>{}) : pick_v(d, nb, integral_constant<int, 4>{});
  };
  auto pick_nb = [&](auto d) {
    return p.group > kQCols ? pick_k(d, integral_constant<int, 2>{}) : pick_k(d, integral_constant<int, 1>{});
  };
  return a.head_dim == 128 ? pick_nb(integral_constant<int, 128>{}) : pick_nb(integral_constant<int, 64>{});
}

}  // namespace uattn
