// Token-wise decode against a cache held in 8 or 4 bits (uattn_mx.h).
//
// The values that the codes stand for are bf16 numbers, and what is done with them is
// what uattn_decode does with a bf16 cache, operation for operation and in the same
// order (uattn_numerics.h): the same products, tiles of 64 keys, chunks of 256,
// references, weights and fold.  So a row has the bits of uattn_decode over a bf16
// cache of the same values, and of uattn_prefill over those rows.
//
// One wave takes one item: (256-key chunk, kv head, entry), the G query heads of the
// kv head in the MFMA columns.  With a quarter (4 bits) of the bytes of a bf16 cache
// there is a quarter of the time for everything else, so an item has no barrier and
// shares nothing: its tiles one after another, each tile's codes in registers while
// the tile before is computed.
//
//   K  a lane (row r = lane % 16 of a 16-key block, group g = lane / 16) loads a quarter
//      of a row, D / 4 elements; the score product's operand wants of every 32-wide
//      step the g-th eight elements, which a 4 x 4 (D = 64: 2 x 4) transposition of
//      the words between the lane groups gives (permlane swaps), still as codes; the
//      conversion's result is the operand;
//   V  a lane (row lane / 4) loads a quarter of a row, converts it and writes it to
//      LDS as the rows that the transposing read of the P V product expects, 32 keys
//      at a time (a wave's own 8 KB, in order: no barrier).
//
// Entries of more than one chunk leave fp32 partials (m, l, acc) in the workspace, and
// a second kernel folds them in chunk order.
#include <type_traits>

#include "uattn_internal.h"
#include "uattn_mx.h"

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
};

// One tile's codes in this lane: its quarter rows of the four 16-key blocks and their scales.
template <int D, int KB, int VB>
struct TileCodes {
  uint32_t k[kKeyBlocks][MxRow<D, KB>::kWords];
  uint32_t v[kKeyBlocks][MxRow<D, VB>::kWords];
  uint32_t ks[kKeyBlocks];  // all scale bytes of row lane % 16
  uint32_t vs[kKeyBlocks];  // the scale byte of this lane's quarter of row lane / 4
};

template <int Words>
__device__ __forceinline__ void load_words(uint32_t (&w)[Words], __amdgpu_buffer_rsrc_t r, int off) {
  if constexpr (Words == 2) {
    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0));
    w[0] = x[0];
    w[1] = x[1];
  } else {
#pragma unroll
    for (int i = 0; i < Words / 4; ++i) {
      const u32x4 x = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off + 16 * i, 0, 0));
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

// Words of octet j of lane group g's quarter, octet kOcts * g + j of the row -> words
// of octet 4 * j + g: what step j of the score product wants of lane group g.
template <class R, int Words>
__device__ __forceinline__ void to_steps(uint32_t (&w)[Words]) {
  static_assert(Words == R::kWords, "a lane's quarter");
#pragma unroll
  for (int x = 0; x < R::kOctWords; ++x) {
    if constexpr (R::kOcts == 4) {
      uint32_t &r0 = w[x], &r1 = w[R::kOctWords + x], &r2 = w[2 * R::kOctWords + x], &r3 = w[3 * R::kOctWords + x];
      swap16(r0, r1);
      swap16(r2, r3);
      swap32(r0, r2);
      swap32(r1, r3);
    } else {
      uint32_t &r0 = w[x], &r1 = w[R::kOctWords + x];
      swap16(r0, r1);
      swap32(r0, r1);
    }
  }
}

template <int D, int NB, int KB, int VB>
__global__ __launch_bounds__(64) void decode_mx_kernel(DecodeMxParams p, const int32_t* __restrict__ seqlens,
                                                       const int32_t* __restrict__ block_table) {
  using TL = TileLayout<D>;
  using RK = MxRow<D, KB>;
  using RV = MxRow<D, VB>;
  constexpr int KS = D / 32;   // K steps of the score product
  constexpr int NDB = D / 16;  // d blocks of the output
  __shared__ __attribute__((aligned(1024))) __bf16 vrows[32 * D];

  const int lane = threadIdx.x;
  const int g = lane >> 4, col = lane & 15;
  // items of one chunk side by side for all kv heads, whose pages' parts lie side by side
  const int item = p.first + blockIdx.x;
  const int kvh = item % p.hkv;
  const int bc = item / p.hkv;
  const int chunk = bc % p.nchunk_max, b = bc / p.nchunk_max;
  const int n = min(seqlens[b], p.max_seqlen);
  if (chunk * kChunkKeys >= n) return;
  const int nch = (n + kChunkKeys - 1) / kChunkKeys;
  const int last_tile = (n - 1) / kTileKeys;

  // the pages of the chunk's sixteen 16-key blocks, one to a lane
  const int my_pos = chunk * kChunkKeys + 16 * col;
  const int my_page = block_table[static_cast<int64_t>(b) * p.maxp + min(my_pos >> p.page_shift, p.maxp - 1)];

  // query operands: column col of block nb, d = 32 * step + 8 * g .. + 7
  bf16x8 qf[NB][KS];
  {
    const __bf16* qb = p.q + (static_cast<int64_t>(b) * p.hq + kvh * p.group) * D;
    const auto rq = buffer_rsrc(qb, p.group * D * 2);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int st = 0; st < KS; ++st)
        qf[nb][st] = __builtin_bit_cast(
            bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rq, (nb * kQCols + col) * D * 2 + 16 * g + 64 * st, 0, 0));
  }

  // Tile t's codes.  Blocks past the context, on a page outside the pool or past the
  // table read as zeros (codes 0, scale byte 0) without touching memory.
  const int k_off = col * RK::kBytes + g * RK::kLaneBytes;
  const int v_row = lane >> 2, v_part = lane & 3;
  const int v_off = lane * RV::kLaneBytes;
  const int vs_off = v_row * RV::kScales + v_part * RV::kScales / 4;
  auto load_tile = [&](int t, TileCodes<D, KB, VB>& x) __attribute__((always_inline)) {
#pragma unroll
    for (int kb = 0; kb < kKeyBlocks; ++kb) {
      const int page = __builtin_amdgcn_readlane(my_page, 4 * t + kb);
      const int pos = chunk * kChunkKeys + t * kTileKeys + 16 * kb;
      const bool ok = page >= 0 && page < p.num_pages && pos < n;
      const int rows = ok ? min(n - pos, 16) : 0;
      const int64_t row =
          ok ? (((static_cast<int64_t>(page) * p.hkv + kvh) << p.page_shift) + (pos & (p.page_size - 1))) : 0;
      const auto rkc = buffer_rsrc(p.kc + row * RK::kBytes, rows * RK::kBytes);
      const auto rks = buffer_rsrc(p.ks + row * RK::kScales, rows * RK::kScales);
      const auto rvc = buffer_rsrc(p.vc + row * RV::kBytes, rows * RV::kBytes);
      const auto rvs = buffer_rsrc(p.vs + row * RV::kScales, rows * RV::kScales);
      load_words(x.k[kb], rkc, k_off);
      if constexpr (D == 128)
        x.ks[kb] = __builtin_amdgcn_raw_buffer_load_b32(rks, 4 * col, 0, 0);
      else
        x.ks[kb] = static_cast<uint16_t>(__builtin_amdgcn_raw_buffer_load_b16(rks, 2 * col, 0, 0));
      load_words(x.v[kb], rvc, v_off);
      x.vs[kb] = static_cast<uint8_t>(__builtin_amdgcn_raw_buffer_load_b8(rvs, vs_off, 0, 0));
    }
  };

  f32x4 acc[NB][NDB], lsum[NB];
  float m[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m[nb] = neg_inf();
    lsum[nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int db = 0; db < NDB; ++db) acc[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = static_cast<__bf16>(1.0f);

  auto compute_tile = [&](int t, TileCodes<D, KB, VB>& x) __attribute__((always_inline)) {
    const int tile = chunk * kTilesPerChunk + t;
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
        for (int st = 0; st < KS; ++st) r = mfma16(a[st], qf[nb][st], r);
        s[nb][kb] = r;
      }
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
      for (int half = 0; half < 2; ++half) {
        const int kb = 2 * st + half;
        const int row = 16 * half + v_row;
        const float scale = mx_scale(x.vs[kb]);
#pragma unroll
        for (int o = 0; o < RV::kOcts; ++o) {
          const int piece = (v_part * RV::kOcts + o) ^ TL::v_swz(row);
          *reinterpret_cast<bf16x8*>(vrows + row * D + 8 * piece) = mx_decode8<VB>(&x.v[kb][o * RV::kOctWords], scale);
        }
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

  TileCodes<D, KB, VB> x[2];
  load_tile(0, x[0]);
#pragma unroll
  for (int t = 0; t < kTilesPerChunk; ++t) {
    if (chunk * kTilesPerChunk + t > last_tile) break;
    if (t + 1 < kTilesPerChunk) load_tile(t + 1, x[(t + 1) & 1]);
    __builtin_amdgcn_sched_barrier(0);
    compute_tile(t, x[t & 1]);
  }

  if (nch == 1) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int gi = kQCols * nb + col;
      if (gi >= p.group) continue;
      const int64_t orow = static_cast<int64_t>(b) * p.hq + kvh * p.group + gi;
#pragma unroll
      for (int db = 0; db < NDB; ++db) {
        bf16x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = finalize_val(acc[nb][db][j], lsum[nb][0]);
        *reinterpret_cast<bf16x4*>(p.out + orow * D + 16 * db + 4 * g) = w;
      }
      if (p.lse != nullptr && g == 0) p.lse[orow] = finalize_lse(m[nb], lsum[nb][0], p.c);
    }
    return;
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int gi = kQCols * nb + col;
    if (gi >= p.group) continue;
    const int64_t slot = (static_cast<int64_t>(b) * p.hq + kvh * p.group + gi) * p.nslot + chunk;
#pragma unroll
    for (int db = 0; db < NDB; ++db) *reinterpret_cast<f32x4*>(p.ws_acc + slot * D + 16 * db + 4 * g) = acc[nb][db];
    if (g == 0) *reinterpret_cast<float2*>(p.ws_ml + slot * 2) = float2{m[nb], lsum[nb][0]};
  }
}

// Folds the partials of one (entry, q head) row in chunk order: D / 4 threads a row,
// four d each, kAhead chunks' partials in flight.
template <int D>
__global__ __launch_bounds__(256) void decode_mx_merge_kernel(DecodeMxParams p) {
  constexpr int kThreads = D / 4, kAhead = 16;
  const int64_t row = (static_cast<int64_t>(p.first) + blockIdx.x) * (256 / kThreads) + threadIdx.x / kThreads;
  if (row >= static_cast<int64_t>(p.batch) * p.hq) return;
  const int n = min(p.seqlens[row / p.hq], p.max_seqlen);
  const int nch = (n + kChunkKeys - 1) / kChunkKeys;
  if (nch < 2) return;  // the item wrote it (or the entry has no keys)
  const int d4 = 4 * (threadIdx.x % kThreads);
  const float* pa = p.ws_acc + row * p.nslot * D + d4;
  const float* pm = p.ws_ml + row * p.nslot * 2;
  float M = 0.f, L = 0.f;
  f32x4 A = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < nch; k0 += kAhead) {
    f32x4 x[kAhead];
    float2 ml[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int k = min(k0 + i, nch - 1);
      x[i] = *reinterpret_cast<const f32x4*>(pa + static_cast<int64_t>(k) * D);
      ml[i] = *reinterpret_cast<const float2*>(pm + 2 * k);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int k = k0 + i;
      if (k == 0) {
        M = ml[i].x;
        L = ml[i].y;
        A = x[i];
      } else if (k < nch) {
        const FoldScale f = fold_scale(M, ml[i].x, p.c);
        L = fold_val(f, L, ml[i].y);
#pragma unroll
        for (int j = 0; j < 4; ++j) A[j] = fold_val(f, A[j], x[i][j]);
        M = f.m_new;
      }
    }
  }
  bf16x4 o;
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] = finalize_val(A[j], L);
  *reinterpret_cast<bf16x4*>(p.out + row * D + d4) = o;
  if (p.lse != nullptr && d4 == 0) p.lse[row] = finalize_lse(M, L, p.c);
}

template <int D, int NB, int KB, int VB>
hipError_t launch(DecodeMxParams p, hipStream_t stream) {
  const int64_t items = static_cast<int64_t>(p.batch) * p.hkv * p.nchunk_max;
  const hipError_t e = launch_parts(items, 64, [&](int first, unsigned n) {
    p.first = first;
    hipLaunchKernelGGL((decode_mx_kernel<D, NB, KB, VB>), dim3(n), dim3(64), 0, stream, p, p.seqlens, p.bt);
  });
  if (e != hipSuccess || p.nchunk_max == 1) return e;
  constexpr int kRows = 256 / (D / 4);
  return launch_parts((static_cast<int64_t>(p.batch) * p.hq + kRows - 1) / kRows, 256, [&](int first, unsigned n) {
    p.first = first;
    hipLaunchKernelGGL(decode_mx_merge_kernel<D>, dim3(n), dim3(256), 0, stream, p);
  });
}

}  // namespace

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
  p.first = 0;
  p.c = a.c;
  using std::integral_constant;
  auto pick = [&](auto d, auto nb, auto kb, auto vb) {
    return launch<decltype(d)::value, decltype(nb)::value, decltype(kb)::value, decltype(vb)::value>(p, stream);
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
