// The KV cache held in 8 or 4 bits: new rows written as codes and scales, rows read
// back as bf16, and the values that a cache would hold for packed rows.
//
// All three move memory and compute next to nothing (a maximum and one conversion an
// element), so what they are built for is wide, coalesced access: a lane's accesses
// are 16 bytes of bf16, a wave's neighbours in memory.
#include "uattn_internal.h"
#include "uattn_mx.h"
#include "uattn_tile_io.h"

namespace uattn {
namespace {

struct KvMxParams {
  const __bf16* k;    // rows given (write, round)
  const __bf16* v;
  __bf16* k_out;      // rows made (read, round)
  __bf16* v_out;
  int64_t stride, out_stride;  // elements from token to token
  const int32_t* bt;
  const int32_t* seq_idx;
  const int32_t* positions;
  uint8_t* kc;
  uint8_t* ks;
  uint8_t* vc;
  uint8_t* vs;
  int first;          // workgroups (of grid.x) of the launches before this one
  int32_t num_tokens, batch, maxp, page_shift, num_pages, hkv;
  bool places;        // there are a table and pages
};

// Row of the pools (codes and scales alike) that holds token n for kv head 0, or -1
// for a token that has no place.  Without branches, so that the loads of several tokens
// go together; where there is no place its loads are those of the table's first entry.
__device__ __forceinline__ int64_t pool_row(const KvMxParams& p, int64_t n) {
  const int32_t pos = p.positions[n];
  const int32_t s = p.seq_idx[n];
  const int32_t lp = pos >> p.page_shift;
  const bool ok = pos >= 0 && s >= 0 && s < p.batch && lp < p.maxp;
  const int32_t page = p.bt[ok ? static_cast<int64_t>(s) * p.maxp + lp : 0];
  const int64_t row = ((static_cast<int64_t>(page) * p.hkv) << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
  return ok && page >= 0 && page < p.num_pages ? row : -1;
}

// kStreamed: past the caches.
template <bool kStreamed>
__device__ __forceinline__ u32x4 load16(const __bf16* at) {
  if constexpr (kStreamed) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at));
  return *reinterpret_cast<const u32x4*>(at);
}
template <bool kStreamed>
__device__ __forceinline__ void store16(__bf16* at, const bf16x8& x) {
  if constexpr (kStreamed)
    __builtin_nontemporal_store(x, reinterpret_cast<bf16x8*>(at));
  else
    *reinterpret_cast<bf16x8*>(at) = x;
}

// The largest magnitude of a block whose elements four lanes hold, eight each.
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
  m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0xB1 /* quad_perm 1 0 3 2 */, 0xF, 0xF, true)));
  return max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0x4E /* quad_perm 2 3 0 1 */, 0xF, 0xF, true)));
}

// The scale byte of the block that lane x's four lanes hold.
template <int Bits>
__device__ __forceinline__ uint32_t block_scale(const u32x4& x) {
  const uint32_t m = mx_max_mag(mx_max_mag(mx_max_mag(0, x[0]), x[1]), mx_max_mag(mx_max_mag(0, x[2]), x[3]));
  return mx_scale_byte<Bits>(quad_max(max(m & 0xFFFFu, m >> 16)));
}

// Write: a lane takes eight elements, four lanes a block, a wave the rows of one kv head of
// 64 / (D / 8) consecutive tokens in each of its rounds.  24,000 tokens of 8 heads of 128: 26
// us in 4 bits (123 MB, 4.7 TB/s), 29 in 8 (147 MB).  A lane to a block, without exchanges
// and with scale bytes side by side: 26 and 32, as its loads, 64 bytes apart, cannot be
// streamed; 64 tokens 2.8 us, so 2.6.
constexpr int write_rounds(bool streamed) { return streamed ? 2 : 1; }
template <int D, int Bits>
__device__ __forceinline__ void write8(const u32x4& x, uint8_t* codes, uint8_t* scales, int64_t row, int piece) {
  const uint32_t byte = block_scale<Bits>(x);
  // a block that reads as NaN: any codes would do, zeros are stored
  MxWords<Bits> w = mx_encode8<Bits>(x, mx_scale(byte == kMxNan ? 127 : byte));
  if (byte == kMxNan) w = {};
  __builtin_memcpy(codes + row * (D * Bits / 8) + piece * Bits, w.w, Bits);
  if (piece % 4 == 0) scales[row * (D / kMxBlock) + piece / 4] = static_cast<uint8_t>(byte);
}

template <int D, int KB, int VB, bool kStreamed>
__global__ __launch_bounds__(256) void kv_write_mx_kernel(KvMxParams p) {
  constexpr int kPieces = D / 8, kTokens = 64 / kPieces, kWriteRounds = write_rounds(kStreamed);
  const int lane = threadIdx.x & 63;
  const int h = blockIdx.y * (blockDim.x >> 6) + (threadIdx.x >> 6), piece = lane % kPieces;
  if (h >= p.hkv) return;
  const int64_t n0 = (static_cast<int64_t>(p.first) + blockIdx.x) * (kTokens * kWriteRounds) + lane / kPieces;
  u32x4 k[kWriteRounds], v[kWriteRounds];
  int64_t row[kWriteRounds];
#pragma unroll
  for (int r = 0; r < kWriteRounds; ++r) {
    const int64_t n = n0 + r * kTokens, at = n < p.num_tokens ? n : p.num_tokens - 1;
    const int64_t src = at * p.stride + h * D + piece * 8;
    k[r] = load16<kStreamed>(p.k + src);
    v[r] = load16<kStreamed>(p.v + src);
    row[r] = n < p.num_tokens ? pool_row(p, at) : -1;
  }
#pragma unroll
  for (int r = 0; r < kWriteRounds; ++r) {
    if (row[r] < 0) continue;  // (a block's four lanes are of one token)
    const int64_t at = row[r] + (static_cast<int64_t>(h) << p.page_shift);
    write8<D, KB>(k[r], p.kc, p.ks, at, piece);
    write8<D, VB>(v[r], p.vc, p.vs, at, piece);
  }
}

// Read: a lane makes eight elements, a wave 64 / (D / 8) tokens' rows of one kv head
// in each of its kRounds rounds.  A token without a place gets zeros.  64,000 tokens of 8
// heads of 128, keys in 8 bits, values in 4 (365 MB): 68 us, 5.4 TB/s; 77 where the rows go
// through the caches.
constexpr int kRounds = 2;
template <int D, int KB, int VB, bool kStreamed>
__global__ __launch_bounds__(256) void kv_read_mx_kernel(KvMxParams p) {
  constexpr int kPieces = D / 8, kTokens = 64 / kPieces;
  const int lane = threadIdx.x & 63;
  const int h = blockIdx.y * (blockDim.x >> 6) + (threadIdx.x >> 6), piece = lane % kPieces;
  if (h >= p.hkv) return;
  const int64_t n0 = (static_cast<int64_t>(p.first) + blockIdx.x) * (kTokens * kRounds) + lane / kPieces;
  int64_t row[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t n = n0 + r * kTokens;
    row[r] = p.places ? pool_row(p, n < p.num_tokens ? n : p.num_tokens - 1) : -1;
  }
  MxWords<KB> kw[kRounds];
  MxWords<VB> vw[kRounds];
  uint32_t ks[kRounds], vs[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    kw[r] = {};
    vw[r] = {};
    ks[r] = vs[r] = 0;
    if (p.places) {
      const int64_t at = row[r] < 0 ? 0 : row[r] + (static_cast<int64_t>(h) << p.page_shift);
      __builtin_memcpy(kw[r].w, p.kc + at * (D * KB / 8) + piece * KB, KB);
      __builtin_memcpy(vw[r].w, p.vc + at * (D * VB / 8) + piece * VB, VB);
      ks[r] = p.ks[at * (D / kMxBlock) + piece / 4];
      vs[r] = p.vs[at * (D / kMxBlock) + piece / 4];
    }
  }
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t n = n0 + r * kTokens;
    if (n >= p.num_tokens) return;
    bf16x8 k = mx_decode8<KB>(kw[r].w, mx_scale(ks[r])), v = mx_decode8<VB>(vw[r].w, mx_scale(vs[r]));
    if (row[r] < 0) k = v = bf16x8{};
    const int64_t dst = n * p.out_stride + h * D + piece * 8;
    store16<kStreamed>(p.k_out + dst, k);
    store16<kStreamed>(p.v_out + dst, v);
  }
}

// Round: a lane takes eight elements, four lanes a block.
template <int Bits>
__device__ __forceinline__ bf16x8 round8(const u32x4& x) {
  const uint32_t byte = block_scale<Bits>(x);
  // (of a block that reads as NaN the codes do not matter)
  const MxWords<Bits> w = mx_encode8<Bits>(x, mx_scale(byte == kMxNan ? 127 : byte));
  return mx_decode8<Bits>(w.w, mx_scale(byte));
}

// A workgroup takes `tokens` tokens of `pieces` 16-byte pieces each, kAhead pieces of a
// lane on their way.  pieces is a multiple of 8, so a block's four lanes are of one row
// and in or out of the range together.  39,855 tokens of 8 heads of 128 (326 MB): 55 us,
// 5.9 TB/s; 62 through the caches.
constexpr int round_ahead(bool streamed) { return streamed ? 2 : 1; }
template <int KB, int VB, bool kStreamed>
__global__ __launch_bounds__(256) void kv_round_mx_kernel(KvMxParams p, Divider pieces, int tokens) {
  constexpr int kAhead = round_ahead(kStreamed);
  const int64_t n0 = (static_cast<int64_t>(p.first) + blockIdx.x) * tokens;
  const int left = static_cast<int>(min(static_cast<int64_t>(tokens), p.num_tokens - n0));
  const uint32_t count = static_cast<uint32_t>(left) * pieces.d;
  const __bf16* k = p.k + n0 * p.stride;
  const __bf16* v = p.v + n0 * p.stride;
  __bf16* ko = p.k_out + n0 * p.out_stride;
  __bf16* vo = p.v_out + n0 * p.out_stride;
  for (uint32_t i0 = threadIdx.x; i0 < count; i0 += 256 * kAhead) {
    u32x4 x[kAhead], y[kAhead];
    int64_t to[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const uint32_t i = i0 + 256 * j;
      if (i < count) {
        const DivMod at = divide(i, pieces);
        const int64_t from = at.q * p.stride + 8 * at.r;
        to[j] = at.q * p.out_stride + 8 * at.r;
        x[j] = load16<kStreamed>(k + from);
        y[j] = load16<kStreamed>(v + from);
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (i0 + 256 * j < count) {
        store16<kStreamed>(ko + to[j], round8<KB>(x[j]));
        store16<kStreamed>(vo + to[j], round8<VB>(y[j]));
      }
    }
  }
}

KvMxParams params(const KvMxLaunch& a) {
  KvMxParams p;
  p.k = static_cast<const __bf16*>(a.k);
  p.v = static_cast<const __bf16*>(a.v);
  p.k_out = static_cast<__bf16*>(a.k_out);
  p.v_out = static_cast<__bf16*>(a.v_out);
  p.stride = a.token_stride;
  p.out_stride = a.out_stride;
  p.bt = a.block_table;
  p.seq_idx = a.seq_idx;
  p.positions = a.positions;
  p.kc = static_cast<uint8_t*>(a.cache.k_codes);
  p.ks = static_cast<uint8_t*>(a.cache.k_scales);
  p.vc = static_cast<uint8_t*>(a.cache.v_codes);
  p.vs = static_cast<uint8_t*>(a.cache.v_scales);
  p.first = 0;
  p.num_tokens = a.num_tokens;
  p.batch = a.batch;
  p.maxp = a.max_pages_per_seq;
  p.page_shift = a.page_size > 0 ? __builtin_ctz(static_cast<unsigned>(a.page_size)) : 0;
  p.num_pages = a.num_pages;
  p.hkv = a.num_kv_heads;
  p.places = a.batch > 0 && a.max_pages_per_seq > 0 && a.num_pages > 0;
  return p;
}

// Calls f with the head size and the two code sizes as constants.
template <class F>
hipError_t with_bits(const MxCache& c, const F& f) {
  using std::integral_constant;
  const integral_constant<int, 8> b8;
  const integral_constant<int, 4> b4;
  if (c.k_bits == 8) return c.v_bits == 8 ? f(b8, b8) : f(b8, b4);
  return c.v_bits == 8 ? f(b4, b8) : f(b4, b4);
}

// Launches f(grid, threads) over workgroups of up to four waves, a kv head to a wave,
// grid.x over runs of `tokens` tokens.
template <class F>
hipError_t per_head(const KvMxLaunch& a, KvMxParams& p, int tokens, const F& f) {
  const int waves = a.num_kv_heads < 4 ? a.num_kv_heads : 4;
  const unsigned groups = (a.num_kv_heads + waves - 1) / waves;
  return launch_parts((static_cast<int64_t>(a.num_tokens) + tokens - 1) / tokens, 64 * waves * groups, [&](int first, unsigned n) {
    p.first = first;
    f(dim3(n, groups), dim3(64 * waves));
  });
}

// The keys' rows as bf16, or the values'.
int64_t rows_bytes(const KvMxLaunch& a) { return int64_t{2} * a.num_tokens * a.num_kv_heads * a.head_dim; }
// Outputs of 64 MB and more go past the caches, as other rows do.
bool streamed(const KvMxLaunch& a) { return rows_bytes(a) >= int64_t{64} << 20; }

}  // namespace

hipError_t launch_kv_write_mx(const KvMxLaunch& a, hipStream_t stream) {
  KvMxParams p = params(a);
  return with_bits(a.cache, [&](auto kb, auto vb) {
    constexpr int KB = decltype(kb)::value, VB = decltype(vb)::value;
    auto run = [&](auto k128, auto k64, int rounds) {
      return per_head(a, p, rounds * 64 * 8 / a.head_dim, [&](dim3 grid, dim3 threads) {
        hipLaunchKernelGGL(a.head_dim == 128 ? k128 : k64, grid, threads, 0, stream, p);
      });
    };
    // (rows of 4 MB that the caches hold are better read through them: 3.4 us, 4.3)
    return rows_bytes(a) >= int64_t{16} << 20
               ? run(kv_write_mx_kernel<128, KB, VB, true>, kv_write_mx_kernel<64, KB, VB, true>, write_rounds(true))
               : run(kv_write_mx_kernel<128, KB, VB, false>, kv_write_mx_kernel<64, KB, VB, false>, write_rounds(false));
  });
}

hipError_t launch_kv_read_mx(const KvMxLaunch& a, hipStream_t stream) {
  KvMxParams p = params(a);
  return with_bits(a.cache, [&](auto kb, auto vb) {
    constexpr int KB = decltype(kb)::value, VB = decltype(vb)::value;
    auto run = [&](auto k128, auto k64) {
      return per_head(a, p, kRounds * 64 * 8 / a.head_dim, [&](dim3 grid, dim3 threads) {
        hipLaunchKernelGGL(a.head_dim == 128 ? k128 : k64, grid, threads, 0, stream, p);
      });
    };
    return streamed(a) ? run(kv_read_mx_kernel<128, KB, VB, true>, kv_read_mx_kernel<64, KB, VB, true>)
                      : run(kv_read_mx_kernel<128, KB, VB, false>, kv_read_mx_kernel<64, KB, VB, false>);
  });
}

hipError_t launch_kv_round_mx(const KvMxLaunch& a, hipStream_t stream) {
  KvMxParams p = params(a);
  const int pieces = a.num_kv_heads * a.head_dim / 8;
  const int per_group = 256 * round_ahead(streamed(a));
  const int tokens = pieces < per_group ? per_group / pieces : 1;
  return with_bits(a.cache, [&](auto kb, auto vb) {
    constexpr int KB = decltype(kb)::value, VB = decltype(vb)::value;
    return launch_parts((static_cast<int64_t>(a.num_tokens) + tokens - 1) / tokens, 256, [&](int first, unsigned n) {
      p.first = first;
      hipLaunchKernelGGL((streamed(a) ? kv_round_mx_kernel<KB, VB, true> : kv_round_mx_kernel<KB, VB, false>), dim3(n), dim3(256), 0,
                         stream, p, divider(pieces), tokens);
    });
  });
}

}  // namespace uattn
