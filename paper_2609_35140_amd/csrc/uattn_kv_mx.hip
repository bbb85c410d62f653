// The KV cache held in 8 or 4 bits: new rows written as codes and scales, rows read
// back as bf16, and the values that a cache would hold for packed rows.
//
// All three move memory and compute next to nothing (a maximum and one conversion an
// element), so what they are built for is wide, coalesced access: a lane's accesses
// are 16 bytes of bf16, a wave's neighbours in memory.
#include "uattn_internal.h"
#include "uattn_mx.h"

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
  int64_t first;      // workgroups of the launches before this one
  int32_t num_tokens, batch, maxp, page_shift, num_pages, hkv;
};

// Row of the pools (codes and scales alike) that holds token n for kv head 0, or -1
// for a token that has no place.
__device__ __forceinline__ int64_t pool_row(const KvMxParams& p, int64_t n) {
  const int32_t pos = p.positions[n];
  const int32_t s = p.seq_idx[n];
  if (pos < 0 || s < 0 || s >= p.batch) return -1;
  const int32_t lp = pos >> p.page_shift;
  if (lp >= p.maxp) return -1;
  const int32_t page = p.bt[static_cast<int64_t>(s) * p.maxp + lp];
  if (page < 0 || page >= p.num_pages) return -1;
  return ((static_cast<int64_t>(page) * p.hkv) << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
}

// Write: a lane takes one block of one row, a wave the rows of one kv head of 64 / (D
// / 32) consecutive tokens, so that consecutive positions' codes and scale bytes are
// one run of stores in the cache's pages (position after position of a head).
template <int D, int Bits>
__device__ __forceinline__ void write_block(const __bf16* src, uint8_t* codes, uint8_t* scales, int64_t row, int block) {
  constexpr int kRowBytes = D * Bits / 8, kBytes = kMxBlock * Bits / 8;
  u32x4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const u32x4*>(src + 8 * i);
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) m = mx_max_mag(m, x[i][j]);
  const uint32_t byte = mx_scale_byte<Bits>(max(m & 0xFFFFu, m >> 16));
  // a block that reads as NaN: any codes would do, zeros are stored
  const float scale = mx_scale(byte == kMxNan ? 127 : byte);
  u32x4 out[Bits / 4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const MxWords<Bits> w = mx_encode8<Bits>(x[i], scale);
#pragma unroll
    for (int j = 0; j < Bits / 4; ++j) {
      const int k = i * (Bits / 4) + j;
      out[k / 4][k % 4] = byte == kMxNan ? 0u : w.w[j];
    }
  }
  uint8_t* dst = codes + row * kRowBytes + block * kBytes;
#pragma unroll
  for (int i = 0; i < Bits / 4; ++i) *reinterpret_cast<u32x4*>(dst + 16 * i) = out[i];
  scales[row * (D / kMxBlock) + block] = static_cast<uint8_t>(byte);
}

template <int D, int KB, int VB>
__global__ __launch_bounds__(256) void kv_write_mx_kernel(KvMxParams p) {
  constexpr int kBlocks = D / kMxBlock, kTokens = 64 / kBlocks;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (p.first + blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t n = unit / p.hkv * kTokens + lane / kBlocks;
  const int h = static_cast<int>(unit % p.hkv), block = lane % kBlocks;
  if (n >= p.num_tokens) return;
  int64_t row = pool_row(p, n);
  if (row < 0) return;
  row += static_cast<int64_t>(h) << p.page_shift;
  const int64_t src = n * p.stride + h * D + block * kMxBlock;
  write_block<D, KB>(p.k + src, p.kc, p.ks, row, block);
  write_block<D, VB>(p.v + src, p.vc, p.vs, row, block);
}

// Read: a lane makes eight elements, a wave 64 / (D / 8) tokens' rows of one kv head
// in each of its kRounds rounds.  A token without a place gets zeros.
template <int D, int KB, int VB>
__global__ __launch_bounds__(256) void kv_read_mx_kernel(KvMxParams p) {
  constexpr int kPieces = D / 8, kTokens = 64 / kPieces, kRounds = 4;
  const int lane = threadIdx.x & 63;
  const int64_t unit = (p.first + blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int64_t n0 = unit / p.hkv * (kTokens * kRounds) + lane / kPieces;
  const int h = static_cast<int>(unit % p.hkv), piece = lane % kPieces;
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int64_t n = n0 + r * kTokens;
    if (n >= p.num_tokens) return;
    int64_t row = pool_row(p, n);
    bf16x8 k = {}, v = {};
    if (row >= 0) {
      row += static_cast<int64_t>(h) << p.page_shift;
      const int64_t srow = row * (D / kMxBlock) + piece / 4;
      MxWords<KB> kw;
      MxWords<VB> vw;
      __builtin_memcpy(kw.w, p.kc + row * (D * KB / 8) + piece * KB, KB);
      __builtin_memcpy(vw.w, p.vc + row * (D * VB / 8) + piece * VB, VB);
      k = mx_decode8<KB>(kw.w, mx_scale(p.ks[srow]));
      v = mx_decode8<VB>(vw.w, mx_scale(p.vs[srow]));
    }
    const int64_t dst = n * p.out_stride + h * D + piece * 8;
    *reinterpret_cast<bf16x8*>(p.k_out + dst) = k;
    *reinterpret_cast<bf16x8*>(p.v_out + dst) = v;
  }
}

// Round: a lane takes eight elements, four lanes a block; the block's maximum by two
// exchanges between them.
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
  m = max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0xB1 /* quad_perm 1 0 3 2 */, 0xF, 0xF, true)));
  return max(m, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(m), 0x4E /* quad_perm 2 3 0 1 */, 0xF, 0xF, true)));
}

template <int Bits>
__device__ __forceinline__ bf16x8 round8(const u32x4& x) {
  const uint32_t m = mx_max_mag(mx_max_mag(mx_max_mag(0, x[0]), x[1]), mx_max_mag(mx_max_mag(0, x[2]), x[3]));
  const uint32_t byte = mx_scale_byte<Bits>(quad_max(max(m & 0xFFFFu, m >> 16)));
  // (of a block that reads as NaN the codes do not matter)
  const MxWords<Bits> w = mx_encode8<Bits>(x, mx_scale(byte == kMxNan ? 127 : byte));
  return mx_decode8<Bits>(w.w, mx_scale(byte));
}

template <int KB, int VB>
__global__ __launch_bounds__(256) void kv_round_mx_kernel(KvMxParams p, int pieces) {
  const int64_t i = (p.first + blockIdx.x) * 256 + threadIdx.x;
  const int64_t n = i / pieces;  // pieces is a multiple of 8: a block's four lanes are of one row
  if (n >= p.num_tokens) return;
  const int64_t at = (i - n * pieces) * 8;
  const u32x4 k = *reinterpret_cast<const u32x4*>(p.k + n * p.stride + at);
  const u32x4 v = *reinterpret_cast<const u32x4*>(p.v + n * p.stride + at);
  *reinterpret_cast<bf16x8*>(p.k_out + n * p.out_stride + at) = round8<KB>(k);
  *reinterpret_cast<bf16x8*>(p.v_out + n * p.out_stride + at) = round8<VB>(v);
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

// Workgroups of four waves, each a kv head of `tokens` tokens.
int64_t workgroups(const KvMxLaunch& a, int tokens) {
  const int64_t units = (static_cast<int64_t>(a.num_tokens) + tokens - 1) / tokens * a.num_kv_heads;
  return (units + 3) / 4;
}

}  // namespace

hipError_t launch_kv_write_mx(const KvMxLaunch& a, hipStream_t stream) {
  KvMxParams p = params(a);
  return with_bits(a.cache, [&](auto kb, auto vb) {
    constexpr int KB = decltype(kb)::value, VB = decltype(vb)::value;
    return launch_parts(workgroups(a, 64 * kMxBlock / a.head_dim), 256, [&](int first, unsigned n) {
      p.first = first;
      if (a.head_dim == 128)
        hipLaunchKernelGGL((kv_write_mx_kernel<128, KB, VB>), dim3(n), dim3(256), 0, stream, p);
      else
        hipLaunchKernelGGL((kv_write_mx_kernel<64, KB, VB>), dim3(n), dim3(256), 0, stream, p);
    });
  });
}

hipError_t launch_kv_read_mx(const KvMxLaunch& a, hipStream_t stream) {
  KvMxParams p = params(a);
  return with_bits(a.cache, [&](auto kb, auto vb) {
    constexpr int KB = decltype(kb)::value, VB = decltype(vb)::value;
    return launch_parts(workgroups(a, 4 * 64 * 8 / a.head_dim), 256, [&](int first, unsigned n) {
      p.first = first;
      if (a.head_dim == 128)
        hipLaunchKernelGGL((kv_read_mx_kernel<128, KB, VB>), dim3(n), dim3(256), 0, stream, p);
      else
        hipLaunchKernelGGL((kv_read_mx_kernel<64, KB, VB>), dim3(n), dim3(256), 0, stream, p);
    });
  });
}

hipError_t launch_kv_round_mx(const KvMxLaunch& a, hipStream_t stream) {
  KvMxParams p = params(a);
  const int pieces = a.num_kv_heads * a.head_dim / 8;
  return with_bits(a.cache, [&](auto kb, auto vb) {
    constexpr int KB = decltype(kb)::value, VB = decltype(vb)::value;
    return launch_parts((static_cast<int64_t>(a.num_tokens) * pieces + 255) / 256, 256, [&](int first, unsigned n) {
      p.first = first;
      hipLaunchKernelGGL((kv_round_mx_kernel<KB, VB>), dim3(n), dim3(256), 0, stream, p, pieces);
    });
  });
}

}  // namespace uattn
