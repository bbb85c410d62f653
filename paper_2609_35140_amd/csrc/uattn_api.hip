// extern "C" boundary of libuattn: argument validation, grid sizing and
// launch on the caller's stream.  No allocation, no synchronization (except
// the opt-in UATTN_VALIDATE debug copies), no global mutable state.
#include <stdlib.h>
#include <string.h>

#include "../../include/uattn.h"
#include "uattn_internal.h"
#include "uattn_numerics.h"

namespace {

using uattn::kChunkKeys;

constexpr double kLog2e = 1.4426950408889634;

bool scale_ok(float s) { return s > 0.f && s < __builtin_inff(); }

bool validate_env() {
  const char* e = getenv("UATTN_VALIDATE");
  return e != nullptr && e[0] != '\0' && e[0] != '0';
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// fp32(scale * log2(e)), the one constant both attention paths fold into exp2.
float exp2_scale(float softmax_scale) { return static_cast<float>(static_cast<double>(softmax_scale) * kLog2e); }

bool is_finite(float x) { return x - x == 0.f; }

// A device array copied back for UATTN_VALIDATE, behind what the call's stream holds already; host is nullptr where
// that fails, as in a stream that is being captured, which runs nothing before its graph does.
template <class T>
struct Copied {
  T* host;
  Copied(const T* dev, size_t n, void* stream) : host(static_cast<T*>(malloc(n > 0 ? n * sizeof(T) : 1))) {
    if (host == nullptr || n == 0) return;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(st, &capture) == hipSuccess && capture == hipStreamCaptureStatusNone &&
        hipMemcpyAsync(host, dev, n * sizeof(T), hipMemcpyDeviceToHost, st) == hipSuccess &&
        hipStreamSynchronize(st) == hipSuccess)
      return;
    (void)hipGetLastError();  // not the next launch's error
    free(host);
    host = nullptr;
  }
  ~Copied() { free(host); }
  Copied(const Copied&) = delete;
  Copied& operator=(const Copied&) = delete;
};

bool all_below(const int32_t* dev, int32_t n, int32_t limit, void* stream) {
  Copied<int32_t> c(dev, static_cast<size_t>(n), stream);
  if (c.host == nullptr) return false;
  for (int32_t i = 0; i < n; ++i)
    if (c.host[i] >= limit) return false;
  return true;
}

// Widths a row of the residual norm may have: 16-byte pieces, held by one workgroup's registers.
bool norm_width_ok(int32_t hidden_dim) { return hidden_dim % 8 == 0 && hidden_dim <= 16384; }

constexpr int32_t kMaxSortedTokens = 1 << 30;
// Past these the kernels' 32-bit columns of a row, and places in the lists of tokens and biases, could overflow.
constexpr int32_t kMaxEmbeddingWidth = 1 << 20;
constexpr int32_t kMaxListed = 1 << 30;

// Ranges [begin, end) of `width` columns: column 0 to the last ascending, inside [0, limit].
bool ranges_ok(const int32_t* dev, int32_t rows, int width, int32_t limit, void* stream) {
  Copied<int32_t> c(dev, static_cast<size_t>(rows) * width, stream);
  if (c.host == nullptr) return false;
  for (size_t r = 0; r < static_cast<size_t>(rows); ++r) {
    int32_t least = 0;
    for (int k = 0; k < width; ++k) {
      const int32_t v = c.host[r * width + k];
      if (v < least || v > limit) return false;
      least = v;
    }
  }
  return true;
}

// Targets inside the vocabulary.
bool targets_ok(const int32_t* dev, int32_t n, int32_t vocab, void* stream) {
  Copied<int32_t> c(dev, static_cast<size_t>(n), stream);
  if (c.host == nullptr) return false;
  for (int32_t i = 0; i < n; ++i)
    if (c.host[i] < 0 || c.host[i] >= vocab) return false;
  return true;
}

// Offsets of packed sequences: from 0 to total_tokens, no sequence longer than max_seqlen.
bool offsets_ok(const int32_t* dev, int32_t num_seqs, int32_t total_tokens, int32_t max_seqlen, void* stream) {
  Copied<int32_t> c(dev, static_cast<size_t>(num_seqs) + 1, stream);
  if (c.host == nullptr || c.host[0] != 0 || c.host[num_seqs] != total_tokens) return false;
  for (int32_t s = 0; s < num_seqs; ++s) {
    const int64_t len = static_cast<int64_t>(c.host[s + 1]) - c.host[s];
    if (len < 0 || len > max_seqlen) return false;
  }
  return true;
}

// Every token that is not padding has a place in the table and the pool.
bool places_ok(const int32_t* block_table, const int32_t* seq_idx, const int32_t* positions, int32_t num_tokens,
               int32_t batch, int32_t max_pages_per_seq, int32_t page_size, int32_t num_pages, void* stream) {
  Copied<int32_t> si(seq_idx, static_cast<size_t>(num_tokens), stream);
  Copied<int32_t> ps(positions, static_cast<size_t>(num_tokens), stream);
  Copied<int32_t> bt(block_table, static_cast<size_t>(batch) * max_pages_per_seq, stream);
  if (si.host == nullptr || ps.host == nullptr || bt.host == nullptr) return false;
  for (int32_t n = 0; n < num_tokens; ++n) {
    const int32_t seq = si.host[n], pos = ps.host[n];
    if (pos < 0) continue;
    if (seq < 0 || seq >= batch || pos / page_size >= max_pages_per_seq) return false;
    const int32_t pg = bt.host[static_cast<size_t>(seq) * max_pages_per_seq + pos / page_size];
    if (pg < 0 || pg >= num_pages) return false;
  }
  return true;
}

bool bits_ok(int32_t k_bits, int32_t v_bits) { return (k_bits == 8 || k_bits == 4) && (v_bits == 8 || v_bits == 4); }

// Token rows of the heads of one tensor, `stride` elements apart.
bool row_stride_ok(int64_t stride, int32_t num_kv_heads, int32_t head_dim) {
  return stride >= static_cast<int64_t>(num_kv_heads) * head_dim && stride % 8 == 0;
}

// What the logit processing and its gradient ask of their common arguments.
uattn_status check_logits(const uattn::LogitsLaunch& a, bool grad, void* stream) {
  if (a.num_rows < 0 || a.vocab <= 0 || a.num_tokens < 0 || a.num_bias < 0 || a.num_masks < 0) return UATTN_EINVAL;
  if (a.logits_stride < a.vocab || (a.logits_stride % 8) != 0 || a.out_stride < a.vocab || (a.out_stride % 8) != 0)
    return UATTN_EINVAL;
  if ((a.history == nullptr) != (a.penalties == nullptr)) return UATTN_EINVAL;
  if (a.history != nullptr && a.num_tokens > 0 && a.tokens == nullptr) return UATTN_EINVAL;
  if (a.bias_rows != nullptr && a.num_bias > 0 && (a.bias_ids == nullptr || a.bias_values == nullptr))
    return UATTN_EINVAL;
  if (a.mask != nullptr && a.mask_stride < (static_cast<int64_t>(a.vocab) + 31) / 32) return UATTN_EINVAL;
  if (a.mask != nullptr && a.mask_rows == nullptr && a.num_masks < a.num_rows) return UATTN_EINVAL;
  if (a.num_tokens > kMaxListed || a.num_bias > kMaxListed) return UATTN_EUNSUPPORTED;
  if (a.num_rows == 0) return UATTN_OK;
  if (!a.logits || !a.out || !aligned16(a.logits) || !aligned16(a.out)) return UATTN_EINVAL;
  // in place the rows have to stay where they are: workgroups read others while this one writes
  const void* in = grad ? a.dout : a.logits;
  if (in == a.out && (grad ? a.dout_stride : a.logits_stride) != a.out_stride && a.num_rows > 1) return UATTN_EINVAL;
  if (validate_env()) {
    if (a.history != nullptr && !ranges_ok(a.history, a.num_rows, 3, a.num_tokens, stream)) return UATTN_EINVAL;
    if (a.bias_rows != nullptr && !ranges_ok(a.bias_rows, a.num_rows, 2, a.num_bias, stream)) return UATTN_EINVAL;
    if (a.mask != nullptr && a.mask_rows != nullptr && !all_below(a.mask_rows, a.num_rows, a.num_masks, stream))
      return UATTN_EINVAL;
  }
  return UATTN_OK;
}

}  // namespace

namespace uattn {
int32_t device_cus() {
  static int32_t cached[64] = {0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  if (cached[dev] > 0) return cached[dev];
  int n = 0;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
  cached[dev] = n;
  return n;
}
}  // namespace uattn

extern "C" {

int32_t uattn_abi_version(void) { return UATTN_ABI_VERSION; }

const char* uattn_status_string(int32_t status) {
  switch (status) {
    case UATTN_OK: return "UATTN_OK";
    case UATTN_EINVAL: return "UATTN_EINVAL: invalid argument";
    case UATTN_EUNSUPPORTED: return "UATTN_EUNSUPPORTED: unsupported shape";
    case UATTN_EWORKSPACE: return "UATTN_EWORKSPACE: workspace missing or too small";
    case UATTN_ELAUNCH: return "UATTN_ELAUNCH: kernel launch failed";
    case UATTN_ESCRATCH: return "UATTN_ESCRATCH: these sizes need more decode scratch than the library's static array holds";
    default: return "UATTN_UNKNOWN_STATUS";
  }
}

uattn_status uattn_prefill(const void* q, const void* k, const void* v, const int32_t* cu_seqlens, int32_t num_seqs,
                           int32_t total_tokens, int32_t max_seqlen, int32_t num_q_heads, int32_t num_kv_heads,
                           int32_t head_dim, float softmax_scale, void* out, float* lse, void* stream) {
  if (num_seqs < 0 || total_tokens < 0 || max_seqlen < 0 || num_q_heads <= 0 || num_kv_heads <= 0)
    return UATTN_EINVAL;
  if (num_q_heads % num_kv_heads != 0 || !scale_ok(softmax_scale)) return UATTN_EINVAL;
  if (head_dim != 64 && head_dim != 128) return UATTN_EUNSUPPORTED;
  if (num_seqs > 65535) return UATTN_EUNSUPPORTED;
  if (num_seqs == 0 || total_tokens == 0 || max_seqlen == 0) return UATTN_OK;
  if (!q || !k || !v || !cu_seqlens || !out) return UATTN_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return UATTN_EINVAL;
  if (validate_env() && !offsets_ok(cu_seqlens, num_seqs, total_tokens, max_seqlen, stream)) return UATTN_EINVAL;
  uattn::PrefillLaunch a;
  a.q = q;
  a.k = k;
  a.v = v;
  a.cu_seqlens = cu_seqlens;
  a.out = out;
  a.lse = lse;
  a.num_seqs = num_seqs;
  a.total_tokens = total_tokens;
  a.max_seqlen = max_seqlen;
  a.num_q_heads = num_q_heads;
  a.num_kv_heads = num_kv_heads;
  a.head_dim = head_dim;
  a.c = exp2_scale(softmax_scale);
  return uattn::launch_prefill(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

size_t uattn_decode_workspace_bytes(int32_t batch, int32_t max_seqlen, int32_t num_q_heads, int32_t head_dim) {
  if (batch <= 0 || max_seqlen <= 0 || num_q_heads <= 0 || head_dim <= 0) return 0;
  const int64_t nchunk = (static_cast<int64_t>(max_seqlen) + kChunkKeys - 1) / kChunkKeys;
  if (nchunk <= 1) return 0;
  return uattn::decode_ws_cnt_bytes(batch, num_q_heads) +
         uattn::decode_ws_acc_bytes(batch, nchunk, num_q_heads, head_dim) +
         uattn::decode_ws_ml_bytes(batch, nchunk, num_q_heads);
}

}  // extern "C"

namespace uattn {
uattn_status decode_prepare(const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                            const int32_t* seqlens, int32_t batch, int32_t max_pages_per_seq, int32_t page_size,
                            int32_t num_pages, int32_t max_seqlen, int32_t num_q_heads, int32_t num_kv_heads,
                            int32_t head_dim, float softmax_scale, void* out, float* lse, void* workspace,
                            size_t workspace_bytes, size_t need, void* stream, DecodeLaunch* launch) {
  if (batch < 0 || max_pages_per_seq < 0 || max_seqlen < 0 || num_pages < 0 || num_q_heads <= 0 ||
      num_kv_heads <= 0)
    return UATTN_EINVAL;
  if (num_q_heads % num_kv_heads != 0 || !scale_ok(softmax_scale)) return UATTN_EINVAL;
  if (head_dim != 64 && head_dim != 128) return UATTN_EUNSUPPORTED;
  if (page_size < 16 || (page_size & (page_size - 1)) != 0) return UATTN_EUNSUPPORTED;
  if (num_q_heads / num_kv_heads > uattn::kMaxGroup) return UATTN_EUNSUPPORTED;
  if (batch > 65535 || num_kv_heads > 65535) return UATTN_EUNSUPPORTED;
  if (max_seqlen > (1 << 24)) return UATTN_EUNSUPPORTED;  // keeps every 32-bit workspace offset in range
  if (batch == 0) {
    launch->batch = 0;
    return UATTN_OK;
  }
  if (max_seqlen == 0 || num_pages == 0) return UATTN_EINVAL;  // every entry holds at least its own token
  if (static_cast<int64_t>(max_pages_per_seq) * page_size < max_seqlen) return UATTN_EINVAL;
  if (!q || !k_pages || !v_pages || !block_table || !seqlens || !out) return UATTN_EINVAL;
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out)) return UATTN_EINVAL;
  if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))) return UATTN_EWORKSPACE;
  const int64_t nchunk = (static_cast<int64_t>(max_seqlen) + kChunkKeys - 1) / kChunkKeys;
  if (validate_env()) {
    Copied<int32_t> sl(seqlens, static_cast<size_t>(batch), stream);
    Copied<int32_t> bt(block_table, static_cast<size_t>(batch) * max_pages_per_seq, stream);
    if (sl.host == nullptr || bt.host == nullptr) return UATTN_EINVAL;
    for (int32_t b = 0; b < batch; ++b) {
      if (sl.host[b] < 1 || sl.host[b] > max_seqlen) return UATTN_EINVAL;
      const int32_t used = (sl.host[b] + page_size - 1) / page_size;
      for (int32_t j = 0; j < used; ++j) {
        const int32_t pg = bt.host[static_cast<size_t>(b) * max_pages_per_seq + j];
        if (pg < 0 || pg >= num_pages) return UATTN_EINVAL;
      }
    }
  }
  DecodeLaunch a;
  a.q = q;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.block_table = block_table;
  a.seqlens = seqlens;
  a.out = out;
  a.lse = lse;
  // counters at the start, partials at the end of the caller's buffer: a
  // workspace sized for one call can be reused by any call it is large enough for
  // without a partial region ever covering a counter that a later call relies on
  // being zero (see the zero-fill rule in uattn.h)
  if (need > 0) {
    const size_t acc_b = uattn::decode_ws_acc_bytes(batch, nchunk, num_q_heads, head_dim);
    const size_t ml_b = uattn::decode_ws_ml_bytes(batch, nchunk, num_q_heads);
    char* end = static_cast<char*>(workspace) + (workspace_bytes & ~static_cast<size_t>(15));
    a.ws_cnt = static_cast<int32_t*>(workspace);
    a.ws_ml = reinterpret_cast<float*>(end - ml_b);
    a.ws_acc = reinterpret_cast<float*>(end - ml_b - acc_b);
  } else {
    a.ws_cnt = nullptr;
    a.ws_ml = nullptr;
    a.ws_acc = nullptr;
  }
  a.batch = batch;
  a.max_pages_per_seq = max_pages_per_seq;
  a.page_size = page_size;
  a.num_pages = num_pages;
  a.max_seqlen = max_seqlen;
  a.nchunk_max = static_cast<int32_t>(nchunk);
  a.num_q_heads = num_q_heads;
  a.num_kv_heads = num_kv_heads;
  a.head_dim = head_dim;
  a.num_cus = uattn::device_cus();
  a.c = exp2_scale(softmax_scale);
  *launch = a;
  return UATTN_OK;
}
}  // namespace uattn

extern "C" {

uattn_status uattn_decode(const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                          const int32_t* seqlens, int32_t batch, int32_t max_pages_per_seq, int32_t page_size,
                          int32_t num_pages, int32_t max_seqlen, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                          float softmax_scale, void* out, float* lse, void* workspace, size_t workspace_bytes,
                          void* stream) {
  uattn::DecodeLaunch a;
  const uattn_status st =
      uattn::decode_prepare(q, k_pages, v_pages, block_table, seqlens, batch, max_pages_per_seq, page_size, num_pages,
                            max_seqlen, num_q_heads, num_kv_heads, head_dim, softmax_scale, out, lse, workspace,
                            workspace_bytes, uattn_decode_workspace_bytes(batch, max_seqlen, num_q_heads, head_dim), stream, &a);
  if (st != UATTN_OK || a.batch == 0) return st;
  return uattn::launch_decode(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

uattn_status uattn_logprob(const void* logits, int64_t row_stride, const int32_t* targets, int32_t num_rows,
                           int32_t vocab, float inv_temperature, float* logp, void* stream) {
  if (num_rows < 0 || vocab <= 0 || row_stride < vocab || !scale_ok(inv_temperature)) return UATTN_EINVAL;
  if (num_rows == 0) return UATTN_OK;
  if (!logits || !targets || !logp) return UATTN_EINVAL;
  if (!aligned16(logits) || (row_stride % 8) != 0) return UATTN_EINVAL;
  if (validate_env() && !targets_ok(targets, num_rows, vocab, stream)) return UATTN_EINVAL;
  uattn::LogprobLaunch a;
  a.logits = logits;
  a.row_stride = row_stride;
  a.targets = targets;
  a.logp = logp;
  a.num_rows = num_rows;
  a.vocab = vocab;
  a.inv_temperature = inv_temperature;
  return uattn::launch_logprob(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

uattn_status uattn_kv_write(const void* k_new, const void* v_new, int64_t token_stride, const int32_t* block_table,
                            const int32_t* seq_idx, const int32_t* positions, int32_t num_tokens, int32_t batch,
                            int32_t max_pages_per_seq, int32_t page_size, int32_t num_pages, int32_t num_kv_heads,
                            int32_t head_dim, void* k_pages, void* v_pages, void* stream) {
  if (num_tokens < 0 || batch < 0 || max_pages_per_seq < 0 || num_pages < 0 || num_kv_heads <= 0) return UATTN_EINVAL;
  if (head_dim != 64 && head_dim != 128) return UATTN_EUNSUPPORTED;
  if (page_size < 16 || (page_size & (page_size - 1)) != 0) return UATTN_EUNSUPPORTED;
  if (token_stride < static_cast<int64_t>(num_kv_heads) * head_dim || (token_stride % 8) != 0) return UATTN_EINVAL;
  if (num_tokens == 0 || batch == 0 || max_pages_per_seq == 0 || num_pages == 0) return UATTN_OK;
  if (!k_new || !v_new || !block_table || !seq_idx || !positions || !k_pages || !v_pages) return UATTN_EINVAL;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(k_pages) || !aligned16(v_pages)) return UATTN_EINVAL;
  if (validate_env() && !places_ok(block_table, seq_idx, positions, num_tokens, batch, max_pages_per_seq, page_size,
                                   num_pages, stream))
    return UATTN_EINVAL;
  uattn::KvWriteLaunch a;
  a.k_new = k_new;
  a.v_new = v_new;
  a.token_stride = token_stride;
  a.block_table = block_table;
  a.seq_idx = seq_idx;
  a.positions = positions;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.num_tokens = num_tokens;
  a.batch = batch;
  a.max_pages_per_seq = max_pages_per_seq;
  a.page_size = page_size;
  a.num_pages = num_pages;
  a.num_kv_heads = num_kv_heads;
  a.head_dim = head_dim;
  return uattn::launch_kv_write(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

uattn_status uattn_qk_norm_rope(const void* q, const void* k, const int32_t* positions, const void* q_weight,
                                const void* k_weight, float eps, const float* cos_sin, int32_t max_position,
                                int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                void* q_out, void* k_out, void* stream) {
  if (num_tokens < 0 || num_q_heads <= 0 || num_kv_heads <= 0 || max_position <= 0) return UATTN_EINVAL;
  if (!(eps >= 0.f) || !(eps < __builtin_inff())) return UATTN_EINVAL;
  if (head_dim != 64 && head_dim != 128) return UATTN_EUNSUPPORTED;
  if (num_tokens == 0) return UATTN_OK;
  if (!q || !k || !positions || !q_weight || !k_weight || !cos_sin || !q_out || !k_out) return UATTN_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(cos_sin) ||
      !aligned16(q_weight) || !aligned16(k_weight))
    return UATTN_EINVAL;
  uattn::NormRopeLaunch a;
  a.q = q;
  a.k = k;
  a.positions = positions;
  a.q_weight = q_weight;
  a.k_weight = k_weight;
  a.cos_sin = cos_sin;
  a.q_out = q_out;
  a.k_out = k_out;
  a.eps = eps;
  a.max_position = max_position;
  a.num_tokens = num_tokens;
  a.num_q_heads = num_q_heads;
  a.num_kv_heads = num_kv_heads;
  a.head_dim = head_dim;
  return uattn::launch_qk_norm_rope(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

uattn_status uattn_rope_cache(float* cos_sin, int32_t max_position, int32_t head_dim, double theta, void* stream) {
  if (max_position < 0 || !(theta > 1.0) || !(theta < 1e300)) return UATTN_EINVAL;
  if (head_dim != 64 && head_dim != 128) return UATTN_EUNSUPPORTED;
  if (max_position == 0) return UATTN_OK;
  if (!cos_sin || !aligned16(cos_sin)) return UATTN_EINVAL;
  return uattn::launch_rope_cache(cos_sin, max_position, head_dim, theta, static_cast<hipStream_t>(stream)) ==
                 hipSuccess
             ? UATTN_OK
             : UATTN_ELAUNCH;
}

uattn_status uattn_lm_head(const void* hidden, int64_t hidden_stride, const void* weight, int64_t weight_stride,
                           int32_t num_rows, int32_t vocab, int32_t hidden_dim, void* logits, int64_t logits_stride,
                           void* stream) {
  if (num_rows < 0 || vocab < 0 || hidden_dim <= 0 || (hidden_dim % 64) != 0) return UATTN_EINVAL;
  if (hidden_stride < hidden_dim || weight_stride < hidden_dim || logits_stride < vocab) return UATTN_EINVAL;
  if ((hidden_stride % 8) != 0 || (weight_stride % 8) != 0 || (logits_stride % 8) != 0) return UATTN_EINVAL;
  if (num_rows == 0 || vocab == 0) return UATTN_OK;
  if (!hidden || !weight || !logits) return UATTN_EINVAL;
  if (!aligned16(hidden) || !aligned16(weight) || !aligned16(logits)) return UATTN_EINVAL;
  uattn::LmHeadLaunch a;
  a.hidden = hidden;
  a.hidden_stride = hidden_stride;
  a.weight = weight;
  a.weight_stride = weight_stride;
  a.logits = logits;
  a.logits_stride = logits_stride;
  a.num_rows = num_rows;
  a.vocab = vocab;
  a.hidden_dim = hidden_dim;
  return uattn::launch_lm_head(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

size_t uattn_lm_head_logprob_workspace_bytes(int32_t num_rows, int32_t vocab) {
  if (num_rows <= 0 || vocab <= 0) return 0;
  return uattn::lm_head_logprob_ws_bytes(num_rows, vocab);
}

uattn_status uattn_lm_head_logprob(const void* hidden, int64_t hidden_stride, const void* weight,
                                   int64_t weight_stride, const int32_t* targets, int32_t num_rows, int32_t vocab,
                                   int32_t hidden_dim, float inv_temperature, float* logp, void* logits,
                                   int64_t logits_stride, void* workspace, size_t workspace_bytes, void* stream) {
  if (num_rows < 0 || vocab < 0 || hidden_dim <= 0 || (hidden_dim % 64) != 0) return UATTN_EINVAL;
  if (hidden_stride < hidden_dim || weight_stride < hidden_dim) return UATTN_EINVAL;
  if ((hidden_stride % 8) != 0 || (weight_stride % 8) != 0) return UATTN_EINVAL;
  if (logits != nullptr && (logits_stride < vocab || (logits_stride % 8) != 0 || !aligned16(logits)))
    return UATTN_EINVAL;
  if (!scale_ok(inv_temperature)) return UATTN_EINVAL;
  if (num_rows == 0) return UATTN_OK;
  if (vocab == 0) return UATTN_EINVAL;  // log-softmax over an empty vocabulary
  if (!hidden || !weight || !targets || !logp) return UATTN_EINVAL;
  if (!aligned16(hidden) || !aligned16(weight)) return UATTN_EINVAL;
  const size_t need = uattn_lm_head_logprob_workspace_bytes(num_rows, vocab);
  if (workspace == nullptr || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 3u) != 0)
    return UATTN_EWORKSPACE;
  if (validate_env() && !targets_ok(targets, num_rows, vocab, stream)) return UATTN_EINVAL;
  uattn::LmHeadLaunch a;
  a.hidden = hidden;
  a.hidden_stride = hidden_stride;
  a.weight = weight;
  a.weight_stride = weight_stride;
  a.logits = logits;
  a.logits_stride = logits != nullptr ? logits_stride : 0;
  a.num_rows = num_rows;
  a.vocab = vocab;
  a.hidden_dim = hidden_dim;
  return uattn::launch_lm_head_logprob(a, targets, inv_temperature, logp, workspace,
                                       static_cast<hipStream_t>(stream)) == hipSuccess
             ? UATTN_OK
             : UATTN_ELAUNCH;
}

size_t uattn_prefill_backward_workspace_bytes(int32_t total_tokens, int32_t num_q_heads) {
  if (total_tokens <= 0 || num_q_heads <= 0) return 0;
  return uattn::backward_ws_bytes(total_tokens, num_q_heads);
}

uattn_status uattn_prefill_backward(const void* q, const void* k, const void* v, const void* out, const void* dout,
                                    const float* lse, const int32_t* cu_seqlens, int32_t num_seqs,
                                    int32_t total_tokens, int32_t max_seqlen, int32_t num_q_heads,
                                    int32_t num_kv_heads, int32_t head_dim, float softmax_scale, void* dq, void* dk,
                                    void* dv, void* workspace, size_t workspace_bytes, void* stream) {
  if (num_seqs < 0 || total_tokens < 0 || max_seqlen < 0 || num_q_heads <= 0 || num_kv_heads <= 0)
    return UATTN_EINVAL;
  if (num_q_heads % num_kv_heads != 0 || !scale_ok(softmax_scale)) return UATTN_EINVAL;
  if (head_dim != 64 && head_dim != 128) return UATTN_EUNSUPPORTED;
  if (num_seqs > 65535) return UATTN_EUNSUPPORTED;
  if (num_seqs == 0 || total_tokens == 0 || max_seqlen == 0) return UATTN_OK;
  if (!q || !k || !v || !out || !dout || !lse || !cu_seqlens || !dq || !dk || !dv) return UATTN_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(dout) || !aligned16(dq) ||
      !aligned16(dk) || !aligned16(dv) || (reinterpret_cast<uintptr_t>(lse) & 3u) != 0)
    return UATTN_EINVAL;
  const size_t need = uattn_prefill_backward_workspace_bytes(total_tokens, num_q_heads);
  if (workspace == nullptr || workspace_bytes < need || !aligned16(workspace)) return UATTN_EWORKSPACE;
  if (validate_env() && !offsets_ok(cu_seqlens, num_seqs, total_tokens, max_seqlen, stream)) return UATTN_EINVAL;
  uattn::BackwardLaunch a;
  a.q = q;
  a.k = k;
  a.v = v;
  a.out = out;
  a.dout = dout;
  a.lse = lse;
  a.cu_seqlens = cu_seqlens;
  a.dq = dq;
  a.dk = dk;
  a.dv = dv;
  a.workspace = workspace;
  a.num_seqs = num_seqs;
  a.total_tokens = total_tokens;
  a.max_seqlen = max_seqlen;
  a.num_q_heads = num_q_heads;
  a.num_kv_heads = num_kv_heads;
  a.head_dim = head_dim;
  a.c = exp2_scale(softmax_scale);
  a.scale = softmax_scale;
  return uattn::launch_backward(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

uattn_status uattn_residual_norm(const void* x, const void* post_weight, const void* gate, int64_t gate_stride,
                                 float scale, const void* residual, const void* pre_weight, float eps,
                                 int32_t num_tokens, int32_t hidden_dim, void* residual_out, void* y, void* stream) {
  if (num_tokens < 0 || hidden_dim <= 0 || !is_finite(scale) || !(eps >= 0.f) || !is_finite(eps)) return UATTN_EINVAL;
  if (!norm_width_ok(hidden_dim)) return UATTN_EUNSUPPORTED;
  if (gate_stride != 0 && gate_stride != hidden_dim) return UATTN_EINVAL;
  if (num_tokens == 0) return UATTN_OK;
  if (!residual || (pre_weight == nullptr) != (y == nullptr) || (x == nullptr) != (residual_out == nullptr))
    return UATTN_EINVAL;
  if (x == nullptr && (post_weight != nullptr || gate != nullptr || y == nullptr)) return UATTN_EINVAL;
  if (!aligned16(x) || !aligned16(post_weight) || !aligned16(gate) || !aligned16(residual) || !aligned16(pre_weight) ||
      !aligned16(residual_out) || !aligned16(y))
    return UATTN_EINVAL;
  uattn::ResidualNormLaunch a;
  a.x = x;
  a.post_weight = post_weight;
  a.gate = gate;
  a.gate_stride = gate_stride;
  a.scale = scale;
  a.residual = residual;
  a.pre_weight = pre_weight;
  a.eps = eps;
  a.num_tokens = num_tokens;
  a.hidden_dim = hidden_dim;
  a.residual_out = residual_out;
  a.y = y;
  return uattn::launch_residual_norm(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

size_t uattn_residual_norm_backward_workspace_bytes(int32_t num_tokens, int32_t hidden_dim) {
  if (num_tokens <= 0 || hidden_dim <= 0 || !norm_width_ok(hidden_dim)) return 0;
  return uattn::residual_norm_backward_ws_bytes(num_tokens, hidden_dim);
}

uattn_status uattn_residual_norm_backward(const void* dy, const void* dresidual_out, const void* residual_out,
                                          const void* pre_weight, const void* x, const void* post_weight,
                                          const void* gate, int64_t gate_stride, float scale, float eps,
                                          int32_t num_tokens, int32_t hidden_dim, void* dresidual, void* dx,
                                          float* dpre_weight, float* dpost_weight, void* dgate, void* workspace,
                                          size_t workspace_bytes, void* stream) {
  if (num_tokens < 0 || hidden_dim <= 0 || !is_finite(scale) || !(eps >= 0.f) || !is_finite(eps)) return UATTN_EINVAL;
  if (!norm_width_ok(hidden_dim)) return UATTN_EUNSUPPORTED;
  if (gate_stride != 0 && gate_stride != hidden_dim) return UATTN_EINVAL;
  // which gradients belong to which of the forward's parts, whatever the number of tokens
  if ((pre_weight == nullptr) != (dpre_weight == nullptr) || (post_weight == nullptr) != (dpost_weight == nullptr) ||
      (gate == nullptr) != (dgate == nullptr))
    return UATTN_EINVAL;
  if (num_tokens > 0) {
    if (!dresidual || (dy == nullptr) != (pre_weight == nullptr)) return UATTN_EINVAL;
    if (dy == nullptr && dresidual_out == nullptr) return UATTN_EINVAL;
    if (dy != nullptr && residual_out == nullptr) return UATTN_EINVAL;
    if ((post_weight != nullptr || gate != nullptr) && (x == nullptr || dx == nullptr)) return UATTN_EINVAL;
  }
  if (!aligned16(dy) || !aligned16(dresidual_out) || !aligned16(residual_out) || !aligned16(pre_weight) || !aligned16(x) ||
      !aligned16(post_weight) || !aligned16(gate) || !aligned16(dresidual) || !aligned16(dx) || !aligned16(dpre_weight) ||
      !aligned16(dpost_weight) || !aligned16(dgate))
    return UATTN_EINVAL;
  const size_t need = uattn_residual_norm_backward_workspace_bytes(num_tokens, hidden_dim);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))) return UATTN_EWORKSPACE;
  uattn::ResidualNormBackwardLaunch a;
  a.dy = dy;
  a.dresidual_out = dresidual_out;
  a.residual_out = residual_out;
  a.pre_weight = pre_weight;
  a.x = x;
  a.post_weight = post_weight;
  a.gate = gate;
  a.gate_stride = gate_stride;
  a.scale = scale;
  a.eps = eps;
  a.num_tokens = num_tokens;
  a.hidden_dim = hidden_dim;
  a.dresidual = dresidual;
  a.dx = dx;
  a.dpre_weight = dpre_weight;
  a.dpost_weight = dpost_weight;
  a.dgate = dgate;
  a.workspace = workspace;
  return uattn::launch_residual_norm_backward(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK
                                                                                                 : UATTN_ELAUNCH;
}

uattn_status uattn_embedding(const int32_t* ids, const void* table, int64_t table_stride, float scale,
                             int32_t num_tokens, int32_t vocab, int32_t hidden_dim, void* out, int64_t out_stride,
                             void* stream) {
  if (num_tokens < 0 || vocab <= 0 || hidden_dim <= 0 || (hidden_dim % 8) != 0 || !is_finite(scale)) return UATTN_EINVAL;
  if (table_stride < hidden_dim || out_stride < hidden_dim || (table_stride % 8) != 0 || (out_stride % 8) != 0)
    return UATTN_EINVAL;
  if (hidden_dim > kMaxEmbeddingWidth) return UATTN_EUNSUPPORTED;
  if (num_tokens == 0) return UATTN_OK;
  if (!ids || !table || !out || !aligned16(table) || !aligned16(out)) return UATTN_EINVAL;
  if (validate_env() && !all_below(ids, num_tokens, vocab, stream)) return UATTN_EINVAL;
  uattn::EmbeddingLaunch a;
  a.ids = ids;
  a.table = table;
  a.table_stride = table_stride;
  a.scale = scale;
  a.num_tokens = num_tokens;
  a.vocab = vocab;
  a.hidden_dim = hidden_dim;
  a.out = out;
  a.out_stride = out_stride;
  return uattn::launch_embedding(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

size_t uattn_embedding_backward_workspace_bytes(int32_t num_tokens, int32_t hidden_dim) {
  if (num_tokens <= 0 || hidden_dim <= 0 || num_tokens > kMaxSortedTokens || hidden_dim > kMaxEmbeddingWidth) return 0;
  return uattn::embedding_backward_ws_bytes(num_tokens, hidden_dim);
}

uattn_status uattn_embedding_backward(const void* dout, int64_t dout_stride, const int32_t* ids, float scale,
                                      int32_t num_tokens, int32_t vocab, int32_t hidden_dim, void* grad,
                                      int64_t grad_stride, int32_t grad_fp32, int32_t accumulate, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  if (num_tokens < 0 || vocab <= 0 || hidden_dim <= 0 || (hidden_dim % 8) != 0 || !is_finite(scale)) return UATTN_EINVAL;
  if ((grad_fp32 & ~1) != 0 || (accumulate & ~1) != 0) return UATTN_EINVAL;
  if (grad_stride < hidden_dim || (grad_stride % (grad_fp32 ? 4 : 8)) != 0) return UATTN_EINVAL;
  if (dout_stride < hidden_dim || (dout_stride % 8) != 0) return UATTN_EINVAL;
  if (num_tokens > kMaxSortedTokens || hidden_dim > kMaxEmbeddingWidth) return UATTN_EUNSUPPORTED;
  if (num_tokens == 0 && accumulate) return UATTN_OK;
  if (!grad || !aligned16(grad)) return UATTN_EINVAL;
  if (num_tokens > 0 && (!dout || !ids || !aligned16(dout))) return UATTN_EINVAL;
  const size_t need = uattn_embedding_backward_workspace_bytes(num_tokens, hidden_dim);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))) return UATTN_EWORKSPACE;
  if (validate_env() && !all_below(ids, num_tokens, vocab, stream)) return UATTN_EINVAL;
  uattn::EmbeddingBackwardLaunch a;
  a.dout = dout;
  a.dout_stride = dout_stride;
  a.ids = ids;
  a.scale = scale;
  a.num_tokens = num_tokens;
  a.vocab = vocab;
  a.hidden_dim = hidden_dim;
  a.grad = grad;
  a.grad_stride = grad_stride;
  a.grad_fp32 = grad_fp32 != 0;
  a.accumulate = accumulate != 0;
  a.workspace = workspace;
  return uattn::launch_embedding_backward(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

uattn_status uattn_logits_process(const void* logits, int64_t logits_stride, int32_t num_rows, int32_t vocab,
                                  const int32_t* tokens, int32_t num_tokens, const int32_t* history,
                                  const float* penalties, const int32_t* bias_ids, const float* bias_values,
                                  int32_t num_bias, const int32_t* bias_rows, const uint32_t* mask,
                                  int64_t mask_stride, int32_t num_masks, const int32_t* mask_rows, void* out,
                                  int64_t out_stride, void* stream) {
  uattn::LogitsLaunch a{};
  a.logits = logits;
  a.logits_stride = logits_stride;
  a.num_rows = num_rows;
  a.vocab = vocab;
  a.tokens = tokens;
  a.num_tokens = num_tokens;
  a.history = history;
  a.penalties = penalties;
  a.bias_ids = bias_ids;
  a.bias_values = bias_values;
  a.num_bias = num_bias;
  a.bias_rows = bias_rows;
  a.mask = mask;
  a.mask_stride = mask_stride;
  a.num_masks = num_masks;
  a.mask_rows = mask_rows;
  a.out = out;
  a.out_stride = out_stride;
  const uattn_status st = check_logits(a, false, stream);
  if (st != UATTN_OK || num_rows == 0) return st;
  return uattn::launch_logits_process(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

uattn_status uattn_logits_process_backward(const void* dout, int64_t dout_stride, const void* logits,
                                           int64_t logits_stride, int32_t num_rows, int32_t vocab,
                                           const int32_t* tokens, int32_t num_tokens, const int32_t* history,
                                           const float* penalties, const uint32_t* mask, int64_t mask_stride,
                                           int32_t num_masks, const int32_t* mask_rows, void* dlogits,
                                           int64_t dlogits_stride, void* stream) {
  uattn::LogitsLaunch a{};
  a.dout = dout;
  a.dout_stride = dout_stride;
  a.logits = logits;
  a.logits_stride = logits_stride;
  a.num_rows = num_rows;
  a.vocab = vocab;
  a.tokens = tokens;
  a.num_tokens = num_tokens;
  a.history = history;
  a.penalties = penalties;
  a.mask = mask;
  a.mask_stride = mask_stride;
  a.num_masks = num_masks;
  a.mask_rows = mask_rows;
  a.out = dlogits;
  a.out_stride = dlogits_stride;
  const uattn_status st = check_logits(a, true, stream);
  if (st != UATTN_OK || num_rows == 0) return st;
  if (!dout || !aligned16(dout) || dout_stride < vocab || (dout_stride % 8) != 0) return UATTN_EINVAL;
  return uattn::launch_logits_process_backward(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK
                                                                                                  : UATTN_ELAUNCH;
}

uattn_status uattn_logprob_backward(const void* logits, int64_t row_stride, const int32_t* targets, const float* dlogp,
                                    int32_t num_rows, int32_t vocab, float inv_temperature, void* dlogits,
                                    int64_t dlogits_stride, void* stream) {
  if (num_rows < 0 || vocab <= 0 || row_stride < vocab || (row_stride % 8) != 0) return UATTN_EINVAL;
  if (dlogits_stride < vocab || (dlogits_stride % 8) != 0) return UATTN_EINVAL;
  // the exponent's factor, inv_temperature * log2(e), has to be finite too
  if (!scale_ok(inv_temperature) || !scale_ok(exp2_scale(inv_temperature))) return UATTN_EINVAL;
  if (num_rows == 0) return UATTN_OK;
  if (!logits || !targets || !dlogp || !dlogits || !aligned16(logits) || !aligned16(dlogits)) return UATTN_EINVAL;
  if (dlogits == logits) return UATTN_EINVAL;  // every wave reads the target's logit, when others may have written theirs
  if (validate_env()) {
    Copied<int32_t> tg(targets, num_rows, stream);
    Copied<float> dl(dlogp, num_rows, stream);
    if (tg.host == nullptr || dl.host == nullptr) return UATTN_EINVAL;
    for (int32_t t = 0; t < num_rows; ++t)
      if (dl.host[t] != 0.f && (tg.host[t] < 0 || tg.host[t] >= vocab)) return UATTN_EINVAL;
  }
  uattn::LogprobBackwardLaunch a;
  a.logits = logits;
  a.row_stride = row_stride;
  a.targets = targets;
  a.dlogp = dlogp;
  a.num_rows = num_rows;
  a.vocab = vocab;
  a.inv_temperature = inv_temperature;
  a.dlogits = dlogits;
  a.dlogits_stride = dlogits_stride;
  return uattn::launch_logprob_backward(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

// ---------------------------------------------------------------------------
// The cache in 8 or 4 bits
// ---------------------------------------------------------------------------
uattn_status uattn_kv_write_mx(const void* k_new, const void* v_new, int64_t token_stride, const int32_t* block_table,
                               const int32_t* seq_idx, const int32_t* positions, int32_t num_tokens, int32_t batch,
                               int32_t max_pages_per_seq, int32_t page_size, int32_t num_pages, int32_t num_kv_heads,
                               int32_t head_dim, int32_t k_bits, int32_t v_bits, void* k_codes, void* k_scales,
                               void* v_codes, void* v_scales, void* stream) {
  if (num_tokens < 0 || batch < 0 || max_pages_per_seq < 0 || num_pages < 0 || num_kv_heads <= 0) return UATTN_EINVAL;
  if (head_dim != 64 && head_dim != 128) return UATTN_EUNSUPPORTED;
  if (page_size < 16 || (page_size & (page_size - 1)) != 0) return UATTN_EUNSUPPORTED;
  if (!bits_ok(k_bits, v_bits) || num_kv_heads > 65535) return UATTN_EUNSUPPORTED;
  if (!row_stride_ok(token_stride, num_kv_heads, head_dim)) return UATTN_EINVAL;
  if (num_tokens == 0 || batch == 0 || max_pages_per_seq == 0 || num_pages == 0) return UATTN_OK;
  if (!k_new || !v_new || !block_table || !seq_idx || !positions) return UATTN_EINVAL;
  if (!k_codes || !k_scales || !v_codes || !v_scales) return UATTN_EINVAL;
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(k_codes) || !aligned16(k_scales) || !aligned16(v_codes) ||
      !aligned16(v_scales))
    return UATTN_EINVAL;
  if (validate_env() && !places_ok(block_table, seq_idx, positions, num_tokens, batch, max_pages_per_seq, page_size,
                                   num_pages, stream))
    return UATTN_EINVAL;
  uattn::KvMxLaunch a = {};
  a.k = k_new;
  a.v = v_new;
  a.token_stride = token_stride;
  a.cache = {k_codes, k_scales, v_codes, v_scales, k_bits, v_bits};
  a.block_table = block_table;
  a.seq_idx = seq_idx;
  a.positions = positions;
  a.num_tokens = num_tokens;
  a.batch = batch;
  a.max_pages_per_seq = max_pages_per_seq;
  a.page_size = page_size;
  a.num_pages = num_pages;
  a.num_kv_heads = num_kv_heads;
  a.head_dim = head_dim;
  return uattn::launch_kv_write_mx(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

uattn_status uattn_kv_read_mx(const void* k_codes, const void* k_scales, const void* v_codes, const void* v_scales,
                              int32_t k_bits, int32_t v_bits, const int32_t* block_table, const int32_t* seq_idx,
                              const int32_t* positions, int32_t num_tokens, int32_t batch, int32_t max_pages_per_seq,
                              int32_t page_size, int32_t num_pages, int32_t num_kv_heads, int32_t head_dim, void* k_out,
                              void* v_out, int64_t out_stride, void* stream) {
  if (num_tokens < 0 || batch < 0 || max_pages_per_seq < 0 || num_pages < 0 || num_kv_heads <= 0) return UATTN_EINVAL;
  if (head_dim != 64 && head_dim != 128) return UATTN_EUNSUPPORTED;
  if (page_size < 16 || (page_size & (page_size - 1)) != 0) return UATTN_EUNSUPPORTED;
  if (!bits_ok(k_bits, v_bits) || num_kv_heads > 65535) return UATTN_EUNSUPPORTED;
  if (!row_stride_ok(out_stride, num_kv_heads, head_dim)) return UATTN_EINVAL;
  if (num_tokens == 0) return UATTN_OK;
  if (!seq_idx || !positions || !k_out || !v_out || !aligned16(k_out) || !aligned16(v_out)) return UATTN_EINVAL;
  if (k_out == v_out) return UATTN_EINVAL;
  // without a table or a pool every token is one without a place
  const bool table = batch > 0 && max_pages_per_seq > 0;
  if (table && !block_table) return UATTN_EINVAL;
  if (table && num_pages > 0 && (!k_codes || !k_scales || !v_codes || !v_scales)) return UATTN_EINVAL;
  if (!aligned16(k_codes) || !aligned16(k_scales) || !aligned16(v_codes) || !aligned16(v_scales)) return UATTN_EINVAL;
  if (validate_env() && !places_ok(block_table, seq_idx, positions, num_tokens, batch, max_pages_per_seq, page_size,
                                   num_pages, stream))
    return UATTN_EINVAL;
  uattn::KvMxLaunch a = {};
  a.k_out = k_out;
  a.v_out = v_out;
  a.out_stride = out_stride;
  // the kernels of this call only read the cache
  a.cache = {const_cast<void*>(k_codes), const_cast<void*>(k_scales), const_cast<void*>(v_codes),
             const_cast<void*>(v_scales), k_bits, v_bits};
  a.block_table = block_table;
  a.seq_idx = seq_idx;
  a.positions = positions;
  a.num_tokens = num_tokens;
  a.batch = batch;
  a.max_pages_per_seq = max_pages_per_seq;
  a.page_size = page_size;
  a.num_pages = num_pages;
  a.num_kv_heads = num_kv_heads;
  a.head_dim = head_dim;
  return uattn::launch_kv_read_mx(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

uattn_status uattn_kv_round_mx(const void* k, const void* v, int64_t token_stride, int32_t num_tokens,
                               int32_t num_kv_heads, int32_t head_dim, int32_t k_bits, int32_t v_bits, void* k_out,
                               void* v_out, int64_t out_stride, void* stream) {
  if (num_tokens < 0 || num_kv_heads <= 0) return UATTN_EINVAL;
  if (head_dim != 64 && head_dim != 128) return UATTN_EUNSUPPORTED;
  if (!bits_ok(k_bits, v_bits) || num_kv_heads > 65535) return UATTN_EUNSUPPORTED;
  if (!row_stride_ok(token_stride, num_kv_heads, head_dim) || !row_stride_ok(out_stride, num_kv_heads, head_dim))
    return UATTN_EINVAL;
  if (num_tokens == 0) return UATTN_OK;
  if (!k || !v || !k_out || !v_out || !aligned16(k) || !aligned16(v) || !aligned16(k_out) || !aligned16(v_out))
    return UATTN_EINVAL;
  // in place the rows have to stay where they are: workgroups read others while this one writes
  if ((k_out == k || v_out == v) && token_stride != out_stride && num_tokens > 1) return UATTN_EINVAL;
  if (k_out == v || v_out == k || k_out == v_out) return UATTN_EINVAL;
  uattn::KvMxLaunch a = {};
  a.k = k;
  a.v = v;
  a.token_stride = token_stride;
  a.k_out = k_out;
  a.v_out = v_out;
  a.out_stride = out_stride;
  a.cache.k_bits = k_bits;
  a.cache.v_bits = v_bits;
  a.num_tokens = num_tokens;
  a.num_kv_heads = num_kv_heads;
  a.head_dim = head_dim;
  return uattn::launch_kv_round_mx(a, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

size_t uattn_decode_mx_workspace_bytes(int32_t batch, int32_t max_seqlen, int32_t num_q_heads, int32_t num_kv_heads,
                                       int32_t head_dim) {
  if (batch <= 0 || max_seqlen <= 0 || num_q_heads <= 0 || num_kv_heads <= 0 || head_dim <= 0) return 0;
  if (num_q_heads % num_kv_heads != 0) return 0;
  const int64_t nchunk = (static_cast<int64_t>(max_seqlen) + kChunkKeys - 1) / kChunkKeys;
  if (nchunk <= 1 || uattn::decode_mx_in_lds(nchunk, num_q_heads / num_kv_heads, head_dim)) return 0;
  return uattn::decode_ws_acc_bytes(batch, nchunk, num_q_heads, head_dim) +
         uattn::decode_ws_ml_bytes(batch, nchunk, num_q_heads);
}

uattn_status uattn_decode_mx(const void* q, const void* k_codes, const void* k_scales, const void* v_codes,
                             const void* v_scales, int32_t k_bits, int32_t v_bits, const int32_t* block_table,
                             const int32_t* seqlens, int32_t batch, int32_t max_pages_per_seq, int32_t page_size,
                             int32_t num_pages, int32_t max_seqlen, int32_t num_q_heads, int32_t num_kv_heads,
                             int32_t head_dim, float softmax_scale, void* out, float* lse, void* workspace,
                             size_t workspace_bytes, void* stream) {
  if (!bits_ok(k_bits, v_bits)) return UATTN_EUNSUPPORTED;
  const size_t need = uattn_decode_mx_workspace_bytes(batch, max_seqlen, num_q_heads, num_kv_heads, head_dim);
  uattn::DecodeLaunch a;
  const uattn_status st =
      uattn::decode_prepare(q, k_codes, v_codes, block_table, seqlens, batch, max_pages_per_seq, page_size, num_pages,
                            max_seqlen, num_q_heads, num_kv_heads, head_dim, softmax_scale, out, lse, workspace,
                            workspace_bytes, need, stream, &a);
  if (st != UATTN_OK || a.batch == 0) return st;
  if (!k_scales || !v_scales || !aligned16(k_scales) || !aligned16(v_scales)) return UATTN_EINVAL;
  // the kernel only reads the cache
  const uattn::MxCache cache = {const_cast<void*>(k_codes), const_cast<void*>(k_scales), const_cast<void*>(v_codes),
                                const_cast<void*>(v_scales), k_bits, v_bits};
  return uattn::launch_decode_mx(a, cache, static_cast<hipStream_t>(stream)) == hipSuccess ? UATTN_OK : UATTN_ELAUNCH;
}

}  // extern "C"
