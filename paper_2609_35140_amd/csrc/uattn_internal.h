// Internal launcher interface between the C-ABI layer and the kernel files.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/uattn.h"

namespace uattn {

struct PrefillLaunch {
  const void* q;
  const void* k;
  const void* v;
  const int32_t* cu_seqlens;
  void* out;
  float* lse;
  int32_t num_seqs;
  int32_t total_tokens;
  int32_t max_seqlen;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;
  float c;  // fp32(scale * log2(e))
};

struct DecodeLaunch {
  const void* q;
  const void* k_pages;
  const void* v_pages;
  const int32_t* block_table;
  const int32_t* seqlens;
  void* out;
  float* lse;
  float* ws_acc;  // [batch][Hq][decode_slots(nchunk_max)][head_dim]
  float* ws_ml;   // [batch][Hq][decode_slots(nchunk_max)][2]
  int32_t* ws_cnt; // [batch][Hkv] arrival counters
  int32_t batch;
  int32_t max_pages_per_seq;
  int32_t page_size;
  int32_t num_pages;
  int32_t max_seqlen;
  int32_t nchunk_max;
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t num_cus;  // compute units of the current device (sizes the persistent grid)
  float c;
};

struct LogprobLaunch {
  const void* logits;
  int64_t row_stride;
  const int32_t* targets;
  float* logp;
  int32_t num_rows;
  int32_t vocab;
  float inv_temperature;
};

struct KvWriteLaunch {
  const void* k_new;
  const void* v_new;
  int64_t token_stride;
  const int32_t* block_table;
  const int32_t* seq_idx;
  const int32_t* positions;
  void* k_pages;
  void* v_pages;
  int32_t num_tokens, batch, max_pages_per_seq, page_size, num_pages, num_kv_heads, head_dim;
};

hipError_t launch_kv_write(const KvWriteLaunch& a, hipStream_t stream);

// The pools of a cache held in 8 or 4 bits: codes and scale bytes of keys and values.
struct MxCache {
  void* k_codes;
  void* k_scales;
  void* v_codes;
  void* v_scales;
  int32_t k_bits, v_bits;
};

struct KvMxLaunch {
  const void* k;         // rows given (write, round)
  const void* v;
  int64_t token_stride;
  void* k_out;           // rows made (read, round)
  void* v_out;
  int64_t out_stride;
  MxCache cache;         // round: the bits alone
  const int32_t* block_table;
  const int32_t* seq_idx;
  const int32_t* positions;
  int32_t num_tokens, batch, max_pages_per_seq, page_size, num_pages, num_kv_heads, head_dim;
};

hipError_t launch_kv_write_mx(const KvMxLaunch& a, hipStream_t stream);
hipError_t launch_kv_read_mx(const KvMxLaunch& a, hipStream_t stream);
hipError_t launch_kv_round_mx(const KvMxLaunch& a, hipStream_t stream);

struct NormRopeLaunch {
  const void* q;
  const void* k;
  const int32_t* positions;
  const void* q_weight;
  const void* k_weight;
  const float* cos_sin;
  void* q_out;
  void* k_out;
  float eps;
  int32_t max_position, num_tokens, num_q_heads, num_kv_heads, head_dim;
};

hipError_t launch_qk_norm_rope(const NormRopeLaunch& a, hipStream_t stream);
hipError_t launch_rope_cache(float* cos_sin, int32_t max_position, int32_t head_dim, double theta, hipStream_t stream);

struct LmHeadLaunch {
  const void* hidden;
  int64_t hidden_stride;
  const void* weight;
  int64_t weight_stride;
  void* logits;
  int64_t logits_stride;
  int32_t num_rows, vocab, hidden_dim;
};

hipError_t launch_lm_head(const LmHeadLaunch& a, hipStream_t stream);
// LM head with the fused log-probability epilogue (a.logits may be nullptr):
// partials in `workspace` (lm_head_logprob_ws_bytes), then their fold into logp.
hipError_t launch_lm_head_logprob(const LmHeadLaunch& a, const int32_t* targets, float inv_temperature, float* logp,
                                  void* workspace, hipStream_t stream);
size_t lm_head_logprob_ws_bytes(int64_t num_rows, int64_t vocab);

struct BackwardLaunch {
  const void* q;
  const void* k;
  const void* v;
  const void* out;
  const void* dout;
  const float* lse;
  const int32_t* cu_seqlens;
  void* dq;
  void* dk;
  void* dv;
  void* workspace;  // backward_ws_bytes(total_tokens, num_q_heads)
  int32_t num_seqs, total_tokens, max_seqlen, num_q_heads, num_kv_heads, head_dim;
  float c;      // fp32(scale * log2(e))
  float scale;  // softmax scale
};

hipError_t launch_backward(const BackwardLaunch& a, hipStream_t stream);
size_t backward_ws_bytes(int64_t total_tokens, int64_t num_q_heads);

struct ResidualNormLaunch {
  const void* x;            // nullptr: no block output, the residual is normalized as it is
  const void* post_weight;  // nullptr: x is not normalized
  const void* gate;         // nullptr, one row (gate_stride 0) or a row per token
  int64_t gate_stride;
  float scale;
  const void* residual;
  const void* pre_weight;   // nullptr with y
  float eps;
  int32_t num_tokens, hidden_dim;
  void* residual_out;       // nullptr with x
  void* y;
};

hipError_t launch_residual_norm(const ResidualNormLaunch& a, hipStream_t stream);

struct ResidualNormBackwardLaunch {
  const void* dy;             // nullptr with pre_weight and dpre_weight
  const void* dresidual_out;  // nullptr: zeros
  const void* residual_out;
  const void* pre_weight;
  const void* x;              // nullptr where neither post_weight nor gate is given
  const void* post_weight;
  const void* gate;
  int64_t gate_stride;
  float scale, eps;
  int32_t num_tokens, hidden_dim;
  void* dresidual;
  void* dx;                   // nullptr: no block output
  float* dpre_weight;
  float* dpost_weight;
  void* dgate;                // fp32 row (gate_stride 0) or bf16 rows
  void* workspace;            // residual_norm_backward_ws_bytes(num_tokens, hidden_dim)
};

hipError_t launch_residual_norm_backward(const ResidualNormBackwardLaunch& a, hipStream_t stream);
size_t residual_norm_backward_ws_bytes(int64_t num_tokens, int64_t hidden_dim);

struct EmbeddingLaunch {
  const int32_t* ids;
  const void* table;
  int64_t table_stride;
  float scale;
  int32_t num_tokens, vocab, hidden_dim;
  void* out;
  int64_t out_stride;
};

hipError_t launch_embedding(const EmbeddingLaunch& a, hipStream_t stream);

struct EmbeddingBackwardLaunch {
  const void* dout;
  int64_t dout_stride;
  const int32_t* ids;
  float scale;
  int32_t num_tokens, vocab, hidden_dim;
  void* grad;
  int64_t grad_stride;
  bool grad_fp32, accumulate;
  void* workspace;  // embedding_backward_ws_bytes(num_tokens, hidden_dim)
};

hipError_t launch_embedding_backward(const EmbeddingBackwardLaunch& a, hipStream_t stream);
size_t embedding_backward_ws_bytes(int64_t num_tokens, int64_t hidden_dim);

struct LogitsLaunch {
  const void* dout;  // backward only
  int64_t dout_stride;
  const void* logits;
  int64_t logits_stride;
  int32_t num_rows, vocab;
  const int32_t* tokens;
  int32_t num_tokens;
  const int32_t* history;    // nullptr: no penalties
  const float* penalties;
  const int32_t* bias_ids;
  const float* bias_values;
  int32_t num_bias;
  const int32_t* bias_rows;  // nullptr: no biases
  const uint32_t* mask;      // nullptr: no mask
  int64_t mask_stride;
  int32_t num_masks;
  const int32_t* mask_rows;
  void* out;
  int64_t out_stride;
};

hipError_t launch_logits_process(const LogitsLaunch& a, hipStream_t stream);
hipError_t launch_logits_process_backward(const LogitsLaunch& a, hipStream_t stream);

struct LogprobBackwardLaunch {
  const void* logits;
  int64_t row_stride;
  const int32_t* targets;
  const float* dlogp;
  int32_t num_rows, vocab;
  float inv_temperature;
  void* dlogits;
  int64_t dlogits_stride;
};

hipError_t launch_logprob_backward(const LogprobBackwardLaunch& a, hipStream_t stream);

// A grid holds fewer than 2^32 threads: past that it starts modulo 2^32, the rest
// is never run and no error is reported.  Calls launch(first, n) for consecutive
// runs of workgroups that fit, each cut at a multiple of the XCD count.
template <class Launch>
hipError_t launch_parts(int64_t workgroups, int threads, const Launch& launch) {
  if (workgroups > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
  const int64_t most = ((int64_t{1} << 32) / threads - 1) / 8 * 8;
  for (int64_t first = 0; first < workgroups; first += most) {
    launch(static_cast<int>(first), static_cast<unsigned>(workgroups - first < most ? workgroups - first : most));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Compute units of the current device (cached per device; 256 if the query fails).
int32_t device_cus();

// Each returns hipSuccess or the launch error.
hipError_t launch_prefill(const PrefillLaunch& a, hipStream_t stream);
hipError_t launch_decode(const DecodeLaunch& a, hipStream_t stream);
hipError_t launch_decode_mx(const DecodeLaunch& a, const MxCache& cache, hipStream_t stream);  // a's pages and counters unused
// Whether all chunks of an entry are folded in LDS, so that no partial goes through the workspace.
bool decode_mx_in_lds(int64_t nchunk, int64_t group, int64_t head_dim);
hipError_t launch_logprob(const LogprobLaunch& a, hipStream_t stream);

// Checks uattn_decode's arguments (every rule of uattn.h) and fills the launch
// record, laying the workspace out as counters at its start and partials at
// its end (`need`: the bytes it has to have); `stream` orders UATTN_VALIDATE's
// copies.  Returns the status uattn_decode reports; `launch->batch` is 0 when there is
// nothing to launch.
uattn_status decode_prepare(const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                            const int32_t* seqlens, int32_t batch, int32_t max_pages_per_seq, int32_t page_size,
                            int32_t num_pages, int32_t max_seqlen, int32_t num_q_heads, int32_t num_kv_heads,
                            int32_t head_dim, float softmax_scale, void* out, float* lse, void* workspace,
                            size_t workspace_bytes, size_t need, void* stream, DecodeLaunch* launch);

// Decode workspace: arrival counters at the start (kept zero between calls),
// the fp32 partials (acc, then m/l) at the end of the caller's buffer.
// Partial slots per (entry, q head) for nchunk chunks: rounded up to even, so
// that the (m, l) pairs of two consecutive chunks are one 16-byte load.
int64_t decode_slots(int64_t nchunk);
size_t decode_ws_acc_bytes(int64_t batch, int64_t nchunk, int64_t num_q_heads, int64_t head_dim);
size_t decode_ws_ml_bytes(int64_t batch, int64_t nchunk, int64_t num_q_heads);
size_t decode_ws_cnt_bytes(int64_t batch, int64_t num_q_heads);

}  // namespace uattn
