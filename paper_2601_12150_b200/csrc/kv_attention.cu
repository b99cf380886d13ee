// kv_cache_attention: argument checks and the choice between the two forms of the kernel.
#include <math.h>

#include "kv_attention.cuh"

namespace {

int32_t check_attn(const spv_kv_cache* c, const spv_kv_seqs* s, const spv_kv_attn_desc* d) {
  int32_t st = spv_kv_check_cache(c);
  if (st != SPV_OK) return st;
  if ((st = spv_kv_check_seqs(c, s)) != SPV_OK) return st;
  if (!d || d->tokens < 1 || d->heads < 1 || d->heads % c->kv_heads) return SPV_ERR_INVALID_ARG;
  if (d->dtype != SPV_BF16 && d->dtype != SPV_FP16) return SPV_ERR_UNSUPPORTED;
  if (d->causal != 0 && d->causal != 1) return SPV_ERR_INVALID_ARG;
  if (!(d->softmax_scale >= 0.0f) || d->softmax_scale > 1e30f) return SPV_ERR_INVALID_ARG;
  if ((int64_t)d->tokens * d->heads > INT32_MAX / 2) return SPV_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)d->tokens * (d->heads / c->kv_heads), most = spv_kv_max_length(c, s);
  // what the kernels number in 31 bits: tiles of 128 rows x 128 keys and the rows of one sequence's dense copies ...
  if ((rows + 255) / 256 * 2 * ((most + 127) / 128) * c->kv_heads > INT32_MAX / 2) return SPV_ERR_UNSUPPORTED;
  if ((most + 127 > rows + 255 ? most + 127 : rows + 255) * c->kv_heads > INT32_MAX / 2) return SPV_ERR_UNSUPPORTED;
  // ... and tiles of 32 slots of all sequences
  if ((int64_t)s->batch * c->kv_heads * ((most + 31) / 32) > INT32_MAX / 2) return SPV_ERR_UNSUPPORTED;
  const int64_t strides[6] = {d->q_stride_b, d->q_stride_tok, d->q_stride_head, d->o_stride_b, d->o_stride_tok, d->o_stride_head};
  for (int64_t x : strides)
    if (x % 8) return SPV_ERR_ALIGNMENT;
  if (d->w_stride_b < 0 || d->w_stride_head < 0) return SPV_ERR_INVALID_ARG;
  return SPV_OK;
}

// Whether the streaming form takes the call: few enough rows share a key head.
bool streams(const spv_kv_cache* c, const spv_kv_attn_desc* d) {
  return (int64_t)d->tokens * (d->heads / c->kv_heads) <= kKvStreamMaxRows;
}

}  // namespace

extern "C" int32_t spv_kv_attention_workspace_size(const spv_kv_cache* cache, const spv_kv_seqs* seqs,
                                                   const spv_kv_attn_desc* d, int32_t want_weights, size_t* bytes) {
  const int32_t st = check_attn(cache, seqs, d);
  if (st != SPV_OK) return st;
  if (!bytes) return SPV_ERR_INVALID_ARG;
  if (streams(cache, d)) *bytes = spv_kv_stream_workspace(cache, seqs, d, want_weights != 0);
  else *bytes = spv_kv_prompt_workspace(cache, seqs, d);
  return SPV_OK;
}

extern "C" int32_t kv_cache_attention(spv_ctx* ctx, const spv_kv_cache* cache, const spv_kv_seqs* seqs,
                                      const spv_kv_attn_desc* d, const void* q, void* o, float* lse, const float* weights_in,
                                      float* weights_out, void* workspace, size_t workspace_bytes, void* stream_) {
  size_t need = 0;
  int32_t st = spv_kv_attention_workspace_size(cache, seqs, d, weights_out != nullptr, &need);
  if (st != SPV_OK) return st;
  if (!q || !o || (weights_in && !weights_out)) return SPV_ERR_INVALID_ARG;
  if (((uintptr_t)q & 15u) || ((uintptr_t)o & 15u) || ((uintptr_t)lse & 3u) || ((uintptr_t)weights_in & 3u) ||
      ((uintptr_t)weights_out & 3u))
    return SPV_ERR_ALIGNMENT;
  if (!ctx || spv_on_device(ctx) != SPV_OK) return SPV_ERR_INVALID_ARG;
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u))) return SPV_ERR_WORKSPACE;
  cudaStream_t stream = (cudaStream_t)stream_;
  KvAttnArgs a;
  a.q = (const uint16_t*)q;
  a.o = (uint16_t*)o;
  a.lse = lse;
  a.w_in = weights_in;
  a.w_out = weights_out;
  a.counts = d->counts;
  a.q_stride_b = d->q_stride_b; a.q_stride_tok = d->q_stride_tok; a.q_stride_head = d->q_stride_head;
  a.o_stride_b = d->o_stride_b; a.o_stride_tok = d->o_stride_tok; a.o_stride_head = d->o_stride_head;
  a.w_stride_b = d->w_stride_b; a.w_stride_head = d->w_stride_head;
  a.batch = seqs->batch;
  a.tokens = d->tokens;
  a.heads = d->heads;
  a.group = d->heads / cache->kv_heads;
  a.block = cache->block;
  a.causal = d->causal;
  a.dtype = d->dtype;
  a.scale = d->softmax_scale > 0.0f ? d->softmax_scale : 1.0f / sqrtf((float)cache->head_dim);
  SpvProfScope prof(ctx, SPV_K_KV_ATTN, stream);
  return streams(cache, d) ? spv_kv_stream_run(ctx, cache, seqs, a, workspace, stream)
                           : spv_kv_prompt_run(ctx, cache, seqs, d, a, workspace, stream);
}
