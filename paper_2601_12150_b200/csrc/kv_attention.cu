// Attention of the newest tokens' queries over the 8-bit key/value cache.
//
//   kv_attn_row_kernel     one CTA per (sequence, query, head): online softmax over chunks of 128 keys;
//   kv_attn_weight_kernel  one thread per key: the probabilities anew from the queries' log-sums, added up over
//                          the queries and the heads of a key head in a fixed order.
#include <type_traits>

#include "kv_attention.cuh"

namespace {

using namespace spv;

// <q, codes of a row> in fp32, from shared memory and a row of the pool.
template <int FMT, int D>
__device__ __forceinline__ float row_dot(const float* q, const uint8_t* row) {
  float s = 0.0f;
#pragma unroll 4
  for (int j = 0; j < D / 16; ++j) {
    const uint4 x = __ldg(reinterpret_cast<const uint4*>(row) + j);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      float y[4];
      kv_decode4<FMT>(w[t], y);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = fmaf(q[16 * j + 4 * t + e], y[e], s);
    }
  }
  return s;
}

template <int FMT, int DT, int D>
__global__ void __launch_bounds__(128) kv_attn_row_kernel(KvView c, KvAttnArgs a) {
  __shared__ float qs[D];
  __shared__ float ps[128];
  __shared__ float red[8];
  const int i = blockIdx.x / a.heads, head = blockIdx.x % a.heads, b = blockIdx.z, hk = head / a.group;
  const int len = kv_clamped(__ldg(c.lengths + b), c.max_length, c.status);
  const int n = a.counts ? kv_clamped(__ldg(a.counts + b), a.tokens, c.status) : a.tokens;
  if (i >= n) return;
  const int end = spv_kv_query_end(len, n, i, a.causal);
  const uint16_t* q = a.q + b * a.q_stride_b + i * a.q_stride_tok + head * a.q_stride_head;
  const int t = threadIdx.x;
  if (t < D / 2) {
    const float2 f = kv_unpack2<DT>(*reinterpret_cast<const uint32_t*>(q + 2 * t));
    qs[2 * t] = f.x * a.scale;
    qs[2 * t + 1] = f.y * a.scale;
  }
  const int32_t* row = c.table + b * c.table_stride;
  float m = -INFINITY, l = 0.0f, o = 0.0f;
  for (int j0 = 0; j0 < end; j0 += 128) {
    __syncthreads();
    const int j = j0 + t;
    float z = -INFINITY;
    if (j < end) {
      const int page = kv_page(row, j / a.block, c.pages, c.status);
      if (page >= 0) {
        const size_t ph = (size_t)page * c.kv_heads + hk;
        z = row_dot<FMT, D>(qs, c.k + spv_kv_row(page, c.kv_heads, hk, a.block, j) * D) * __ldg(c.k_scale + ph);
      }
    }
    float top = z;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
    if ((t & 31) == 0) red[t >> 5] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float m2 = fmaxf(m, top);
    if (m2 == -INFINITY) continue;                 // nothing seen yet (uniform over the CTA)
    const float p = z == -INFINITY ? 0.0f : expf(z - m2);
    ps[t] = p;
    float sum = p;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
    if ((t & 31) == 0) red[4 + (t >> 5)] = sum;
    __syncthreads();
    const float f = m == -INFINITY ? 0.0f : expf(m - m2);
    l = l * f + ((red[4] + red[5]) + (red[6] + red[7]));
    o *= f;
    m = m2;
    if (t < D) {
      const int keys = min(128, end - j0);
      for (int s = 0; s < keys; ++s) {
        const int page = __ldg(row + (j0 + s) / a.block);
        if ((uint32_t)page >= (uint32_t)c.pages) continue;
        const size_t ph = (size_t)page * c.kv_heads + hk;
        const uint32_t code = __ldg(c.v + (ph * a.block + (j0 + s) % a.block) * D + t);
        float y[4];
        kv_decode4<FMT>(code, y);
        o = fmaf(ps[s] * __ldg(c.v_scale + ph), y[0], o);
      }
    }
  }
  if (t < D) {
    const float r = l > 0.0f ? o / l : 0.0f;
    const uint32_t u = kv_pack2<DT>(r, 0.0f);
    a.o[b * a.o_stride_b + i * a.o_stride_tok + head * a.o_stride_head + t] = (uint16_t)u;
  }
  if (t == 0 && a.lse) a.lse[((size_t)b * a.tokens + i) * a.heads + head] = l > 0.0f ? m + logf(l) : -INFINITY;
}

template <int FMT, int DT, int D>
__global__ void __launch_bounds__(128) kv_attn_weight_kernel(KvView c, KvAttnArgs a) {
  __shared__ float qs[D];
  __shared__ float s_lse;
  const int b = blockIdx.z, hk = blockIdx.y, j = blockIdx.x * 128 + threadIdx.x;
  const int len = kv_clamped(__ldg(c.lengths + b), c.max_length, c.status);
  const int n = a.counts ? kv_clamped(__ldg(a.counts + b), a.tokens, c.status) : a.tokens;
  if (blockIdx.x * 128 >= len) return;
  const int page = j < len ? kv_page(c.table + b * c.table_stride, j / a.block, c.pages, c.status) : -1;
  const size_t ph = (size_t)max(page, 0) * c.kv_heads + hk;
  const uint8_t* key = c.k + (ph * a.block + j % a.block) * D;
  const float ks = __ldg(c.k_scale + ph);
  float w = 0.0f;
  for (int r = 0; r < n * a.group; ++r) {
    const int i = r / a.group, head = hk * a.group + r % a.group;
    __syncthreads();
    if (threadIdx.x < D / 2) {
      const uint16_t* q = a.q + b * a.q_stride_b + i * a.q_stride_tok + head * a.q_stride_head;
      const float2 f = kv_unpack2<DT>(*reinterpret_cast<const uint32_t*>(q + 2 * threadIdx.x));
      qs[2 * threadIdx.x] = f.x * a.scale;
      qs[2 * threadIdx.x + 1] = f.y * a.scale;
    }
    if (threadIdx.x == 0) s_lse = a.lse[((size_t)b * a.tokens + i) * a.heads + head];
    __syncthreads();
    if (page >= 0 && j < spv_kv_query_end(len, n, i, a.causal)) w += expf(row_dot<FMT, D>(qs, key) * ks - s_lse);
  }
  if (j < len) {
    const int64_t at = b * a.w_stride_b + hk * a.w_stride_head + j;
    a.w_out[at] = (a.w_in ? a.w_in[at] : 0.0f) + w;
  }
}

int32_t check_attn(const spv_kv_cache* c, const spv_kv_seqs* s, const spv_kv_attn_desc* d) {
  int32_t st = spv_kv_check_cache(c);
  if (st != SPV_OK) return st;
  if ((st = spv_kv_check_seqs(c, s)) != SPV_OK) return st;
  if (!d || d->tokens < 1 || d->heads < 1 || d->heads % c->kv_heads) return SPV_ERR_INVALID_ARG;
  if (d->dtype != SPV_BF16 && d->dtype != SPV_FP16) return SPV_ERR_UNSUPPORTED;
  if (d->causal != 0 && d->causal != 1) return SPV_ERR_INVALID_ARG;
  if (!(d->softmax_scale >= 0.0f) || d->softmax_scale > 1e30f) return SPV_ERR_INVALID_ARG;
  if ((int64_t)d->tokens * d->heads > INT32_MAX / 2) return SPV_ERR_UNSUPPORTED;
  // tiles of 32 slots are numbered in 31 bits
  if ((int64_t)s->batch * c->kv_heads * ((spv_kv_max_length(c, s) + 31) / 32) > INT32_MAX / 2) return SPV_ERR_UNSUPPORTED;
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
  else *bytes = want_weights ? spv_align_up((size_t)seqs->batch * d->tokens * d->heads * sizeof(float), 256) : 0;
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
  const KvView view = kv_view(ctx, cache, seqs);
  KvAttnArgs a;
  a.q = (const uint16_t*)q;
  a.o = (uint16_t*)o;
  a.lse = lse ? lse : (float*)(weights_out ? workspace : nullptr);
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
  if (streams(cache, d)) {
    a.lse = lse;
    return spv_kv_stream_run(ctx, cache, seqs, a, workspace, stream);
  }
  const dim3 rows(d->tokens * d->heads, 1, seqs->batch);
  const dim3 keys((view.max_length + 127) / 128, cache->kv_heads, seqs->batch);
  auto launch = [&](auto fmt, auto dt, auto dim) {
    kv_attn_row_kernel<fmt(), dt(), dim()><<<rows, 128, 0, stream>>>(view, a);
    if (weights_out) kv_attn_weight_kernel<fmt(), dt(), dim()><<<keys, 128, 0, stream>>>(view, a);
  };
  auto by_dim = [&](auto fmt, auto dt) {
    if (cache->head_dim == 64) launch(fmt, dt, std::integral_constant<int, 64>());
    else launch(fmt, dt, std::integral_constant<int, 128>());
  };
  auto by_type = [&](auto fmt) {
    if (d->dtype == SPV_BF16) by_dim(fmt, std::integral_constant<int, SPV_BF16>());
    else by_dim(fmt, std::integral_constant<int, SPV_FP16>());
  };
  if (cache->format == SPV_KV_INT8) by_type(std::integral_constant<int, SPV_KV_INT8>());
  else by_type(std::integral_constant<int, SPV_KV_E4M3>());
  return spv_launch_ok(ctx, weights_out ? 2 : 1);
}
