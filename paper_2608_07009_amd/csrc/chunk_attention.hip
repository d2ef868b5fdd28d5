// Attention of chunks of new tokens over token records (hisparse_chunk_attention).
//
// For new token i of a request with n new and len cached tokens, and query head e on kv head h:
//   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j - m),  m the largest score,
// over the cached tokens j that it sees: j < len, j <= len - n + i (causal), j > len - n + i -
// window, and its record not padding.
//
// One wave per (new token, query head); its lanes share the dims, tokens one after the other with
// the running maximum and sum in fp32.
#include <math.h>

#include <algorithm>

#include "tokens.h"

namespace hisparse {
namespace {

struct ChunkArgs {
  const uint8_t* pool;
  const int32_t *table, *start, *kv_len;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  int64_t record_stride, head_stride, request_stride;
  int64_t q_stride, out_stride, table_request_stride, table_head_stride;
  int64_t num_records;
  KvLayout l;
  int32_t requests, kv_heads, g, total, max_chunk, max_tokens, window, causal;
  float scale_log2;
};

__device__ inline float bf16_to_f32(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ inline uint16_t f32_to_bf16(float x) {
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}

template <bool LATENT, bool FP8>
__global__ __launch_bounds__(64) void chunk_rows_kernel(ChunkArgs a) {
  constexpr int NQ = LATENT ? 9 : 2, NV = LATENT ? 8 : 2;
  const int H = a.kv_heads * a.g, lane = threadIdx.x;
  const int tok = blockIdx.x / H, e = blockIdx.x - tok * H, h = e / a.g;
  int req = -1, begin = 0, end = 0;
  if (a.start) {
    for (int r = 0; r < a.requests; ++r) {
      begin = min(max(a.start[r], 0), a.total);
      end = min(max(a.start[r + 1], begin), a.total);
      if (tok >= begin && tok < end) {
        req = r;
        break;
      }
    }
  } else if (tok < a.requests * a.max_chunk) {
    req = tok / a.max_chunk;
    begin = req * a.max_chunk;
    end = begin + a.max_chunk;
  }
  if (req < 0) return;
  const int len = a.kv_len ? min(max(a.kv_len[req], 0), a.max_tokens) : a.max_tokens;
  const int pos = len - (end - begin) + (tok - begin);
  const int hi = a.causal ? min(len, pos + 1) : len;
  const int lo = a.window ? max(0, pos - a.window + 1) : 0;
  const uint16_t* q = a.q + tok * a.q_stride + (int64_t)e * (LATENT ? 576 : 128);
  float qv[NQ], acc[NV], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int i = 0; i < NQ; ++i) qv[i] = bf16_to_f32(q[lane + 64 * i]);
#pragma unroll
  for (int i = 0; i < NV; ++i) acc[i] = 0.f;
  const int32_t* table = a.table + req * a.table_request_stride + h * a.table_head_stride;
  for (int j = lo; j < hi; ++j) {
    const int32_t r = table[j >> a.l.tpr_shift];
    if (r < 0 || r >= a.num_records) continue;
    const uint8_t* rec = a.pool + req * a.request_stride + h * a.head_stride + r * a.record_stride;
    const int t = j & ((1 << a.l.tpr_shift) - 1);
    const uint8_t* row = rec + (int64_t)t * a.l.row_bytes;
    float kv[NQ], vv[NV];
    if constexpr (!FP8) {
      const uint16_t* x = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
      for (int i = 0; i < NQ; ++i) kv[i] = bf16_to_f32(x[lane + 64 * i]);
#pragma unroll
      for (int i = 0; i < NV; ++i) vv[i] = LATENT ? kv[i] : bf16_to_f32(x[128 + lane + 64 * i]);
    } else {
      const float* sc = reinterpret_cast<const float*>(rec + a.l.scale_offset);
      const float sk = sc[LATENT ? t : 2 * t];
#pragma unroll
      for (int i = 0; i < (LATENT ? 8 : 2); ++i)
        kv[i] = __builtin_amdgcn_cvt_f32_fp8(row[lane + 64 * i], 0) * sk;
      if constexpr (LATENT)
        kv[8] = bf16_to_f32(
            reinterpret_cast<const uint16_t*>(rec + a.l.rope_offset + t * 128)[lane]);
#pragma unroll
      for (int i = 0; i < NV; ++i)
        vv[i] = LATENT ? kv[i]
                       : __builtin_amdgcn_cvt_f32_fp8(row[128 + lane + 64 * i], 0) * sc[2 * t + 1];
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NQ; ++i) s += qv[i] * kv[i];
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) s += __shfl_xor(s, x, 64);
    s *= a.scale_log2;
    const float m_new = fmaxf(m, s);
    const float alpha = exp2f(m - m_new), p = exp2f(s - m_new);
    l = l * alpha + p;
#pragma unroll
    for (int i = 0; i < NV; ++i) acc[i] = acc[i] * alpha + p * vv[i];
    m = m_new;
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  uint16_t* o = a.out + tok * a.out_stride + (int64_t)e * (LATENT ? 512 : 128);
#pragma unroll
  for (int i = 0; i < NV; ++i) o[lane + 64 * i] = f32_to_bf16(acc[i] * inv);
  if (a.lse && lane == 0)
    a.lse[(int64_t)tok * H + e] = l > 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace
}  // namespace hisparse

extern "C" {

hisparse_status_t hisparse_validate_chunk(const hisparse_kv_desc_t* kv,
                                          const hisparse_chunk_desc_t* c) {
  const hisparse_status_t st = hisparse_validate_kv(kv);
  if (st != HISPARSE_OK) return st;
  if (!c || c->num_requests < 1 || c->kv_heads < 1 || c->q_heads < 1 || c->q_heads > 256 ||
      (int64_t)c->num_requests * c->kv_heads > (1 << 20))
    return HISPARSE_ERR_INVALID_ARG;
  if (c->total_tokens < 0 || c->max_chunk < 1 || c->max_records < 1 ||
      (int64_t)c->max_records * kv->tokens_per_record > (1 << 30))
    return HISPARSE_ERR_INVALID_ARG;
  const int64_t H = (int64_t)c->kv_heads * c->q_heads;
  const int64_t d_v = kv->layout == HISPARSE_KV_GROUPED ? 128 : 512;
  if (c->q_token_stride < 0 || c->out_token_stride < H * d_v || c->table_request_stride < 0 ||
      c->table_head_stride < 0)
    return HISPARSE_ERR_INVALID_ARG;
  if ((c->flags & ~HISPARSE_CHUNK_CAUSAL) != 0 || c->window < 0 ||
      (c->window > 0 && !(c->flags & HISPARSE_CHUNK_CAUSAL)) || c->num_splits < 0 ||
      c->num_splits > 64)
    return HISPARSE_ERR_INVALID_ARG;
  if (!(c->scale > 0.f) || c->scale > 1e6f) return HISPARSE_ERR_INVALID_ARG;
  if (c->total_tokens * H > (int64_t)INT32_MAX) return HISPARSE_ERR_UNSUPPORTED;
  return HISPARSE_OK;
}

size_t hisparse_chunk_workspace_bytes(const hisparse_kv_desc_t* kv,
                                      const hisparse_chunk_desc_t* c) {
  if (hisparse_validate_chunk(kv, c) != HISPARSE_OK) return 0;
  return 0;
}

hisparse_status_t hisparse_chunk_attention(const hisparse_kv_desc_t* kv,
                                           const hisparse_chunk_desc_t* c, const void* d_pool,
                                           const int32_t* d_table, const int32_t* d_chunk_start,
                                           const int32_t* d_kv_len, const void* d_q, void* d_out,
                                           float* d_lse, void* d_workspace,
                                           size_t workspace_bytes, void* stream) {
  using namespace hisparse;
  const hisparse_status_t st = hisparse_validate_chunk(kv, c);
  if (st != HISPARSE_OK) return st;
  if (!d_chunk_start && (int64_t)c->num_requests * c->max_chunk > c->total_tokens)
    return HISPARSE_ERR_INVALID_ARG;
  if (c->total_tokens == 0) return HISPARSE_OK;
  if (!d_pool || !d_table || !d_q || !d_out || (uintptr_t)d_pool % 16 != 0 ||
      (uintptr_t)d_table % 4 != 0 || (uintptr_t)d_chunk_start % 4 != 0 ||
      (uintptr_t)d_kv_len % 4 != 0 || (uintptr_t)d_q % 2 != 0 || (uintptr_t)d_out % 2 != 0 ||
      (uintptr_t)d_lse % 4 != 0)
    return HISPARSE_ERR_INVALID_ARG;
  ChunkArgs a{};
  a.pool = reinterpret_cast<const uint8_t*>(d_pool);
  a.table = d_table;
  a.start = d_chunk_start;
  a.kv_len = d_kv_len;
  a.q = reinterpret_cast<const uint16_t*>(d_q);
  a.out = reinterpret_cast<uint16_t*>(d_out);
  a.lse = d_lse;
  a.record_stride = kv->record_stride;
  a.head_stride = kv->head_stride;
  a.request_stride = kv->request_stride;
  a.q_stride = c->q_token_stride;
  a.out_stride = c->out_token_stride;
  a.table_request_stride = c->table_request_stride;
  a.table_head_stride = c->table_head_stride;
  a.num_records = kv->num_records;
  a.l = kv_layout(*kv);
  a.requests = c->num_requests;
  a.kv_heads = c->kv_heads;
  a.g = c->q_heads;
  a.total = c->total_tokens;
  a.max_chunk = c->max_chunk;
  a.max_tokens = c->max_records << a.l.tpr_shift;
  a.window = c->window;
  a.causal = (c->flags & HISPARSE_CHUNK_CAUSAL) != 0;
  a.scale_log2 = c->scale * 1.4426950408889634f;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const StreamDevice device(s);
  const dim3 grid((unsigned)(c->total_tokens * c->kv_heads * c->q_heads));
  const bool fp8 = kv->type == HISPARSE_KV_FP8;
  if (kv->layout == HISPARSE_KV_GROUPED) {
    if (fp8) hipLaunchKernelGGL((chunk_rows_kernel<false, true>), grid, dim3(64), 0, s, a);
    else hipLaunchKernelGGL((chunk_rows_kernel<false, false>), grid, dim3(64), 0, s, a);
  } else {
    if (fp8) hipLaunchKernelGGL((chunk_rows_kernel<true, true>), grid, dim3(64), 0, s, a);
    else hipLaunchKernelGGL((chunk_rows_kernel<true, false>), grid, dim3(64), 0, s, a);
  }
  return hipGetLastError() == hipSuccess ? HISPARSE_OK : HISPARSE_ERR_HIP;
}

}  // extern "C"
