// Index rows of records from their keys (hisparse_summarize_records).
//
//   bounds: least_d = min_t K_td, largest_d = max_t K_td     means: mean_d = sum_t K_td / tokens
// over the tokens t that the record holds.
//
// A wave owns a record of one kv head. A row of keys is 16 (bf16) or 8 (8-bit) lanes of 16 bytes, so the
// wave takes 4 or 8 tokens at a time, four of those in flight. Its groups of lanes are joined at the end,
// each step over half of the elements of the one before, so that 16 tokens' records are not mostly joining (all
// elements at each step, through LDS: 8-bit bounds of 16 tokens 70 us, now 36). HBM-bound: the keys are
// read once (half of each record's bytes), one or two rows written. 4 prompts of 32768 tokens, 8 kv heads,
// records of 64: bf16 268 MB of keys in 45 us (means) and 47 (bounds), 5.7 to 6 TB/s; 8-bit 142 MB with the
// scales in 25 and 29. What single tokens write to, and few prompts, is a launch and a chain of loads: 3.7 us.
//
// Which records a wave has follows from the lengths alone: request q may own the waves from
//   floor(start_q / t) + 2 q   on, of which it has floor(start_q+1 / t) - floor(start_q / t) + 2,
// at least floor(n / t) + 2, and n new tokens lie in at most floor((n + t - 2) / t) + 1 records, which is
// no more. So a batch takes total / t + 2 requests of them whatever its lengths are.
#include <math.h>

#include "batch.h"
#include "fetch_device.h"

namespace hisparse {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

struct SummarizeArgs : BatchArgs {
  const uint8_t* pool;
  uint8_t* index;
  int64_t record_stride, head_stride, request_stride, num_records;
  int64_t index_record, index_head, index_request, index_records;
  int32_t row_bytes, scale_offset;
  uint32_t waves;      // of one kv head
  FastDiv div_waves;
};

// minNum drops a NaN: what propagates it.
__device__ __forceinline__ float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float most(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <bool BOUNDS>
struct Sums {
  float lo, hi;  // means: the sum in lo
  __device__ __forceinline__ void start() {
    lo = BOUNDS ? INFINITY : 0.f;
    hi = -INFINITY;
  }
  __device__ __forceinline__ void add(float x) {
    if (BOUNDS) {
      lo = least(lo, x);
      hi = most(hi, x);
    } else {
      lo += x;
    }
  }
  __device__ __forceinline__ void add(const Sums& x) {
    if (BOUNDS) {
      lo = least(lo, x.lo);
      hi = most(hi, x.hi);
    } else {
      lo += x.lo;
    }
  }
};

// a and b joined over lanes `lanes` (8, 16 or 32) apart: a in lanes without that bit, b in those with it.
template <int lanes>
__device__ __forceinline__ void exchange(float& a, float& b) {
  if constexpr (lanes == 8) {
    const bool up = threadIdx.x & 8;
    const float other = __shfl_xor(up ? a : b, 8);
    a = up ? b : a;
    b = other;
  } else {
    const auto r =
        lanes == 16
            ? __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false)
            : __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    a = __uint_as_float(r[0]);
    b = __uint_as_float(r[1]);
  }
}
template <int lanes, int N, bool BOUNDS, int E>
__device__ __forceinline__ void join(Sums<BOUNDS> (&sum)[E]) {
#pragma unroll
  for (int e = 0; e < N; ++e) {
    exchange<lanes>(sum[e].lo, sum[e + N].lo);
    if (BOUNDS) exchange<lanes>(sum[e].hi, sum[e + N].hi);
    sum[e].add(sum[e + N]);
  }
}

__device__ __forceinline__ uint32_t pack(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2_t));
}

// Request of wave w of a kv head, and the number of its first wave.
__device__ __forceinline__ int request_of_wave(const SummarizeArgs& a, int w, int& first) {
  auto first_of = [&](int q) {
    return (min(max(a.start[q], 0), a.total) >> a.tpr_shift) + 2 * q;
  };
  if (!a.start) {
    const int q = w / ((a.max_chunk >> a.tpr_shift) + 2);
    first = q * ((a.max_chunk >> a.tpr_shift) + 2);
    return min(q, a.requests);
  }
  int lo = 0, hi = a.requests;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first_of(mid) <= w) lo = mid;
    else hi = mid;
  }
  first = first_of(lo);
  return lo;
}

template <bool FP8, bool BOUNDS>
__global__ __launch_bounds__(256) void summarize_kernel(SummarizeArgs a) {
  constexpr int LANES = FP8 ? 8 : 16, E = kIndexDims / LANES;  // lanes of a row, elements of a lane
  constexpr int GROUPS = 64 / LANES, DEEP = 4;
  const int lane = threadIdx.x & 63, col = lane & (LANES - 1), group = lane / LANES;
  const uint32_t wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = (int)fastdiv(wave, a.div_waves);
  if (h >= a.heads) return;
  const int w = (int)(wave - (uint32_t)h * a.waves);
  int first;
  const int q = request_of_wave(a, w, first);
  if (q >= a.requests) return;
  const RequestRows rows = rows_of(a, q);
  const int t = 1 << a.tpr_shift;
  const int j = (max(rows.len - rows.n, 0) >> a.tpr_shift) + w - first;  // its record
  if (rows.n == 0 || w < first || j > ((rows.len - 1) >> a.tpr_shift) || rows.len == 0) return;
  const int64_t rec =
      a.table ? a.table[q * a.table_request_stride + h * a.table_head_stride + j] : j;
  if (rec < 0 || rec >= a.num_records || rec >= a.index_records) return;
  const uint8_t* record =
      a.pool + q * a.request_stride + h * a.head_stride + rec * a.record_stride;
  const int count = min(t, rows.len - (j << a.tpr_shift));
  Sums<BOUNDS> sum[E];
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e].start();
  for (int base = 0; base < count; base += GROUPS * DEEP) {
    u32x4 x[DEEP];
    float scale[DEEP];
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
      const int tok = base + d * GROUPS + group;
      if (tok < count) {
        x[d] = *reinterpret_cast<const u32x4*>(record + (int64_t)tok * a.row_bytes + col * 16);
        if (FP8) scale[d] = *reinterpret_cast<const float*>(record + a.scale_offset + tok * 8);
      }
    }
#pragma unroll
    for (int d = 0; d < DEEP; ++d) {
      if (base + d * GROUPS + group >= count) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (FP8) {
          const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[d][i], false);
          const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[d][i], true);
          sum[4 * i].add(lo[0] * scale[d]);
          sum[4 * i + 1].add(lo[1] * scale[d]);
          sum[4 * i + 2].add(hi[0] * scale[d]);
          sum[4 * i + 3].add(hi[1] * scale[d]);
        } else {
          sum[2 * i].add(__uint_as_float(x[d][i] << 16));
          sum[2 * i + 1].add(__uint_as_float(x[d][i] & 0xffff0000u));
        }
      }
    }
  }
  // each step leaves a lane half of its elements, at last two
  join<32, E / 2>(sum);
  join<16, E / 4>(sum);
  if constexpr (FP8) join<8, E / 8>(sum);
  const int at = col * E + (lane >> 5) * (E / 2) + (lane >> 4 & 1) * (E / 4) + (FP8 ? (lane >> 3 & 1) * 2 : 0);
  const float tokens = (float)count;
  uint32_t* out = reinterpret_cast<uint32_t*>(a.index + q * a.index_request + h * a.index_head +
                                              rec * a.index_record) + at / 2;
  *out = BOUNDS ? pack(sum[0].lo, sum[1].lo) : pack(sum[0].lo / tokens, sum[1].lo / tokens);
  if (BOUNDS) out[kIndexRowBytes / 4] = pack(sum[0].hi, sum[1].hi);
}

int32_t index_record_bytes(const hisparse_index_desc_t& d) {
  return d.kind == HISPARSE_INDEX_KEYS ? d.tokens_per_record * kIndexRowBytes
         : d.kind == HISPARSE_INDEX_BOUNDS ? 2 * kIndexRowBytes : kIndexRowBytes;
}

}  // namespace
}  // namespace hisparse

extern "C" {

hisparse_status_t hisparse_validate_index(const hisparse_index_desc_t* d) {
  if (!d || d->kind < HISPARSE_INDEX_KEYS || d->kind > HISPARSE_INDEX_MEANS)
    return HISPARSE_ERR_INVALID_ARG;
  const int32_t t = d->tokens_per_record;
  if (t < 1 || t > 4096 || (t & (t - 1)) != 0) return HISPARSE_ERR_INVALID_ARG;
  if (d->num_records < 1 || d->num_records > 0x7FFFFFFFLL) return HISPARSE_ERR_INVALID_ARG;
  if (d->record_stride < hisparse::index_record_bytes(*d) || d->record_stride > INT32_MAX ||
      d->record_stride % 16 != 0 || d->head_stride < 0 || d->head_stride % 16 != 0 ||
      d->request_stride < 0 || d->request_stride % 16 != 0)
    return HISPARSE_ERR_INVALID_ARG;
  return HISPARSE_OK;
}

hisparse_status_t hisparse_summarize_records(const hisparse_kv_desc_t* kv,
                                             const hisparse_index_desc_t* index,
                                             const hisparse_batch_desc_t* b, const void* d_pool,
                                             const int32_t* d_table, const int32_t* d_chunk_start,
                                             const int32_t* d_kv_len, void* d_index,
                                             void* stream) {
  using namespace hisparse;
  hisparse_status_t st = hisparse_validate_kv(kv);
  if (st == HISPARSE_OK) st = hisparse_validate_index(index);
  if (st == HISPARSE_OK) st = hisparse_validate_batch(b);
  if (st != HISPARSE_OK) return st;
  if (index->kind == HISPARSE_INDEX_KEYS || kv->tokens_per_record != b->tokens_per_record ||
      index->tokens_per_record != b->tokens_per_record)
    return HISPARSE_ERR_INVALID_ARG;
  if (b->kv_heads > 1 && index->head_stride < index_record_bytes(*index))
    return HISPARSE_ERR_INVALID_ARG;
  if (!d_chunk_start && (int64_t)b->num_requests * b->max_chunk > b->total_tokens)
    return HISPARSE_ERR_INVALID_ARG;
  if ((uintptr_t)d_pool % 16 != 0 || (uintptr_t)d_index % 16 != 0 || (uintptr_t)d_table % 4 != 0 ||
      (uintptr_t)d_chunk_start % 4 != 0 || (uintptr_t)d_kv_len % 4 != 0)
    return HISPARSE_ERR_INVALID_ARG;
  if (kv->layout != HISPARSE_KV_GROUPED) return HISPARSE_ERR_UNSUPPORTED;
  if (b->total_tokens == 0) return HISPARSE_OK;
  if (!d_pool || !d_index) return HISPARSE_ERR_INVALID_ARG;
  SummarizeArgs a{};
  static_cast<BatchArgs&>(a) = batch_args(*b, d_table, d_chunk_start, d_kv_len);
  a.pool = reinterpret_cast<const uint8_t*>(d_pool);
  a.index = reinterpret_cast<uint8_t*>(d_index);
  a.record_stride = kv->record_stride;
  a.head_stride = kv->head_stride;
  a.request_stride = kv->request_stride;
  a.num_records = kv->num_records;
  a.index_record = index->record_stride;
  a.index_head = index->head_stride;
  a.index_request = index->request_stride;
  a.index_records = index->num_records;
  const KvLayout l = kv_layout(*kv);
  a.row_bytes = l.row_bytes;
  a.scale_offset = l.scale_offset;
  const int64_t waves =
      d_chunk_start ? (b->total_tokens >> a.tpr_shift) + 2 * (int64_t)b->num_requests
                    : b->num_requests * (((int64_t)b->max_chunk >> a.tpr_shift) + 2);
  const int64_t all = waves * b->kv_heads;
  if ((all + 3) * 64 > (int64_t)UINT32_MAX) return HISPARSE_ERR_UNSUPPORTED;
  a.waves = (uint32_t)waves;
  a.div_waves = make_fastdiv(a.waves);
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const StreamDevice device(s);
  const dim3 grid((unsigned)((all + 3) / 4));
  const bool bounds = index->kind == HISPARSE_INDEX_BOUNDS, fp8 = kv->type == HISPARSE_KV_FP8;
  if (fp8 && bounds) hipLaunchKernelGGL((summarize_kernel<true, true>), grid, dim3(256), 0, s, a);
  else if (fp8) hipLaunchKernelGGL((summarize_kernel<true, false>), grid, dim3(256), 0, s, a);
  else if (bounds) hipLaunchKernelGGL((summarize_kernel<false, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((summarize_kernel<false, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError() == hipSuccess ? HISPARSE_OK : HISPARSE_ERR_HIP;
}

}  // extern "C"
