// Block tables, slot maps and positions of a batch from its lengths (hisparse_plan_tokens).
//
//   start_q = sum of the new tokens n of the requests before q, kv_q' = kv_q + n_q
//   request q begins records have_q .. want_q - 1, have = ceil(kv / t), want = ceil((kv + n) / t);
//   they are entries used + P_q, used + P_q + 1, ... of the free list, P_q = sum of want - have before q
//   token i of q: position p = kv_q + i, slot = record(p / t) * t + p % t
//
// Two prefix sums over the requests and a few words a row: a call is its launches. Small batches take one
// workgroup, which does the requests and then the rows. Larger ones take a second launch for the rows, whose
// workgroups each add up the requests' records again: that needs nothing kept between the launches
// but the outputs themselves, so the lengths may be updated in place. 64 requests of a token: 4.5 us; of 512:
// 6.6 us, most of both the launches.
#include "batch.h"

namespace hisparse {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
// Rows and requests up to which one workgroup does it all (of 64 requests, 64 rows: 4.5 us, 5.6 in two
// launches; 2048 rows: 5.8 and 6.3; 4096 rows: 7.8 and 6.5).
constexpr int kOneGroupRows = 2048, kOneGroupRequests = 2048;

struct PlanArgs {
  const int32_t *new_len, *kv_len, *free_list, *free_used;
  int32_t *table, *start, *kv_out, *used_out, *positions;
  int64_t* slots;
  int64_t table_stride;
  int32_t requests, total, max_chunk, max_len, tpr_shift, num_free;
};

struct Shared {
  uint32_t wave_sum[kWaves];
  int start[kThreads + 1], old[kThreads], prefix[kThreads];
};

// Exclusive prefix sum over the workgroup, sums held to cap; total: of all threads.
__device__ __forceinline__ uint32_t group_exclusive(uint32_t x, uint32_t cap, uint32_t* wave_sum,
                                                    uint32_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t inc = wave_inclusive_held(x, cap);
  __syncthreads();  // the last round's readers of wave_sum are done
  if (lane == 63) wave_sum[wave] = inc;
  __syncthreads();
  uint32_t s = lane < kWaves ? wave_sum[lane] : 0;
  s = wave_inclusive_held(s, cap);
  total = (uint32_t)last_lane((int)s);
  const uint32_t before = wave ? (uint32_t)__builtin_amdgcn_readlane((int)s, wave - 1) : 0;
  const uint32_t prev = (uint32_t)__shfl_up((int)inc, 1);
  return min(before + (lane ? prev : 0), cap);
}

// Requests' starts and lengths. One workgroup.
__device__ __forceinline__ void plan_requests(const PlanArgs& a, Shared& s) {
  const uint32_t cap = (uint32_t)a.total;
  const int t1 = (1 << a.tpr_shift) - 1;
  const int used = a.free_used ? min(max(*a.free_used, 0), a.num_free) : 0;
  uint32_t begin = 0;
  int records = 0;
  for (int base = 0; base < a.requests; base += kThreads) {
    const int r = base + threadIdx.x;
    int n = 0, old = 0;
    if (r < a.requests) {
      old = a.kv_len ? min(max(a.kv_len[r], 0), a.max_len) : 0;
      n = min(min(max(a.new_len[r], 0), a.max_chunk), a.max_len - old);
      n = min(n, a.total);
    }
    uint32_t sum, fresh;
    const uint32_t mine = min(begin + group_exclusive((uint32_t)n, cap, s.wave_sum, sum), cap);
    n = (int)min((uint32_t)n, cap - mine);
    group_exclusive((uint32_t)(((old + n + t1) >> a.tpr_shift) - ((old + t1) >> a.tpr_shift)), cap,
                    s.wave_sum, fresh);
    if (r < a.requests) {
      a.start[r] = (int)mine;
      a.kv_out[r] = old + n;
    }
    begin = min(begin + sum, cap);
    records += (int)fresh;  // at most one per row, so at most total
  }
  if (threadIdx.x == 0) {
    a.start[a.requests] = (int)begin;
    if (a.used_out) *a.used_out = used + records;
  }
}

// Rows [row0, row1): reads the starts and lengths that plan_requests has written.
__device__ __forceinline__ void plan_rows(const PlanArgs& a, Shared& s, int row0, int row1,
                                          int used_before) {
  const uint32_t cap = (uint32_t)a.total;
  const int t = 1 << a.tpr_shift;
  int taken = 0;
  for (int base = 0; base < a.requests; base += kThreads) {
    const int r = base + threadIdx.x, count = min(kThreads, a.requests - base);
    int begin = 0, n = 0, old = 0;
    if (r < a.requests) {
      begin = a.start[r];
      n = a.start[r + 1] - begin;
      old = a.kv_out[r] - n;
    }
    uint32_t fresh;
    const int mine = (int)group_exclusive(
        (uint32_t)(((old + n + t - 1) >> a.tpr_shift) - ((old + t - 1) >> a.tpr_shift)), cap,
        s.wave_sum, fresh);
    if ((int)threadIdx.x < count) {
      s.start[threadIdx.x] = begin;
      s.old[threadIdx.x] = old;
      s.prefix[threadIdx.x] = taken + mine;
      if ((int)threadIdx.x == count - 1) s.start[count] = begin + n;
    }
    taken += (int)fresh;
    __syncthreads();
    const int first = max(row0, s.start[0]), last = min(row1, s.start[count]);
    for (int row = first + (int)threadIdx.x; row < last; row += kThreads) {
      int lo = 0, hi = count;  // the last request that starts at or before the row
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s.start[mid] <= row) lo = mid;
        else hi = mid;
      }
      const int kv = s.old[lo], p = kv + row - s.start[lo], e = p >> a.tpr_shift;
      const int have = (kv + t - 1) >> a.tpr_shift;
      int32_t* entry = a.table + (int64_t)(base + lo) * a.table_stride + e;
      int rec;
      if (a.free_list && e >= have) {
        const int at = used_before + s.prefix[lo] + e - have;
        rec = at < a.num_free ? a.free_list[at] : -1;
        if ((p & (t - 1)) == 0) *entry = rec;  // each record's first token writes its entry
      } else {
        rec = *entry;
      }
      if (a.positions) a.positions[row] = p;
      if (a.slots) a.slots[row] = rec < 0 ? -1 : ((int64_t)rec << a.tpr_shift) + (p & (t - 1));
    }
    __syncthreads();
  }
  for (int row = max(row0, a.start[a.requests]) + (int)threadIdx.x; row < row1; row += kThreads) {
    if (a.positions) a.positions[row] = 0;
    if (a.slots) a.slots[row] = -1;
  }
}

__global__ __launch_bounds__(kThreads) void plan_kernel(PlanArgs a) {
  __shared__ Shared s;
  const int used = a.free_used ? min(max(*a.free_used, 0), a.num_free) : 0;
  plan_requests(a, s);
  __syncthreads();  // the starts and lengths are read back by other threads of this workgroup
  plan_rows(a, s, 0, a.total, used);
}

__global__ __launch_bounds__(kThreads) void plan_requests_kernel(PlanArgs a) {
  __shared__ Shared s;
  plan_requests(a, s);
}

// free_used may be used_out: the first launch has overwritten it, so what it held is that less the records.
__global__ __launch_bounds__(kThreads) void plan_rows_kernel(PlanArgs a) {
  __shared__ Shared s;
  int used = 0;
  if (a.free_used && a.free_used != a.used_out) {
    used = min(max(*a.free_used, 0), a.num_free);
  } else if (a.free_used) {
    const int t = 1 << a.tpr_shift;
    int records = 0;
    for (int base = 0; base < a.requests; base += kThreads) {
      const int r = base + threadIdx.x;
      int mine = 0;
      if (r < a.requests) {
        const int now = a.kv_out[r], old = now - (a.start[r + 1] - a.start[r]);
        mine = ((now + t - 1) >> a.tpr_shift) - ((old + t - 1) >> a.tpr_shift);
      }
      uint32_t sum;
      group_exclusive((uint32_t)mine, (uint32_t)a.total, s.wave_sum, sum);
      records += (int)sum;
    }
    used = *a.used_out - records;
  }
  const int64_t row0 = (int64_t)blockIdx.x * kThreads;
  plan_rows(a, s, (int)row0, (int)min(row0 + kThreads, (int64_t)a.total), used);
}

}  // namespace
}  // namespace hisparse

extern "C" {

hisparse_status_t hisparse_validate_batch(const hisparse_batch_desc_t* b) {
  if (!b || b->num_requests < 1 || b->kv_heads < 1 ||
      (int64_t)b->num_requests * b->kv_heads > (1 << 20))
    return HISPARSE_ERR_INVALID_ARG;
  const int32_t t = b->tokens_per_record;
  if (t < 1 || t > 4096 || (t & (t - 1)) != 0) return HISPARSE_ERR_INVALID_ARG;
  if (b->total_tokens < 0 || b->max_chunk < 1 || b->max_records < 1 ||
      (int64_t)b->max_records * t > (1 << 30))
    return HISPARSE_ERR_INVALID_ARG;
  if (b->table_request_stride < 0 || b->table_head_stride < 0) return HISPARSE_ERR_INVALID_ARG;
  return HISPARSE_OK;
}

hisparse_status_t hisparse_plan_tokens(const hisparse_batch_desc_t* b, const int32_t* d_new_len,
                                       const int32_t* d_kv_len, const int32_t* d_free,
                                       int32_t num_free, const int32_t* d_free_used,
                                       int32_t* d_table, int32_t* d_chunk_start,
                                       int32_t* d_kv_len_out, int32_t* d_free_used_out,
                                       int32_t* d_positions, int64_t* d_slots, void* stream) {
  using namespace hisparse;
  const hisparse_status_t st = hisparse_validate_batch(b);
  if (st != HISPARSE_OK) return st;
  if (!d_new_len || !d_table || !d_chunk_start || !d_kv_len_out || num_free < 0 ||
      (num_free > 0) != (d_free != nullptr))
    return HISPARSE_ERR_INVALID_ARG;
  for (const void* p : {(const void*)d_new_len, (const void*)d_kv_len, (const void*)d_free,
                        (const void*)d_free_used, (const void*)d_table, (const void*)d_chunk_start,
                        (const void*)d_kv_len_out, (const void*)d_free_used_out,
                        (const void*)d_positions})
    if ((uintptr_t)p % 4 != 0) return HISPARSE_ERR_INVALID_ARG;
  if ((uintptr_t)d_slots % 8 != 0) return HISPARSE_ERR_INVALID_ARG;
  if (b->table_head_stride != 0 ||
      (d_free && b->num_requests > 1 && b->table_request_stride < b->max_records))
    return HISPARSE_ERR_INVALID_ARG;
  if ((int64_t)num_free + b->total_tokens > INT32_MAX) return HISPARSE_ERR_UNSUPPORTED;
  PlanArgs a{};
  a.new_len = d_new_len;
  a.kv_len = d_kv_len;
  a.free_list = d_free;
  a.free_used = d_free_used;
  a.table = d_table;
  a.start = d_chunk_start;
  a.kv_out = d_kv_len_out;
  a.used_out = d_free_used_out;
  a.positions = d_positions;
  a.slots = d_slots;
  a.table_stride = b->table_request_stride;
  a.requests = b->num_requests;
  a.total = b->total_tokens;
  a.max_chunk = b->max_chunk;
  a.max_len = b->max_records * b->tokens_per_record;
  a.tpr_shift = shift_of(b->tokens_per_record);
  a.num_free = num_free;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const StreamDevice device(s);
  if (a.total <= kOneGroupRows && a.requests <= kOneGroupRequests) {
    hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kThreads), 0, s, a);
  } else {
    hipLaunchKernelGGL(plan_requests_kernel, dim3(1), dim3(kThreads), 0, s, a);
    if (a.total > 0) {
      const unsigned groups = (unsigned)(((int64_t)a.total + kThreads - 1) / kThreads);
      hipLaunchKernelGGL(plan_rows_kernel, dim3(groups), dim3(kThreads), 0, s, a);
    }
  }
  return hipGetLastError() == hipSuccess ? HISPARSE_OK : HISPARSE_ERR_HIP;
}

}  // extern "C"
