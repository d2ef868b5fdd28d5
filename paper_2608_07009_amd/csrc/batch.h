// What the calls that take a hisparse_batch_desc_t share: host checks, which request a row of new tokens
// belongs to, sums and prefix sums across a wave.
#pragma once

#include "internal.h"
#include "tokens.h"

namespace hisparse {

constexpr int kIndexDims = 128;
constexpr int kIndexRowBytes = 2 * kIndexDims;

inline int shift_of(int32_t power_of_two) {
  int s = 0;
  while ((1 << s) < power_of_two) ++s;
  return s;
}

struct BatchArgs {
  const int32_t *table, *start, *kv_len;  // any may be null
  int64_t table_request_stride, table_head_stride;
  int32_t requests, heads, total, max_chunk, max_len, tpr_shift;
};

inline BatchArgs batch_args(const hisparse_batch_desc_t& b, const int32_t* table,
                            const int32_t* start, const int32_t* kv_len) {
  BatchArgs a{};
  a.table = table;
  a.start = start;
  a.kv_len = kv_len;
  a.table_request_stride = b.table_request_stride;
  a.table_head_stride = b.table_head_stride;
  a.requests = b.num_requests;
  a.heads = b.kv_heads;
  a.total = b.total_tokens;
  a.max_chunk = b.max_chunk;
  a.max_len = b.max_records * b.tokens_per_record;
  a.tpr_shift = shift_of(b.tokens_per_record);
  return a;
}

// New tokens [begin, begin + n) and cached tokens of request r, as hisparse_chunk_attention reads them.
struct RequestRows {
  int begin, n, len;
};
__device__ __forceinline__ RequestRows rows_of(const BatchArgs& a, int r) {
  RequestRows q;
  if (a.start) {
    q.begin = min(max(a.start[r], 0), a.total);
    q.n = min(min(max(a.start[r + 1], q.begin), a.total) - q.begin, a.max_chunk);
  } else {
    q.begin = r * a.max_chunk;  // at most total
    q.n = a.max_chunk;
  }
  q.len = a.kv_len ? min(max(a.kv_len[r], 0), a.max_len) : a.max_len;
  return q;
}

// The last request that starts at or before row t (0 if none does).
__device__ __forceinline__ int request_at(const BatchArgs& a, int t) {
  if (!a.start) return min(t / a.max_chunk, a.requests - 1);
  int lo = 0, hi = a.requests;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a.start[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Lane moves inside the vector unit.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int lane_moved(int x) {  // 0 where nothing comes from
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_inclusive(int x) {
  x += lane_moved<0x111>(x);  // 16 lanes: shifts by 1, 2, 4, 8
  x += lane_moved<0x112>(x);
  x += lane_moved<0x114>(x);
  x += lane_moved<0x118>(x);
  x += lane_moved<0x142, 0xa>(x);         // lane 15 of rows 0 and 2 to the row behind
  return x + lane_moved<0x143, 0xc>(x);  // lane 31 to the upper half
}
// The same with sums held to cap (values in [0, cap]): in unsigned arithmetic none wraps.
__device__ __forceinline__ uint32_t wave_inclusive_held(uint32_t x, uint32_t cap) {
  x = min(x + (uint32_t)lane_moved<0x111>((int)x), cap);
  x = min(x + (uint32_t)lane_moved<0x112>((int)x), cap);
  x = min(x + (uint32_t)lane_moved<0x114>((int)x), cap);
  x = min(x + (uint32_t)lane_moved<0x118>((int)x), cap);
  x = min(x + (uint32_t)lane_moved<0x142, 0xa>((int)x), cap);
  return min(x + (uint32_t)lane_moved<0x143, 0xc>((int)x), cap);
}
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }

}  // namespace hisparse
