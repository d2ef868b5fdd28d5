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

// The last request that starts at or before row t (0 if none does). The same in all lanes of a wave, which
// look at 64 starts at a time.
__device__ __forceinline__ int request_at(const BatchArgs& a, int t) {
  if (!a.start) return min(t / a.max_chunk, a.requests - 1);
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.requests;
  while (n > 1) {
    const int step = (n + 63) >> 6, at = lane * step;
    const bool before = at < n && a.start[lo + min(at, n - 1)] <= t;
    const int c = max((int)__popcll(__ballot(before)) - 1, 0);  // (no start: the first request)
    lo += c * step;
    n = min(step, n - c * step);
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
// f of all lanes' values; `none` is its neutral one. (Six moves in the vector unit: a shuffle by way of LDS
// takes ten times as long.)
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lane_moved_or(uint32_t none, uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)x, CTRL, ROWS, 0xf, false);
}
template <class F>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t x, uint32_t none, F f) {
  x = f(x, lane_moved_or<0x111, 0xf>(none, x));
  x = f(x, lane_moved_or<0x112, 0xf>(none, x));
  x = f(x, lane_moved_or<0x114, 0xf>(none, x));
  x = f(x, lane_moved_or<0x118, 0xf>(none, x));
  x = f(x, lane_moved_or<0x142, 0xa>(none, x));
  x = f(x, lane_moved_or<0x143, 0xc>(none, x));
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double lane_moved64(double x) {  // 0 where nothing comes from
  const uint64_t b = (uint64_t)__double_as_longlong(x);
  const uint32_t lo = (uint32_t)lane_moved<CTRL, ROWS>((int)(uint32_t)b);
  const uint32_t hi = (uint32_t)lane_moved<CTRL, ROWS>((int)(uint32_t)(b >> 32));
  return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
// The sum over the lanes, in lane 63.
__device__ __forceinline__ double wave_sum64(double x) {
  x += lane_moved64<0x111>(x);
  x += lane_moved64<0x112>(x);
  x += lane_moved64<0x114>(x);
  x += lane_moved64<0x118>(x);
  x += lane_moved64<0x142, 0xa>(x);
  return x + lane_moved64<0x143, 0xc>(x);
}
// The sum over each 16 lanes, in all of them (rotations).
__device__ __forceinline__ double sum16_64(double x) {
  x += lane_moved64<0x128>(x);
  x += lane_moved64<0x124>(x);
  x += lane_moved64<0x122>(x);
  return x + lane_moved64<0x121>(x);
}
__device__ __forceinline__ int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }

}  // namespace hisparse
