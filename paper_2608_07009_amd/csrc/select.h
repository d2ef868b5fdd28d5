// Selection of records by a cheap score: what its scores (select.hip) and its choice (select_choose.hip)
// share.
#pragma once

#include <math.h>

#include "batch.h"

namespace hisparse {

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef u32x4_t any_u32x4_t __attribute__((aligned(2)));  // queries may start at any element

// What the scores of padding, and (by the choice) of chosen candidates, are marked with; scores that are
// NaN are kNan.
constexpr uint32_t kPad = 0xffffffffu, kWin = 0x7fffffffu, kNan = 0x7fc00000u;
constexpr int kLongBins = 2048;       // of a long row's division
// Candidates of a long row's part. (64 heads, a row of 131072: 55 us; with parts of 8192 53, of 32768 59. 16 rows of
// 1048576: 344; 366 and 335.)
constexpr int kPart = 16384;
constexpr int kRegisterRow = 32768;   // a longer row is long
constexpr int kMaxParts = 1024;
// New tokens of a request from which waves have new tokens of their own; fewer are scored one by one, which
// reads the index for each. (Eight requests, 64 heads over 32768 keys: chunks of 3 take 69 us one by one and
// 86 by teams, of 4, 79 and 75. Bounds of 8192 pages, 4 requests x 8 kv heads: 2, 65 and 70; 4, 102 and 70.)
template <int KIND>
constexpr int kTeamChunk = KIND == HISPARSE_INDEX_KEYS ? 4 : 3;

struct TileFacts {
  // Largest norm of a tile's rows (of chunks of teams, only the step's last new token has it),
  // its least and largest score.
  float norm, least, most;
};

struct SelectArgs : BatchArgs {
  const uint8_t* index;
  const uint16_t* q;
  const float* weights;
  int32_t *sel, *records, *sel_len;
  // of this step's rows, each [rows][heads]:
  float* scores;       // [row_pad]
  TileFacts* facts;    // [tiles]
  // long rows:
  uint32_t* hist;      // [kLongBins]; null: no row is long
  int32_t* survivors;  // [row_pad], a part of kPart each
  int32_t* part_count; // [parts]
  float* bound;        // [3]: the error bound, the range of the scores
  int64_t record_stride, head_stride, request_stride, num_records, q_stride;
  int64_t row_pad;
  int32_t row0, rows;     // this step's rows of new tokens
  int32_t tiles, parts;   // of a row
  int32_t tile_size;      // candidates of a tile (log2)
  int32_t q_heads, top_k, first, last;
  int32_t cand_shift;     // tokens of a candidate (log2)
  int32_t tokens_of_request;  // that are scored one by one, at most
};

// Chooses from the scores of the step's rows; `candidates`: the most that a row has.
hipError_t launch_choose(const SelectArgs& a, int kind, int64_t candidates, hipStream_t stream);

template <int KIND>
struct IndexShape {
  static constexpr bool KEYS = KIND == HISPARSE_INDEX_KEYS;
  static constexpr int DIMS = KIND == HISPARSE_INDEX_BOUNDS ? 2 * kIndexDims : kIndexDims;
};

__device__ __forceinline__ float low_half(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high_half(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// Candidates that the new token at position p sees.
__device__ __forceinline__ int seen_at(const SelectArgs& a, int p) {
  return p < 0 ? 0 : (p >> a.cand_shift) + 1;
}

// Index row of candidate j of request q, kv head h; false if it is padding. record: what the caller
// knows the candidate by.
template <bool KEYS>
__device__ __forceinline__ bool find_row(const SelectArgs& a, int q, int h, int j,
                                         const uint8_t*& row, int& record) {
  const int entry = KEYS ? j >> a.tpr_shift : j;
  const int rec =
      a.table ? a.table[q * a.table_request_stride + h * a.table_head_stride + entry] : entry;
  if (rec < 0 || rec >= a.num_records) return false;
  const int in = KEYS ? j & ((1 << a.tpr_shift) - 1) : 0;
  row = a.index + q * a.request_stride + h * a.head_stride + (int64_t)rec * a.record_stride +
        in * kIndexRowBytes;
  record = KEYS ? (int)(((uint32_t)rec << a.tpr_shift) + in) : rec;
  return true;
}

// Bounds and means: the sums in 64 bits of dims 8 c .. 8 c + 7 over heads e0, e0 + step, .. of a kv head's
// queries, positive and negative ones apart (means: all in pos).
template <int KIND, int UNROLL>
__device__ __forceinline__ void query_sums(const SelectArgs& a, int token, int h, int c, int e0, int step,
                                           double (&pos)[8], double (&neg)[8]) {
  const uint16_t* q =
      a.q + (int64_t)token * a.q_stride + (int64_t)h * a.q_heads * kIndexDims + 8 * c;
#pragma unroll
  for (int i = 0; i < 8; ++i) pos[i] = neg[i] = 0.0;
#pragma unroll UNROLL
  for (int e = e0; e < a.q_heads; e += step) {
    const u32x4_t x = *reinterpret_cast<const any_u32x4_t*>(q + e * kIndexDims);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double v = i & 1 ? high_half(x[i >> 1]) : low_half(x[i >> 1]);
      if (KIND == HISPARSE_INDEX_BOUNDS && v < 0.0) neg[i] += v;
      else pos[i] += v;
    }
  }
}

}  // namespace hisparse
