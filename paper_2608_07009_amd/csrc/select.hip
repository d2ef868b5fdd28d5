// Scores of a selection's candidates (hisparse_select_records), and its host side.
//
//   keys   s_j = sum_e w_e max(0, q_e . k_j)
//   bounds s_j = largest_j . q+ + least_j . q-,  q+ = sum_e max(q_e, 0), q- = sum_e min(q_e, 0)
//   means  s_j = mean_j . sum_e q_e
//
// Products from bf16 MFMAs, 16 query rows by 16 candidates, sums in fp32. Which candidates these choose is
// settled in select_choose.hip.
#include "select.h"

namespace hisparse {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

constexpr int kScoreThreads = 256;
constexpr int kRowPad = 256;          // a row of scores is a multiple of this
constexpr size_t kMostScoreBytes = (size_t)1 << 30;

__device__ __forceinline__ uint16_t to_bf16(float x) {
  return (uint16_t)__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{x, 0.f}, bf16x2_t));
}

// ---- scores ----------------------------------------------------------------------------------

template <int KIND>
struct Shape : IndexShape<KIND> {
  using IndexShape<KIND>::KEYS;
  static constexpr int STEPS = IndexShape<KIND>::DIMS / 32;  // MFMAs of 16 rows x 16 candidates
  static constexpr int ROWS = KEYS ? 1 : 4;        // new tokens of a workgroup
  static constexpr int TILE = KEYS ? 1024 : 512;   // candidates of a workgroup
};

// Bounds and means: the sums over the heads of a token, exact in 64 bits, as three bf16 parts (24 bits:
// off by 2^-25 of the value). Row 4 i + part of the A operand, i the token; the fourth is zero.
template <int KIND>
__device__ __forceinline__ void linear_rows(const SelectArgs& a, int token0, int tokens, int h,
                                            uint16_t* s_a) {
  constexpr int DIMS = Shape<KIND>::DIMS, PITCH = DIMS + 8;
  for (int x = threadIdx.x; x < 4 * kIndexDims; x += kScoreThreads) {
    const int i = x / kIndexDims, d = x % kIndexDims;
    double pos = 0.0, neg = 0.0;
    if (i < tokens) query_sums<KIND>(a, token0 + i, h, d, pos, neg);
    auto put = [&](int at, double v) {
#pragma unroll
      for (int part = 0; part < 3; ++part) {
        const uint16_t b = to_bf16((float)v);
        s_a[(4 * i + part) * PITCH + at] = b;
        v -= bf16_value(b);
      }
      s_a[(4 * i + 3) * PITCH + at] = 0;
    };
    if (KIND == HISPARSE_INDEX_BOUNDS) put(d, neg);
    put(KIND == HISPARSE_INDEX_BOUNDS ? kIndexDims + d : d, pos);
  }
}

template <int KIND, int MT>
__global__ __launch_bounds__(kScoreThreads) void score_kernel(SelectArgs a) {
  using S = Shape<KIND>;
  constexpr bool KEYS = S::KEYS;
  __shared__ uint32_t s_norm[4];
  __shared__ float s_least[4][S::ROWS], s_most[4][S::ROWS];
  __shared__ __align__(16) uint16_t s_a[KEYS ? 8 : 16 * (S::DIMS + 8)];
  const int lane = threadIdx.x & 63, col = lane & 15, group = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t block = blockIdx.x, rest = block / (uint32_t)a.tiles;
  const int kt = (int)(block - rest * (uint32_t)a.tiles);
  const int tile = (int)(rest / (uint32_t)a.heads), h = (int)(rest - (uint32_t)tile * a.heads);
  const int row0 = a.row0 + tile * S::ROWS, row1 = min(row0 + S::ROWS, a.row0 + a.rows);
  for (int t = row0; t < row1;) {
    const int q = request_at(a, t);
    const RequestRows r = rows_of(a, q);
    if (t < r.begin || t >= r.begin + r.n) {
      ++t;
      continue;
    }
    const int token0 = t, tokens = min(row1, r.begin + r.n) - t;
    t += tokens;
    const int seen = seen_at(a, r.len - r.n + token0 + tokens - 1 - r.begin);
    if (seen <= a.top_k || kt * S::TILE >= seen) continue;
    bf16x8_t A[MT][S::STEPS];
    float w[KEYS ? MT * 4 : 1];
    if constexpr (KEYS) {
      const uint16_t* qrow = a.q + (int64_t)token0 * a.q_stride +
                             (int64_t)h * a.q_heads * kIndexDims + group * 8;
      const float* wrow = a.weights ? a.weights + ((int64_t)token0 * a.heads + h) * a.q_heads
                                    : nullptr;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int e = m * 16 + col;
#pragma unroll
        for (int k = 0; k < S::STEPS; ++k) {
          u32x4_t x = {};
          if (e < a.q_heads)
            x = *reinterpret_cast<const any_u32x4_t*>(qrow + e * kIndexDims + k * 32);
          A[m][k] = __builtin_bit_cast(bf16x8_t, x);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int y = m * 16 + group * 4 + i;
          w[m * 4 + i] = y < a.q_heads ? (wrow ? wrow[y] : 1.f) : 0.f;
        }
      }
    } else {
      __syncthreads();  // the last segment's operands are read
      linear_rows<KIND>(a, token0, tokens, h, s_a);
      __syncthreads();
#pragma unroll
      for (int k = 0; k < S::STEPS; ++k)
        A[0][k] = *reinterpret_cast<const bf16x8_t*>(s_a + col * (S::DIMS + 8) + k * 32 + group * 8);
    }
    float norm = 0.f;      // the largest sum of squares; NaN stays (its bits are above infinity's)
    uint32_t bits = 0;
    float least = INFINITY, most = -INFINITY;  // of this lane's row
    const int64_t out = ((int64_t)(token0 - a.row0) * a.heads + h) * a.row_pad;
    for (int base = kt * S::TILE + wave * (S::TILE / 4), end = min(base + S::TILE / 4, seen);
         base < end; base += 64) {
      u32x4_t x[4][S::STEPS];
      bool valid[4];
#pragma unroll
      for (int sub = 0; sub < 4; ++sub) {
        const int j = base + sub * 16 + col;
        const uint8_t* row = nullptr;
        int record;
        valid[sub] = j < end && find_row<KEYS>(a, q, h, j, row, record);
#pragma unroll
        for (int k = 0; k < S::STEPS; ++k) {
          x[sub][k] = u32x4_t{};
          if (valid[sub]) x[sub][k] = *reinterpret_cast<const u32x4_t*>(row + k * 64 + group * 16);
        }
      }
      float v[4];
#pragma unroll
      for (int sub = 0; sub < 4; ++sub) {
        float sq = 0.f, sum = 0.f;
#pragma unroll
        for (int k = 0; k < S::STEPS; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t b = x[sub][k][i];
            bits |= b & 0x7fff7fffu;
            sq += low_half(b) * low_half(b) + high_half(b) * high_half(b);
          }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          f32x4_t acc = {};
#pragma unroll
          for (int k = 0; k < S::STEPS; ++k)
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                A[m][k], __builtin_bit_cast(bf16x8_t, x[sub][k]), acc, 0, 0, 0);
          if constexpr (KEYS) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += w[m * 4 + i] * fmaxf(acc[i], 0.f);
          } else {
            sum = acc[0] + acc[1] + acc[2];
          }
        }
        if constexpr (KEYS) {
          sum += __shfl_xor(sum, 16);
          sum += __shfl_xor(sum, 32);
        }
        sq += __shfl_xor(sq, 16);
        sq += __shfl_xor(sq, 32);
        norm = __uint_as_float(max(__float_as_uint(norm), __float_as_uint(sq)));
        if (sum != sum) sum = __uint_as_float(kNan);
        v[sub] = valid[sub] ? sum : __uint_as_float(kPad);
      }
      if constexpr (KEYS) {
        const float s = group == 0 ? v[0] : group == 1 ? v[1] : group == 2 ? v[2] : v[3];
        if (base + lane < end) {
          a.scores[out + base + lane] = s;
          least = fminf(least, s);  // (a NaN, as padding is, is passed over)
          most = fmaxf(most, s);
        }
      } else {
        if (group < tokens)
#pragma unroll
          for (int sub = 0; sub < 4; ++sub)
            if (base + sub * 16 + col < end) {
              a.scores[out + group * a.heads * a.row_pad + base + sub * 16 + col] = v[sub];
              least = fminf(least, v[sub]);
              most = fmaxf(most, v[sub]);
            }
      }
    }
    // Largest norm of this tile's rows: 0 only if all are zero. Squares below the float range are made
    // up for.
    uint32_t nb = __float_as_uint(norm);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      nb = max(nb, (uint32_t)__shfl_xor((int)nb, d));
      bits |= (uint32_t)__shfl_xor((int)bits, d);
      if (KEYS || d < 16) {
        least = fminf(least, __shfl_xor(least, d));
        most = fmaxf(most, __shfl_xor(most, d));
      }
    }
    if (lane == 0)
      s_norm[wave] =
          bits ? __float_as_uint(sqrtf(__uint_as_float(nb)) * 1.01f + 0x1p-58f) : 0;
    if (KEYS ? lane == 0 : col == 0) {
      s_least[wave][KEYS ? 0 : group] = least;
      s_most[wave][KEYS ? 0 : group] = most;
    }
    __syncthreads();
    if (threadIdx.x < (unsigned)tokens) {
      uint32_t n = 0;
      least = INFINITY, most = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        n = max(n, s_norm[i]);
        least = fminf(least, s_least[i][threadIdx.x]);
        most = fmaxf(most, s_most[i][threadIdx.x]);
      }
      a.facts[((int64_t)(token0 + (int)threadIdx.x - a.row0) * a.heads + h) * a.tiles + kt] =
          TileFacts{__uint_as_float(n), least, most};
    }
    if (a.hist && kt == 0)  // added to by the next kernel
      for (int i = 0; i < tokens; ++i)
        for (int x = threadIdx.x; x < kLongBins; x += kScoreThreads)
          a.hist[((int64_t)(token0 + i - a.row0) * a.heads + h) * kLongBins + x] = 0;
    __syncthreads();
  }
}

// ---- host ------------------------------------------------------------------------------------

struct SelectPlan {
  int64_t candidates, row_pad, tiles, parts;
  bool is_long;
  int64_t row_bytes;  // of a new token, all kv heads
  int32_t tile_rows, tile_size;
};

int64_t whole(int64_t n, int64_t of) { return (n + of - 1) / of; }

SelectPlan plan_select(const hisparse_index_desc_t& x, const hisparse_batch_desc_t& b) {
  SelectPlan p{};
  const bool keys = x.kind == HISPARSE_INDEX_KEYS;
  p.candidates = keys ? (int64_t)b.max_records * b.tokens_per_record : b.max_records;
  const int tile = keys ? Shape<HISPARSE_INDEX_KEYS>::TILE : Shape<HISPARSE_INDEX_MEANS>::TILE;
  p.tile_size = shift_of(tile);
  p.tiles = whole(p.candidates, tile);
  p.parts = whole(p.candidates, kPart);
  const bool big = p.candidates > kRegisterRow;
  p.is_long = big && p.parts <= kMaxParts;
  p.row_pad = whole(p.candidates, big ? kPart : kRowPad) * (big ? kPart : kRowPad);
  // (those of rows of too many parts too: a workspace serves smaller batches)
  const int64_t words =
      p.row_pad + 3 * p.tiles + (big ? p.row_pad + kLongBins + p.parts + 3 : 0);
  p.row_bytes = words * 4 * b.kv_heads;
  p.tile_rows = keys ? 1 : Shape<HISPARSE_INDEX_MEANS>::ROWS;
  return p;
}

hipError_t launch_select(const SelectArgs& a, int kind, const SelectPlan& p, hipStream_t s) {
  const unsigned row_tiles = (unsigned)((a.rows + p.tile_rows - 1) / p.tile_rows);
  const dim3 grid(row_tiles * (unsigned)a.heads * (unsigned)a.tiles), block(kScoreThreads);
  constexpr int K = HISPARSE_INDEX_KEYS, B = HISPARSE_INDEX_BOUNDS, M = HISPARSE_INDEX_MEANS;
  if (kind == B) {
    hipLaunchKernelGGL((score_kernel<B, 1>), grid, block, 0, s, a);
  } else if (kind == M) {
    hipLaunchKernelGGL((score_kernel<M, 1>), grid, block, 0, s, a);
  } else {
    if (a.q_heads <= 16) hipLaunchKernelGGL((score_kernel<K, 1>), grid, block, 0, s, a);
    else if (a.q_heads <= 32) hipLaunchKernelGGL((score_kernel<K, 2>), grid, block, 0, s, a);
    else if (a.q_heads <= 64) hipLaunchKernelGGL((score_kernel<K, 4>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((score_kernel<K, 8>), grid, block, 0, s, a);
  }
  return launch_choose(a, kind, p.candidates, s);
}

}  // namespace
}  // namespace hisparse

extern "C" {

hisparse_status_t hisparse_validate_select(const hisparse_index_desc_t* x,
                                           const hisparse_batch_desc_t* b,
                                           const hisparse_select_desc_t* d) {
  hisparse_status_t st = hisparse_validate_index(x);
  if (st == HISPARSE_OK) st = hisparse_validate_batch(b);
  if (st != HISPARSE_OK) return st;
  if (!d || x->tokens_per_record != b->tokens_per_record) return HISPARSE_ERR_INVALID_ARG;
  if (d->q_heads < 1 || d->q_heads > (x->kind == HISPARSE_INDEX_KEYS ? 128 : 256) ||
      d->top_k < 1 || d->top_k > hisparse::kMaxTopK || d->first_records < 0 ||
      d->last_records < 0 || (int64_t)d->first_records + d->last_records > d->top_k ||
      d->q_token_stride < 0)
    return HISPARSE_ERR_INVALID_ARG;
  const hisparse::SelectPlan p = hisparse::plan_select(*x, *b);
  if ((int64_t)b->total_tokens * b->kv_heads > (int64_t)INT32_MAX ||
      p.candidates * b->kv_heads >= (1ll << 30))
    return HISPARSE_ERR_UNSUPPORTED;
  return HISPARSE_OK;
}

size_t hisparse_select_workspace_bytes(const hisparse_index_desc_t* x,
                                       const hisparse_batch_desc_t* b,
                                       const hisparse_select_desc_t* d) {
  using namespace hisparse;
  if (hisparse_validate_select(x, b, d) != HISPARSE_OK) return 0;
  const SelectPlan p = plan_select(*x, *b);
  const int64_t rows = b->total_tokens > 1 ? b->total_tokens : 1;
  const size_t tile = (size_t)(p.tile_rows * p.row_bytes);
  size_t bytes = (size_t)rows <= kMostScoreBytes / (size_t)p.row_bytes ? (size_t)(rows * p.row_bytes)
                                                                      : kMostScoreBytes;
  if (bytes < tile) bytes = tile;
  return (bytes + 255) / 256 * 256;
}

hisparse_status_t hisparse_select_records(const hisparse_index_desc_t* x,
                                          const hisparse_batch_desc_t* b,
                                          const hisparse_select_desc_t* d, const void* d_index,
                                          const int32_t* d_table, const int32_t* d_chunk_start,
                                          const int32_t* d_kv_len, const void* d_q,
                                          const float* d_weights, int32_t* d_sel,
                                          int32_t* d_records, int32_t* d_sel_len,
                                          void* d_workspace, size_t workspace_bytes, void* stream) {
  using namespace hisparse;
  const hisparse_status_t st = hisparse_validate_select(x, b, d);
  if (st != HISPARSE_OK) return st;
  const bool keys = x->kind == HISPARSE_INDEX_KEYS;
  if ((d_weights && !keys) || (d_sel_len && d->last_records == 0)) return HISPARSE_ERR_INVALID_ARG;
  if (!d_chunk_start && (int64_t)b->num_requests * b->max_chunk > b->total_tokens)
    return HISPARSE_ERR_INVALID_ARG;
  if ((uintptr_t)d_index % 16 != 0 || (uintptr_t)d_table % 4 != 0 ||
      (uintptr_t)d_chunk_start % 4 != 0 || (uintptr_t)d_kv_len % 4 != 0 || (uintptr_t)d_q % 2 != 0 ||
      (uintptr_t)d_weights % 4 != 0 || (uintptr_t)d_sel % 4 != 0 || (uintptr_t)d_records % 4 != 0 ||
      (uintptr_t)d_sel_len % 4 != 0 || (uintptr_t)d_workspace % 16 != 0)
    return HISPARSE_ERR_INVALID_ARG;
  if (keys && d_records && x->num_records * x->tokens_per_record > (int64_t)INT32_MAX)
    return HISPARSE_ERR_UNSUPPORTED;
  if (b->total_tokens == 0) return HISPARSE_OK;
  const SelectPlan p = plan_select(*x, *b);
  if (!d_index || !d_q || !d_sel || !d_workspace ||
      workspace_bytes < (size_t)(p.tile_rows * p.row_bytes))
    return HISPARSE_ERR_INVALID_ARG;
  // rows of a step: what the workspace holds, in whole tiles, and a launch's 2^32 threads
  int64_t step = (int64_t)(workspace_bytes / (size_t)p.row_bytes);
  const int64_t blocks_of_tile = p.tiles * b->kv_heads;
  const int64_t most = ((int64_t)UINT32_MAX / kScoreThreads / blocks_of_tile) * p.tile_rows;
  const int64_t most_chosen =
      (int64_t)UINT32_MAX / 1024 / ((p.is_long ? p.parts : 1) * b->kv_heads);
  if (step > most) step = most;
  if (step > most_chosen) step = most_chosen;
  if (step > b->total_tokens) step = b->total_tokens;
  else step = step / p.tile_rows * p.tile_rows;
  if (step < 1) return HISPARSE_ERR_UNSUPPORTED;
  SelectArgs a{};
  static_cast<BatchArgs&>(a) = batch_args(*b, d_table, d_chunk_start, d_kv_len);
  a.index = reinterpret_cast<const uint8_t*>(d_index);
  a.q = reinterpret_cast<const uint16_t*>(d_q);
  a.weights = d_weights;
  a.sel = d_sel;
  a.records = d_records;
  a.sel_len = d_sel_len;
  a.record_stride = x->record_stride;
  a.head_stride = x->head_stride;
  a.request_stride = x->request_stride;
  a.num_records = x->num_records;
  a.q_stride = d->q_token_stride;
  a.row_pad = p.row_pad;
  a.tiles = (int32_t)p.tiles;
  a.q_heads = d->q_heads;
  a.top_k = d->top_k;
  a.first = d->first_records;
  a.last = d->last_records;
  a.cand_shift = keys ? 0 : a.tpr_shift;
  a.tile_size = p.tile_size;
  a.parts = (int32_t)p.parts;
  const int64_t n = step * b->kv_heads;  // rows of scores
  a.scores = reinterpret_cast<float*>(d_workspace);
  a.facts = reinterpret_cast<TileFacts*>(a.scores + n * p.row_pad);
  if (p.is_long) {
    a.survivors = reinterpret_cast<int32_t*>(a.facts + n * p.tiles);
    a.hist = reinterpret_cast<uint32_t*>(a.survivors + n * p.row_pad);
    a.part_count = reinterpret_cast<int32_t*>(a.hist + n * kLongBins);
    a.bound = reinterpret_cast<float*>(a.part_count + n * p.parts);
  }
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const StreamDevice device(s);
  for (int64_t row0 = 0; row0 < b->total_tokens; row0 += step) {
    a.row0 = (int32_t)row0;
    a.rows = (int32_t)(b->total_tokens - row0 < step ? b->total_tokens - row0 : step);
    if (launch_select(a, x->kind, p, s) != hipSuccess) return HISPARSE_ERR_HIP;
  }
  return HISPARSE_OK;
}

}  // extern "C"
