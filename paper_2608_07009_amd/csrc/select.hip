// The best candidates of each new token by a cheap score (hisparse_select_records).
//
//   keys   s_j = sum_e w_e max(0, q_e . k_j)
//   bounds s_j = largest_j . q+ + least_j . q-,  q+ = sum_e max(q_e, 0), q- = sum_e min(q_e, 0)
//   means  s_j = mean_j . sum_e q_e
//
// Two kernels. score_kernel takes all s_j from bf16 MFMAs with fp32 sums. The choice is that of scores in
// 64 bits, which fp32 scores settle but for a few candidates: with
//   |s_j - exact| <= eps = 1.25 * 2^-15 A N,  A = sum_e |w_e| |q_e|, N = the largest |k_j| seen
// (keys: sums of 128 products, each step off by at most 2^-23, and of up to 128 heads, 2^-24 a step:
// 2^-16 + 2^-17; the others: 256 products, 2^-15, their three parts and what is left of q+ and q-, 2^-22)
// and with T in [lo, hi] the m-th largest s, candidates above hi + 2 eps are among the best m, those below
// lo - 2 eps are not, and those between are scored again in 64 bits (choose_kernel).
#include <math.h>

#include "batch.h"

namespace hisparse {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 any_u32x4 __attribute__((aligned(2)));  // queries may start at any element

constexpr int kScoreThreads = 256, kChooseThreads = 1024, kChooseWaves = kChooseThreads / 64;
constexpr int kBins = 2048;
constexpr int kList = 1024;           // candidates scored again that are kept in LDS
constexpr int kRowPad = 256;          // a row of scores is a multiple of this
constexpr size_t kMostScoreBytes = (size_t)1 << 30;
// What the scores of padding, and of candidates chosen among those scored again, are marked with.
constexpr uint32_t kPad = 0xffffffffu, kWin = 0x7fffffffu, kNan = 0x7fc00000u;

struct SelectArgs : BatchArgs {
  const uint8_t* index;
  const uint16_t* q;
  const float* weights;
  int32_t *sel, *records, *sel_len;
  float *scores, *norms;  // of this step's rows: [rows][heads][row_pad], [rows][heads][tiles]
  int64_t record_stride, head_stride, request_stride, num_records, q_stride;
  int64_t row_pad;
  int32_t row0, rows;     // this step's rows of new tokens
  int32_t tiles;          // key tiles of a row
  int32_t q_heads, top_k, first, last;
  int32_t cand_shift;     // tokens of a candidate (log2)
};

__device__ __forceinline__ float low(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
__device__ __forceinline__ uint16_t to_bf16(float x) {
  return (uint16_t)__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, 0.f}, bf16x2_t));
}
__device__ __forceinline__ float bf16_value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

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

// ---- scores ----------------------------------------------------------------------------------

template <int KIND>
struct Shape {
  static constexpr bool KEYS = KIND == HISPARSE_INDEX_KEYS;
  static constexpr int DIMS = KIND == HISPARSE_INDEX_BOUNDS ? 2 * kIndexDims : kIndexDims;
  static constexpr int STEPS = DIMS / 32;          // MFMAs of 16 rows x 16 candidates
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
    if (i < tokens) {
      const uint16_t* q = a.q + (int64_t)(token0 + i) * a.q_stride +
                          (int64_t)h * a.q_heads * kIndexDims + d;
      for (int e = 0; e < a.q_heads; ++e) {
        const double v = bf16_value(q[e * kIndexDims]);
        if (KIND == HISPARSE_INDEX_BOUNDS && v < 0.0) neg += v;
        else pos += v;
      }
    }
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
  __shared__ float s_norm[4];
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
          u32x4 x = {};
          if (e < a.q_heads)
            x = *reinterpret_cast<const any_u32x4*>(qrow + e * kIndexDims + k * 32);
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
    const int64_t out = ((int64_t)(token0 - a.row0) * a.heads + h) * a.row_pad;
    for (int base = kt * S::TILE + wave * (S::TILE / 4), end = min(base + S::TILE / 4, seen);
         base < end; base += 64) {
      u32x4 x[4][S::STEPS];
      bool valid[4];
#pragma unroll
      for (int sub = 0; sub < 4; ++sub) {
        const int j = base + sub * 16 + col;
        const uint8_t* row = nullptr;
        int record;
        valid[sub] = j < end && find_row<KEYS>(a, q, h, j, row, record);
#pragma unroll
        for (int k = 0; k < S::STEPS; ++k) {
          x[sub][k] = u32x4{};
          if (valid[sub]) x[sub][k] = *reinterpret_cast<const u32x4*>(row + k * 64 + group * 16);
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
            sq += low(b) * low(b) + high(b) * high(b);
          }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          f32x4 acc = {};
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
        if (base + lane < end) a.scores[out + base + lane] = s;
      } else {
        if (group < tokens)
#pragma unroll
          for (int sub = 0; sub < 4; ++sub)
            if (base + sub * 16 + col < end)
              a.scores[out + group * a.heads * a.row_pad + base + sub * 16 + col] = v[sub];
      }
    }
    // Largest norm of this tile's rows: 0 only if all are zero. Squares below the float range are made
    // up for.
    uint32_t nb = __float_as_uint(norm);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      nb = max(nb, (uint32_t)__shfl_xor((int)nb, d));
      bits |= (uint32_t)__shfl_xor((int)bits, d);
    }
    if (lane == 0)
      s_norm[wave] = bits ? sqrtf(__uint_as_float(nb)) * 1.01f + 0x1p-58f : 0.f;
    __syncthreads();
    if (threadIdx.x < (unsigned)tokens) {
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) most = max(most, __float_as_uint(s_norm[i]));
      a.norms[((int64_t)(token0 + (int)threadIdx.x - a.row0) * a.heads + h) * a.tiles + kt] =
          __uint_as_float(most);
    }
    __syncthreads();
  }
}

// ---- the choice ------------------------------------------------------------------------------

// 64-bit scores in the order of the choice: NaN above everything, -0 as 0.
__device__ __forceinline__ uint64_t ordered(double x) {
  if (x != x) return ~0ull;
  const int64_t b = __double_as_longlong(x + 0.0);
  return b < 0 ? ~(uint64_t)b : (uint64_t)b | 0x8000000000000000ull;
}

struct ChooseShared {
  uint32_t hist[kBins];
  uint64_t score[kList];
  int list[kList];
  double q[2 * kIndexDims];            // bounds and means: the sums over the heads
  uint32_t wave_a[kChooseWaves], wave_b[kChooseWaves];
  double wave_d[kChooseWaves], wave_e[kChooseWaves], wave_f[kChooseWaves];
  int count, bin, above, in_bin;
};
// Behind it for keys: the queries, [q_heads] rows of 128 and 4 more (their lanes' banks apart).
constexpr int kQPitch = kIndexDims + 4;

template <class F>
__device__ __forceinline__ uint32_t group_reduce(uint32_t x, uint32_t* waves, F&& f) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x = f(x, (uint32_t)__shfl_xor((int)x, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  x = waves[0];
  for (int i = 1; i < kChooseWaves; ++i) x = f(x, waves[i]);
  return x;
}
__device__ __forceinline__ uint32_t ordered32(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered32(uint32_t b) {
  return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}

template <int KIND>
struct Chooser {
  static constexpr bool KEYS = Shape<KIND>::KEYS;
  const SelectArgs& a;
  ChooseShared& s;
  const uint16_t* s_q;
  const float* wrow;
  float* row;           // this row's scores
  int q, h, seen, first, last0;  // forced: j < first, j >= last0
  int lane, wave;
  int lo, hi;           // this wave's candidates
  bool all;             // every candidate is scored again
  float sure, maybe;    // above sure: chosen; below maybe: not
  bool zero;            // every score is 0

  __device__ __forceinline__ bool rankable(int j, float x) const {
    return __float_as_uint(x) != kPad && j >= first && j < last0;
  }
  __device__ __forceinline__ bool is_sure(float x) const { return !all && x > sure; }
  __device__ __forceinline__ bool is_open(float x) const { return all || (x >= maybe && !(x > sure)); }

  // f(j, score) for this wave's candidates, four in a row per lane.
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    for (int base = lo + lane * 4; base < hi; base += 256) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(row + base);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (base + i < hi) f(base + i, x[i]);
    }
  }

  // The score of candidate j in 64 bits. j is the same in all lanes, and so is the result.
  __device__ __forceinline__ uint64_t exact(int j) const {
    const uint8_t* key = nullptr;
    int record;
    find_row<KEYS>(a, q, h, j, key, record);
    double sum = 0.0;
    if constexpr (KEYS) {
      const u32x4* k = reinterpret_cast<const u32x4*>(key);
      for (int e = lane; e < a.q_heads; e += 64) {
        double dot = 0.0;
#pragma unroll 4
        for (int p = 0; p < kIndexDims / 8; ++p) {
          const u32x4 kx = k[p];
          const uint16_t* qe = s_q + e * kQPitch + p * 8;
          const u32x2 q0 = *reinterpret_cast<const u32x2*>(qe);
          const u32x2 q1 = *reinterpret_cast<const u32x2*>(qe + 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t y = i < 2 ? q0[i] : q1[i - 2];
            dot = fma((double)low(kx[i]), (double)low(y), dot);
            dot = fma((double)high(kx[i]), (double)high(y), dot);
          }
        }
        const double positive = dot > 0.0 ? dot : dot == dot ? 0.0 : dot;
        sum += (wrow ? (double)wrow[e] : 1.0) * positive;
      }
    } else {
      constexpr int PER = Shape<KIND>::DIMS / 64;
#pragma unroll
      for (int i = 0; i < PER / 2; ++i) {
        const int d = lane * PER + 2 * i;
        const uint32_t x = *reinterpret_cast<const uint32_t*>(key + 2 * d);
        sum = fma((double)low(x), s.q[d], sum);
        sum = fma((double)high(x), s.q[d + 1], sum);
      }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    return ordered(sum);
  }

  // eps, and the queries in LDS.
  __device__ __forceinline__ float error_bound(int token, uint16_t* s_qw, const float* norms,
                                               int tiles) {
    const uint16_t* qrow = a.q + (int64_t)token * a.q_stride + (int64_t)h * a.q_heads * kIndexDims;
    double A = 0.0, W = 0.0, Q = 0.0;  // sums over this wave's heads; all lanes alike
    if constexpr (KEYS) {
      for (int e = wave; e < a.q_heads; e += kChooseWaves) {
        const uint16_t x0 = qrow[e * kIndexDims + 2 * lane], x1 = qrow[e * kIndexDims + 2 * lane + 1];
        s_qw[e * kQPitch + 2 * lane] = x0;
        s_qw[e * kQPitch + 2 * lane + 1] = x1;
        const double f0 = bf16_value(x0), f1 = bf16_value(x1);
        double sq = f0 * f0 + f1 * f1;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sq += __shfl_xor(sq, d);
        const double n = sqrt(sq), w = wrow ? fabs((double)wrow[e]) : 1.0;
        A += w * n;
        W += w;
        Q = n > Q || n != n ? n : Q;
      }
    } else {
      if (threadIdx.x < kIndexDims) {
        double pos = 0.0, neg = 0.0;
        for (int e = 0; e < a.q_heads; ++e) {
          const double v = bf16_value(qrow[e * kIndexDims + threadIdx.x]);
          if (KIND == HISPARSE_INDEX_BOUNDS && v < 0.0) neg += v;
          else pos += v;
        }
        if (KIND == HISPARSE_INDEX_BOUNDS) {
          s.q[threadIdx.x] = neg;
          s.q[kIndexDims + threadIdx.x] = pos;
        } else {
          s.q[threadIdx.x] = pos;
        }
        double sq = pos * pos + neg * neg;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sq += __shfl_xor(sq, d);
        A = Q = sqrt(sq);  // the two waves' parts: their sum bounds the whole
        W = 0.5;
      }
    }
    if (lane == 0) {
      s.wave_d[wave] = A;
      s.wave_e[wave] = W;
      s.wave_f[wave] = Q;
    }
    uint32_t most = 0;
    for (int i = threadIdx.x; i < tiles; i += kChooseThreads)
      most = max(most, __float_as_uint(norms[i]));
    const float N = __uint_as_float(
        group_reduce(most, s.wave_a, [](uint32_t x, uint32_t y) { return max(x, y); }));
    A = W = Q = 0.0;
    for (int i = 0; i < kChooseWaves; ++i) {
      A += s.wave_d[i];
      W += s.wave_e[i];
      Q += s.wave_f[i];
    }
    // the last term: what inputs and sums below the normal range are off by
    const float AN = (float)A * 1.01f * N;
    const float eps = AN * 0x1.4p-15f + (float)W * (N + (float)Q + 1.f) * 0x1p-118f;
    return A == 0.0 && N < INFINITY ? 0.f : N == 0.f && A < INFINITY ? 0.f : eps;
  }

  // Marks the m best of the rankable candidates: those above `sure`, and others by marks in their scores.
  __device__ void choose(int m, float eps) {
    zero = eps == 0.f;
    all = zero || !(eps < INFINITY);
    if (!all) {
      uint32_t least = ~0u, most = 0, count = 0;
      each([&](int j, float x) {
        if (!rankable(j, x)) return;
        ++count;
        least = min(least, ordered32(x));
        most = max(most, ordered32(x));
      });
      float from = unordered32(group_reduce(least, s.wave_a, [](uint32_t x, uint32_t y) { return min(x, y); }));
      float to = unordered32(group_reduce(most, s.wave_b, [](uint32_t x, uint32_t y) { return max(x, y); }));
      const int rankables = (int)group_reduce(count, s.wave_a, [](uint32_t x, uint32_t y) { return x + y; });
      all = rankables <= m;  // nothing to choose
      int need = m;
      for (int round = 0; round < 4 && from < to && !all; ++round) {
        const float scale = (float)kBins / (to - from);
        auto bin_of = [&](float x) { return min((int)((x - from) * scale), kBins - 1); };
        for (int i = threadIdx.x; i < kBins; i += kChooseThreads) s.hist[i] = 0;
        __syncthreads();
        each([&](int j, float x) {
          if (rankable(j, x) && x >= from && x <= to) atomicAdd(&s.hist[bin_of(x)], 1u);
        });
        __syncthreads();
        find_bin(need);
        const int bin = s.bin, in_bin = s.in_bin;
        need -= s.above;
        least = ~0u;
        most = 0;
        each([&](int j, float x) {
          if (!rankable(j, x) || !(x >= from && x <= to) || bin_of(x) != bin) return;
          least = min(least, ordered32(x));
          most = max(most, ordered32(x));
        });
        from = unordered32(group_reduce(least, s.wave_a, [](uint32_t x, uint32_t y) { return min(x, y); }));
        to = unordered32(group_reduce(most, s.wave_b, [](uint32_t x, uint32_t y) { return max(x, y); }));
        if (in_bin <= kList / 4) break;
      }
      // rounded outwards
      sure = nextafterf(to + 2.f * eps, INFINITY);
      maybe = nextafterf(from - 2.f * eps, -INFINITY);
    }
    // how many are sure, which are open
    if (threadIdx.x == 0) s.count = 0;
    __syncthreads();
    uint32_t n_sure = 0;
    each([&](int j, float x) {
      if (!rankable(j, x)) return;
      if (is_sure(x)) {
        ++n_sure;
      } else if (is_open(x)) {
        const int at = atomicAdd(&s.count, 1);
        if (at < kList) s.list[at] = j;
      }
    });
    const int need = m - (int)group_reduce(n_sure, s.wave_a, [](uint32_t x, uint32_t y) { return x + y; });
    const int open = s.count;
    __syncthreads();
    if (need >= open) {  // (all of them: fewer rankable candidates than asked for)
      each([&](int j, float x) {
        if (rankable(j, x) && is_open(x)) row[j] = __uint_as_float(kWin);
      });
    } else if (open <= kList && !zero) {
      for (int i = wave; i < open; i += kChooseWaves) {
        const uint64_t x = exact(s.list[i]);
        if (lane == 0) s.score[i] = x;
      }
      __syncthreads();
      for (int i = threadIdx.x; i < open; i += kChooseThreads) {
        const uint64_t x = s.score[i];
        const int j = s.list[i];
        int better = 0;
        for (int y = 0; y < open; ++y)
          better += s.score[y] > x || (s.score[y] == x && s.list[y] < j);
        if (better < need) row[j] = __uint_as_float(kWin);
      }
    } else {
      choose_many(need);
    }
    __syncthreads();  // the marks are read by other waves
  }

  // The bin in which the need-th from the top lies.
  __device__ __forceinline__ void find_bin(int need) {
    // thread t has bins kBins - 1 - 2 t and the next lower one
    const int t = threadIdx.x;
    const uint32_t c0 = s.hist[kBins - 1 - 2 * t], c1 = s.hist[kBins - 2 - 2 * t];
    const int inc = wave_inclusive((int)(c0 + c1));
    if (lane == 63) s.wave_a[wave] = (uint32_t)inc;
    __syncthreads();
    int before = inc - (int)(c0 + c1);
    for (int i = 0; i < wave; ++i) before += (int)s.wave_a[i];
    if (before < need && before + (int)c0 >= need) {
      s.bin = kBins - 1 - 2 * t;
      s.above = before;
      s.in_bin = (int)c0;
    } else if (before + (int)c0 < need && before + (int)(c0 + c1) >= need) {
      s.bin = kBins - 2 - 2 * t;
      s.above = before + (int)c0;
      s.in_bin = (int)c1;
    }
    __syncthreads();
  }

  // More open candidates than the list holds (thousands of equal scores, or no error bound): the need-th
  // largest in 64 bits is found 8 bits at a time, the scores worked out anew each time.
  __device__ void choose_many(int need) {
    uint64_t prefix = zero ? ordered(0.0) : 0;
    for (int shift = 56; shift >= 0 && !zero; shift -= 8) {
      for (int i = threadIdx.x; i < kBins; i += kChooseThreads) s.hist[i] = 0;
      __syncthreads();
      open_ones([&](int j) {
        const uint64_t x = exact(j);
        if (lane == 0 && (shift == 56 || x >> (shift + 8) == prefix))
          atomicAdd(&s.hist[(int)(x >> shift) & 255], 1u);
      });
      __syncthreads();
      find_bin(need);
      prefix = prefix << 8 | (uint64_t)s.bin;
      need -= s.above;
      __syncthreads();
    }
    const int equal = need;  // of the need-th score, how many are wanted
    uint32_t mine = 0;
    open_ones([&](int j) { mine += zero || exact(j) == prefix; });
    if (lane == 0) s.wave_b[wave] = mine;
    __syncthreads();
    int before = 0;
    for (int i = 0; i < wave; ++i) before += (int)s.wave_b[i];
    open_ones([&](int j) {
      const uint64_t x = zero ? prefix : exact(j);
      const bool wins = x > prefix || (x == prefix && before < equal);
      before += x == prefix;
      if (wins && lane == 0) row[j] = __uint_as_float(kWin);
    });
  }
  // f(j) for this wave's open candidates in ascending order, j the same in all lanes.
  template <class F>
  __device__ __forceinline__ void open_ones(F&& f) const {
    for (int base = lo; base < hi; base += 64) {
      const int j = base + lane;
      const float x = j < hi ? row[j] : 0.f;
      uint64_t todo = __ballot(j < hi && rankable(j, x) && is_open(x));
      while (todo) {
        f(base + __builtin_ctzll(todo));
        todo &= todo - 1;
      }
    }
  }
};

template <int KIND>
__global__ __launch_bounds__(kChooseThreads) void choose_kernel(SelectArgs a) {
  constexpr bool KEYS = Shape<KIND>::KEYS;
  extern __shared__ __align__(16) uint8_t s_mem[];
  ChooseShared& s = *reinterpret_cast<ChooseShared*>(s_mem);
  uint16_t* s_q = reinterpret_cast<uint16_t*>(s_mem + sizeof(ChooseShared));
  const int local = (int)(blockIdx.x / (uint32_t)a.heads), h = (int)(blockIdx.x - (uint32_t)local * a.heads);
  const int token = a.row0 + local;
  const int q = request_at(a, token);
  const RequestRows r = rows_of(a, q);
  if (token < r.begin || token >= r.begin + r.n) return;
  const int p = r.len - r.n + token - r.begin;
  const int seen = seen_at(a, p), chosen = min(seen, a.top_k);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int span = (((seen + kChooseWaves - 1) / kChooseWaves) + 255) & ~255;
  const int64_t slot = (int64_t)local * a.heads + h;
  Chooser<KIND> c{a, s, s_q,
                  KEYS && a.weights ? a.weights + ((int64_t)token * a.heads + h) * a.q_heads : nullptr,
                  a.scores + slot * a.row_pad, q, h, seen, min(a.first, seen), max(seen - a.last, 0),
                  lane, wave, (int)min((int64_t)wave * span, (int64_t)seen),
                  (int)min((int64_t)(wave + 1) * span, (int64_t)seen), false, 0.f, 0.f, false};
  const bool scored = seen > a.top_k;
  if (scored) {
    const float eps = c.error_bound(token, s_q, a.norms + slot * a.tiles,
                                    (seen + Shape<KIND>::TILE - 1) / Shape<KIND>::TILE);
    // the places that forced candidates take (the newest one's is kept even if it is padding)
    uint32_t forced = 0;
    for (int i = threadIdx.x; i < a.first + a.last; i += kChooseThreads) {
      const int j = i < a.first ? i : seen - 1 - (i - a.first);
      forced += __float_as_uint(c.row[j]) != kPad || j == seen - 1;
    }
    const int taken = (int)group_reduce(forced, s.wave_a, [](uint32_t x, uint32_t y) { return x + y; });
    if (a.top_k > taken) {
      c.choose(a.top_k - taken, eps);
    } else {
      c.sure = INFINITY;
    }
  }
  // The chosen ones in ascending order; the newest has a place of its own.
  const int own = a.last > 0 ? seen - 1 : -1;
  auto is_in = [&](int j) {
    if (j == own) return false;
    if (!scored) {
      const uint8_t* at;
      int record;
      return find_row<KEYS>(a, q, h, j, at, record);
    }
    const float x = c.row[j];
    const uint32_t b = __float_as_uint(x);
    if (b == kPad) return false;
    return b == kWin || j < c.first || j >= c.last0 || c.is_sure(x);
  };
  int mine = 0;
  for (int base = c.lo; base < c.hi; base += 64)
    mine += __popcll(__ballot(base + lane < c.hi && is_in(base + lane)));
  __syncthreads();
  if (lane == 0) s.wave_a[wave] = (uint32_t)mine;
  __syncthreads();
  int at = 0, total = 0;
  for (int i = 0; i < kChooseWaves; ++i) {
    if (i < wave) at += (int)s.wave_a[i];
    total += (int)s.wave_a[i];
  }
  const int64_t out = ((int64_t)token * a.heads + h) * a.top_k;
  auto put = [&](int place, int j) {
    const uint8_t* x;
    int record = -1;
    const bool there = j >= 0 && find_row<KEYS>(a, q, h, j, x, record);
    a.sel[out + place] = there ? j : -1;
    if (a.records) a.records[out + place] = there ? record : -1;
  };
  for (int base = c.lo; base < c.hi; base += 64) {
    const int j = base + lane;
    const bool in = j < c.hi && is_in(j);
    const uint64_t mask = __ballot(in);
    if (in) put(at + __popcll(mask & ((1ull << lane) - 1)), j);
    at += __popcll(mask);
  }
  for (int i = total + (int)threadIdx.x; i < a.top_k; i += kChooseThreads)
    if (own < 0 || i != chosen - 1) put(i, -1);
  if (threadIdx.x == 0) {
    if (own >= 0) put(chosen - 1, own);
    if (a.sel_len && h == 0) {
      const int t = 1 << a.cand_shift;
      a.sel_len[token] = chosen > 0 ? (chosen - 1) * t + (p & (t - 1)) + 1 : 0;
    }
  }
}

// ---- host ------------------------------------------------------------------------------------

struct SelectPlan {
  int64_t candidates, row_pad, tiles, row_bytes;  // bytes of one new token's scores
  int32_t tile_rows;
};

SelectPlan plan_select(const hisparse_index_desc_t& x, const hisparse_batch_desc_t& b) {
  SelectPlan p{};
  const bool keys = x.kind == HISPARSE_INDEX_KEYS;
  p.candidates = keys ? (int64_t)b.max_records * b.tokens_per_record : b.max_records;
  p.row_pad = (p.candidates + kRowPad - 1) / kRowPad * kRowPad;
  const int tile = keys ? Shape<HISPARSE_INDEX_KEYS>::TILE : Shape<HISPARSE_INDEX_MEANS>::TILE;
  p.tiles = (p.candidates + tile - 1) / tile;
  p.row_bytes = (p.row_pad + p.tiles) * b.kv_heads * 4;
  p.tile_rows = keys ? 1 : Shape<HISPARSE_INDEX_MEANS>::ROWS;
  return p;
}

template <int KIND>
void launch_choose(const SelectArgs& a, hipStream_t s) {
  const size_t lds = sizeof(ChooseShared) + (KIND == HISPARSE_INDEX_KEYS ? a.q_heads * kQPitch * 2 : 0);
  hipLaunchKernelGGL(choose_kernel<KIND>, dim3((unsigned)(a.rows * a.heads)), dim3(kChooseThreads),
                     lds, s, a);
}

void launch_select(const SelectArgs& a, int kind, int tile_rows, hipStream_t s) {
  const unsigned row_tiles = (unsigned)((a.rows + tile_rows - 1) / tile_rows);
  const dim3 grid(row_tiles * (unsigned)a.heads * (unsigned)a.tiles), block(kScoreThreads);
  constexpr int K = HISPARSE_INDEX_KEYS, B = HISPARSE_INDEX_BOUNDS, M = HISPARSE_INDEX_MEANS;
  if (kind == K) {
    if (a.q_heads <= 16) hipLaunchKernelGGL((score_kernel<K, 1>), grid, block, 0, s, a);
    else if (a.q_heads <= 32) hipLaunchKernelGGL((score_kernel<K, 2>), grid, block, 0, s, a);
    else if (a.q_heads <= 64) hipLaunchKernelGGL((score_kernel<K, 4>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((score_kernel<K, 8>), grid, block, 0, s, a);
    launch_choose<K>(a, s);
  } else if (kind == B) {
    hipLaunchKernelGGL((score_kernel<B, 1>), grid, block, 0, s, a);
    launch_choose<B>(a, s);
  } else {
    hipLaunchKernelGGL((score_kernel<M, 1>), grid, block, 0, s, a);
    launch_choose<M>(a, s);
  }
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
  const int64_t most_chosen = (int64_t)UINT32_MAX / kChooseThreads / b->kv_heads;
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
  a.scores = reinterpret_cast<float*>(d_workspace);
  a.norms = a.scores + step * b->kv_heads * p.row_pad;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const StreamDevice device(s);
  for (int64_t row0 = 0; row0 < b->total_tokens; row0 += step) {
    a.row0 = (int32_t)row0;
    a.rows = (int32_t)(b->total_tokens - row0 < step ? b->total_tokens - row0 : step);
    launch_select(a, x->kind, p.tile_rows, s);
  }
  return hipGetLastError() == hipSuccess ? HISPARSE_OK : HISPARSE_ERR_HIP;
}

}  // extern "C"
