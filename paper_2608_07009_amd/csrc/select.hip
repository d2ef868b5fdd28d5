// Scores of a selection's candidates (hisparse_select_records), and its host side.
//
//   keys   s_j = sum_e w_e max(0, q_e . k_j)
//   bounds s_j = largest_j . q+ + least_j . q-,  q+ = sum_e max(q_e, 0), q- = sum_e min(q_e, 0)
//   means  s_j = mean_j . sum_e q_e
//
// Products from bf16 MFMAs, 16 query rows by 16 candidates, sums in fp32. Which candidates these choose is
// settled in select_choose.hip.
#include <algorithm>

#include "select.h"

namespace hisparse {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kRowPad = 256;          // a row of scores is a multiple of this
// Workgroups that tiles of candidates are made small for, and the least tile (log2).
constexpr int kWantedGroups = 512, kLeastTile = 8;
constexpr int64_t kMostGroups = (1 << 23) - 1;
constexpr size_t kMostScoreBytes = (size_t)1 << 30;

// ---- scores ----------------------------------------------------------------------------------

template <int KIND>
struct Shape : IndexShape<KIND> {
  using IndexShape<KIND>::KEYS;
  using IndexShape<KIND>::DIMS;
  static constexpr int STEPS = DIMS / 32;          // MFMAs of 16 rows x 16 candidates
  static constexpr int PIECES = DIMS / 8;          // 16-byte pieces of an index row
};

// Sum of the squares of eight bf16 values, and acc.
__device__ __forceinline__ float squares(u32x4_t x, float acc) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t b = x[i];
    const bf16x2_t y = __builtin_bit_cast(bf16x2_t, b);
    acc = __builtin_amdgcn_fdot2_f32_bf16(y, y, acc, false);
  }
  return acc;
}
// x, or 0 if that is more, without a rounding or a look for signalling NaN: by its sign.
__device__ __forceinline__ float positive(float x) {
  return __int_as_float(max(__float_as_int(x), 0));
}
// Over the 16 lanes of a row, in all of them.
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __int_as_float(lane_moved<CTRL>(__float_as_int(x)));
}
__device__ __forceinline__ float sum16(float x) {
  x += moved<0x128>(x);
  x += moved<0x124>(x);
  x += moved<0x122>(x);
  return x + moved<0x121>(x);
}
__device__ __forceinline__ float least16(float x) {
  x = fminf(x, moved<0x128>(x));
  x = fminf(x, moved<0x124>(x));
  x = fminf(x, moved<0x122>(x));
  return fminf(x, moved<0x121>(x));
}
struct Largest {
  __device__ __forceinline__ uint32_t operator()(uint32_t x, uint32_t y) const { return max(x, y); }
};
struct Either {
  __device__ __forceinline__ uint32_t operator()(uint32_t x, uint32_t y) const { return x | y; }
};
// x's halves added in the lower half of the wave, y's in the upper.
__device__ __forceinline__ float halves(float x, float y) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The totals over the four rows of 16 lanes of v0 .. v3: that of v_r in row r.
__device__ __forceinline__ float totals(float v0, float v1, float v2, float v3) {
  const float x = halves(v0, v2), y = halves(v1, v3);
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Bounds and means: the sums over the heads of a token, exact in 64 bits, as three bf16 parts (24 bits:
// off by 2^-25 of the value). Row 4 i + part of the A operand, i the token; the fourth is zero.
template <int KIND, int T>
__device__ __forceinline__ void linear_rows(const SelectArgs& a, int token0, int tokens, int rows, int h,
                                            uint16_t* s_a) {
  constexpr int DIMS = Shape<KIND>::DIMS, PITCH = DIMS + 8;
  for (int x = threadIdx.x; x < rows * 16; x += T) {
    const int i = x >> 4, c = x & 15;
    double pos[8], neg[8];
    query_sums<KIND, 16>(a, token0 + i, h, c, i < tokens ? 0 : a.q_heads, 1, pos, neg);
    auto put = [&](int at, double (&v)[8]) {
#pragma unroll
      for (int part = 0; part < 4; ++part) {
        u32x4_t y = {};
        if (part < 3)
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const bf16x2_t b =
                __builtin_convertvector(f32x2_t{(float)v[2 * d], (float)v[2 * d + 1]}, bf16x2_t);
            const uint32_t bits = __builtin_bit_cast(uint32_t, b);
            v[2 * d] -= low_half(bits);
            v[2 * d + 1] -= high_half(bits);
            y[d] = bits;
          }
        *reinterpret_cast<u32x4_t*>(s_a + (4 * i + part) * PITCH + at) = y;
      }
    };
    if (KIND == HISPARSE_INDEX_BOUNDS) put(8 * c, neg);
    put(KIND == HISPARSE_INDEX_BOUNDS ? kIndexDims + 8 * c : 8 * c, pos);
  }
}

// A tile of candidates, first .. end - 1, that a workgroup scores for new tokens of one request and kv head.
template <int KIND>
struct Tile {
  static constexpr bool KEYS = Shape<KIND>::KEYS;
  const SelectArgs& a;
  const int32_t* table;
  const uint8_t* index;
  int kt, first, end;

  __device__ __forceinline__ Tile(const SelectArgs& args, int q, int h, int tile, int seen)
      : a(args),
        table(args.table ? args.table + q * args.table_request_stride + h * args.table_head_stride : nullptr),
        index(args.index + q * args.request_stride + h * args.head_stride),
        kt(tile),
        first(tile << args.tile_size),
        end(min(first + (1 << args.tile_size), seen)) {}
  // The table's entry for candidate j, as it is; j past the last (of [.., stop)) has the last one's.
  __device__ __forceinline__ int entry_of(int j, int stop) const {
    j = min(j, stop - 1);
    const int e = KEYS ? j >> a.tpr_shift : j;
    return table ? table[e] : e;
  }
  // Padding is loaded as record 0 is, and left out of everything.
  __device__ __forceinline__ bool there(int entry, int j, int stop) const {
    return j < stop && entry >= 0 && entry < a.num_records;
  }
  __device__ __forceinline__ const uint8_t* row_of(int entry, bool valid, int j) const {
    return index + (uint64_t)(uint32_t)(valid ? entry : 0) * (uint32_t)a.record_stride +
           (KEYS ? (j & ((1 << a.tpr_shift) - 1)) * kIndexRowBytes : 0);
  }
  // Whether 64 candidates from a multiple of 64 on lie in one record, one behind the other.
  __device__ __forceinline__ bool one_record() const { return KEYS && a.tpr_shift >= 6; }
};

// The largest sum of squares of index rows (NaN stays: its bits are above infinity's), and all their bits.
struct Norm {
  float largest = 0.f;
  uint32_t bits = 0;
  __device__ __forceinline__ void add(float squares, uint32_t row_bits, bool valid) {
    const uint32_t sq = valid ? __float_as_uint(squares) : 0;
    largest = __uint_as_float(max(__float_as_uint(largest), sq));
    bits |= valid ? row_bits & 0x7fff7fffu : 0;
    // now, and not where they are used: the rows' registers are loaded again
    asm volatile("" : "+v"(bits), "+v"(largest));
  }
};
__device__ __forceinline__ uint32_t any_bits(u32x4_t x) { return x[0] | x[1] | x[2] | x[3]; }

// Writes down score s of candidate j, and takes it into the least and the largest.
__device__ __forceinline__ void put_score(float s, bool valid, float* row, int j, float& least, float& most) {
  if (s != s) s = __uint_as_float(kNan);
  if (valid) {
    least = fminf(least, s);  // (NaN is passed over)
    most = fmaxf(most, s);
  }
  row[j] = valid ? s : __uint_as_float(kPad);
}

// The tile's facts, of the `tokens` new tokens from token0 on. least, most: of the workgroup's token threadIdx.x.
// The largest norm is 0 only if all rows are zero; squares below the float range are made up for.
template <int WAVES>
__device__ __forceinline__ void put_facts(const SelectArgs& a, int token0, int tokens, int h, int kt,
                                          const uint32_t* norms, const uint32_t* bits, float least,
                                          float most) {
  if (threadIdx.x < (unsigned)tokens) {
    uint32_t n = 0, any = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      n = max(n, norms[i]);
      any |= bits[i];
    }
    a.facts[((int64_t)(token0 + (int)threadIdx.x - a.row0) * a.heads + h) * a.tiles + kt] =
        TileFacts{any ? sqrtf(__uint_as_float(n)) * 1.01f + 0x1p-58f : 0.f, least, most};
  }
  if (a.hist && kt == 0)  // added to by the next kernel
    for (int i = 0; i < tokens; ++i)
      for (int x = threadIdx.x; x < kLongBins; x += 64 * WAVES)
        a.hist[((int64_t)(token0 + i - a.row0) * a.heads + h) * kLongBins + x] = 0;
}

// ---- one new token at a time -------------------------------------------------------------------

// A operands of 16 rows: keys, MT tiles of 16 queries of a new token and their weights; the others, of the
// sums of four new tokens (linear_rows).
template <int KIND, int MT>
struct Rows16 {
  using S = Shape<KIND>;
  static constexpr bool KEYS = S::KEYS;
  bf16x8_t A[MT][S::STEPS];
  float w[KEYS ? MT * 4 : 1];

  __device__ __forceinline__ void load(const SelectArgs& a, int token, int h) {  // keys
    const int lane = threadIdx.x & 63, col = lane & 15, group = lane >> 4;
    const uint16_t* q = a.q + (int64_t)token * a.q_stride + (int64_t)h * a.q_heads * kIndexDims + group * 8;
    const float* wr = a.weights ? a.weights + ((int64_t)token * a.heads + h) * a.q_heads : nullptr;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int e = m * 16 + col;
#pragma unroll
      for (int k = 0; k < S::STEPS; ++k) {
        u32x4_t x = {};
        if (e < a.q_heads) x = *reinterpret_cast<const any_u32x4_t*>(q + e * kIndexDims + k * 32);
        A[m][k] = __builtin_bit_cast(bf16x8_t, x);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int y = m * 16 + group * 4 + i;
        w[m * 4 + i] = y < a.q_heads ? (wr ? wr[y] : 1.f) : 0.f;
      }
    }
  }
  __device__ __forceinline__ void load(const uint16_t* s_a, int tile) {  // the others
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < S::STEPS; ++k)
      A[0][k] = *reinterpret_cast<const bf16x8_t*>(s_a + (tile * 16 + (lane & 15)) * (S::DIMS + 8) +
                                                   k * 32 + (lane >> 4) * 8);
  }
  // Scores of 16 candidates, x their rows: keys, this lane's four heads' share of a tile's; the others, of
  // new token group and candidate col, whole.
  __device__ __forceinline__ float score(const u32x4_t (&x)[S::STEPS]) const {
    f32x4_t acc[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) acc[m] = f32x4_t{};
#pragma unroll
    for (int k = 0; k < S::STEPS; ++k)
#pragma unroll
      for (int m = 0; m < MT; ++m)
        acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A[m][k], __builtin_bit_cast(bf16x8_t, x[k]),
                                                         acc[m], 0, 0, 0);
    float v = 0.f;
    if constexpr (KEYS) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) v += w[m * 4 + i] * positive(acc[m][i]);
    } else {
      v = acc[0][0] + acc[0][1] + acc[0][2];
    }
    asm volatile("" : "+v"(v));  // here, and not where it is used: the accumulators are free
    return v;
  }
};

// New token i of request q (of those with fewer than kTeamChunk), a tile of candidates: each wave has a
// quarter of it and loads rows as operands, 32 ahead. HBM-bound from a few requests on: 32 requests of up to
// 32768 tokens, 64 heads, 200 MB of keys in 40 us.
// s_a: 16 rows of an operand, not used for keys.
template <int KIND, int MT>
__device__ __forceinline__ void score_token(const SelectArgs& a, uint32_t block, uint16_t* s_a) {
  using S = Shape<KIND>;
  constexpr bool KEYS = S::KEYS;
  constexpr int WAVES = 4, T = 64 * WAVES;
  __shared__ uint32_t s_norm[WAVES], s_bits[WAVES];
  __shared__ float s_least[WAVES], s_most[WAVES];
  const int lane = threadIdx.x & 63, col = lane & 15, group = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // request and token first: workgroups of one request are far apart
  const uint32_t per = (uint32_t)a.tokens_of_request;
  const uint32_t n_rows = (uint32_t)a.requests * per;
  const uint32_t rest = block / n_rows, row = block - rest * n_rows;
  const int q = (int)(row / per), i = (int)(row - (uint32_t)q * per);
  const int kt = (int)(rest / (uint32_t)a.heads), h = (int)(rest - (uint32_t)kt * a.heads);
  const RequestRows r = rows_of(a, q);
  const int token = r.begin + i;
  if (i >= r.n || r.n >= kTeamChunk<KIND> || token < a.row0 || token >= a.row0 + a.rows) return;
  const int seen = seen_at(a, r.len - r.n + i);
  const Tile<KIND> tile(a, q, h, kt, seen);
  if (seen <= a.top_k || tile.first >= seen) return;
  Rows16<KIND, MT> rows;
  if constexpr (KEYS) {
    rows.load(a, token, h);
  } else {
    linear_rows<KIND, T>(a, token, 1, 4, h, s_a);
    __syncthreads();
    rows.load(s_a, 0);
  }
  float* out = a.scores + ((int64_t)(token - a.row0) * a.heads + h) * a.row_pad;
  float least = INFINITY, most = -INFINITY;
  Norm norm;
  const int share = (1 << a.tile_size) / WAVES;
  const int from = tile.first + wave * share, to = min(from + share, tile.end);
  if (from < to) {
    const bool one_record = tile.one_record();
    auto fetch = [&](u32x4_t (&y)[S::STEPS], int entries, int base, int sub) {
      const uint8_t* x;
      if (one_record) {
        const int e = __builtin_amdgcn_readfirstlane(entries);
        x = tile.row_of(e, tile.there(e, base, to), base + sub * 16) + col * kIndexRowBytes;
      } else {
        const int j = base + sub * 16 + col, e = __shfl(entries, sub * 16 + col);
        x = tile.row_of(e, tile.there(e, j, to), min(j, to - 1));
      }
#pragma unroll
      for (int k = 0; k < S::STEPS; ++k)
        y[k] = *reinterpret_cast<const u32x4_t*>(x + k * 64 + group * 16);
    };
    u32x4_t x[2][S::STEPS];  // two times 16 candidates, the next ones on their way
    int entry = tile.entry_of(from + lane, to);      // of candidate base + lane
    int next = tile.entry_of(from + 64 + lane, to);  // and of the next step's
    fetch(x[0], entry, from, 0);
    fetch(x[1], entry, from, 1);
#pragma unroll 1
    for (int base = from; base < to; base += 64) {
      const uint64_t mask = __ballot(tile.there(entry, base + lane, to));
      const int after = tile.entry_of(base + 128 + lane, to);
      float v[4];
#pragma unroll
      for (int sub = 0; sub < 4; ++sub) {
        float sq = 0.f;
        uint32_t bits = 0;
#pragma unroll
        for (int k = 0; k < S::STEPS; ++k) {
          bits |= any_bits(x[sub & 1][k]);
          sq = squares(x[sub & 1][k], sq);
        }
        sq += __shfl_xor(sq, 16);
        sq += __shfl_xor(sq, 32);
        norm.add(sq, bits, mask >> (sub * 16 + col) & 1);
        v[sub] = rows.score(x[sub & 1]);
        __builtin_amdgcn_sched_barrier(0);
        // (past the end: the last candidate again)
        if (sub < 2) fetch(x[sub & 1], entry, base, sub + 2);
        else fetch(x[sub & 1], next, base + 64, sub - 2);
      }
      // keys: a lane has candidate base + lane; the others: the first 16 lanes have the new token's
      if constexpr (KEYS) {
        const float s = totals(v[0], v[1], v[2], v[3]);
        if (base + lane < to) put_score(s, mask >> lane & 1, out, base + lane, least, most);
      } else {
#pragma unroll
        for (int sub = 0; sub < 4; ++sub) {
          const int at = sub * 16 + col;
          if (group == 0 && base + at < to)
            put_score(v[sub], mask >> at & 1, out, base + at, least, most);
        }
      }
      entry = next;
      next = after;
    }
  }
  const uint32_t nb = wave_reduce(__float_as_uint(norm.largest), 0u, Largest());
  const uint32_t bits = wave_reduce(norm.bits, 0u, Either());
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    least = fminf(least, __shfl_xor(least, d));
    most = fmaxf(most, __shfl_xor(most, d));
  }
  if (lane == 0) {
    s_norm[wave] = nb;
    s_bits[wave] = bits;
    s_least[wave] = least;
    s_most[wave] = most;
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < WAVES; ++x) {
    least = fminf(least, s_least[x]);
    most = fmaxf(most, s_most[x]);
  }
  put_facts<WAVES>(a, token, 1, h, kt, s_norm, s_bits, least, most);
}

template <int KIND, int MT, int OCCUPANCY>
__global__ __launch_bounds__(256, OCCUPANCY) void score_token_kernel(SelectArgs a) {
  __shared__ __align__(16) uint16_t s_a[Shape<KIND>::KEYS ? 8 : 16 * (Shape<KIND>::DIMS + 8)];
  score_token<KIND, MT>(a, blockIdx.x, s_a);
}

// ---- chunks of new tokens ----------------------------------------------------------------------

// The workgroup's candidates, 64 at a time, on their way from memory to one of two buffers in LDS by way of
// registers. Thread t has piece t % PIECES of rows t / PIECES + i * (T / PIECES); piece p of row r lies in
// slot p ^ (r & 15), so that 16 rows' pieces p are in 16 slots of the banks.
template <int KIND, int T>
struct Stage {
  static constexpr int P = Shape<KIND>::PIECES, LOADS = 64 * P / T, BYTES = 64 * P * 16;
  const Tile<KIND>& tile;
  u32x4_t x[LOADS];
  uint64_t mask, ready;  // which of the 64 are not padding: of those in registers, stored last
  int entry;             // of candidate base + lane of the next 64
  Norm norm;
  bool with_norm;

  __device__ __forceinline__ Stage(const Tile<KIND>& t, bool norms) : tile(t), with_norm(norms) {
    entry = tile.entry_of(tile.first + (threadIdx.x & 63), tile.end);
  }
  __device__ __forceinline__ void fetch(int base) {
    const int lane = threadIdx.x & 63, piece = threadIdx.x % P;
    mask = __ballot(tile.there(entry, base + lane, tile.end));
    if (tile.one_record()) {
      const uint8_t* from = tile.row_of(__builtin_amdgcn_readfirstlane(entry), mask & 1, base);
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        x[i] = *reinterpret_cast<const u32x4_t*>(from + (threadIdx.x + i * T) * 16);
    } else {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int row = threadIdx.x / P + i * (T / P), e = __shfl(entry, row);
        x[i] = *reinterpret_cast<const u32x4_t*>(tile.row_of(e, mask >> row & 1, base + row) + piece * 16);
      }
    }
    entry = tile.entry_of(base + 64 + lane, tile.end);
  }
  __device__ __forceinline__ void store(uint8_t* buf) {
    const int piece = threadIdx.x % P;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int row = threadIdx.x / P + i * (T / P);
      *reinterpret_cast<u32x4_t*>(buf + row * (P * 16) + ((piece ^ (row & 15)) << 4)) = x[i];
    }
    if (with_norm)
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        float sq = sum16(squares(x[i], 0.f));
        if (P == 32) sq += __shfl_xor(sq, 16);
        norm.add(sq, any_bits(x[i]), mask >> (threadIdx.x / P + i * (T / P)) & 1);
      }
    ready = mask;
  }
  // The first 64 candidates to buf, the next ones to registers.
  __device__ __forceinline__ void start(uint8_t* buf) {
    fetch(tile.first);
    store(buf);
    if (tile.first + 64 < tile.end) fetch(tile.first + 64);
  }
  // While the 64 from base on are scored: the next ones to buf, those behind them to registers. between()
  // writes down scores: after what was loaded is here, before the next loads, so that no wait for a load is
  // one for a store as well.
  template <class F>
  __device__ __forceinline__ void move(int base, uint8_t* buf, F&& between) {
    if (base + 64 < tile.end) store(buf);
    asm volatile("" : "+v"(entry));
    between();
    if (base + 128 < tile.end) fetch(base + 128);
  }
};

// Keys: the queries of TOKENS new tokens as 32-row A operands, HEADS rows each (16, 32, 64 or 128).
template <int HEADS>
struct Rows32 {
  static constexpr int TILES = HEADS == 128 ? 4 : 2, TOKENS = 32 * TILES / HEADS, STEPS = kIndexDims / 16;
  bf16x8_t A[TILES][STEPS];
  float w[TILES][16];

  // The row of a tile that accumulator i of this lane has.
  static __device__ __forceinline__ int row_of(int i) {
    return 8 * (i >> 2) + 4 * ((threadIdx.x & 63) >> 5) + (i & 3);
  }
  __device__ __forceinline__ void load(const SelectArgs& a, int token0, int live, int h) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const int row = t * 32 + (lane & 31), n = row / HEADS, e = row % HEADS;
      const bool there = n < live && e < a.q_heads;
      const uint16_t* q = a.q + (int64_t)(token0 + n) * a.q_stride +
                          ((int64_t)h * a.q_heads + e) * kIndexDims + (lane >> 5) * 8;
#pragma unroll
      for (int k = 0; k < STEPS; ++k) {
        u32x4_t x = {};
        if (there) x = *reinterpret_cast<const any_u32x4_t*>(q + k * 16);
        A[t][k] = __builtin_bit_cast(bf16x8_t, x);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int y = t * 32 + row_of(i), m = y / HEADS, f = y % HEADS;
        float x = 0.f;
        if (m < live && f < a.q_heads)
          x = a.weights ? a.weights[((int64_t)(token0 + m) * a.heads + h) * a.q_heads + f] : 1.f;
        w[t][i] = x;
      }
    }
  }
  // Tile t's products with 32 candidates.
  __device__ __forceinline__ f32x16_t multiply(int t, const u32x4_t (&x)[STEPS]) const {
    f32x16_t acc = {};
#pragma unroll
    for (int k = 0; k < STEPS; ++k)
      acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(A[t][k], __builtin_bit_cast(bf16x8_t, x[k]), acc, 0,
                                                    0, 0);
    return acc;
  }
  // What they add to this lane's share (half of the heads) of its new tokens' scores.
  __device__ __forceinline__ void add_up(int t, const f32x16_t& acc, float (&v)[TOKENS]) const {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      v[(t * 32 + 8 * (i >> 2)) / HEADS] += w[t][i] * positive(acc[i]);
#pragma unroll
    for (int n = 0; n < TOKENS; ++n) asm volatile("" : "+v"(v[n]));
  }
};

// WAVES times Rows32::TOKENS new tokens (of one or more requests that have kTeamChunk or more, one after the
// other), a tile of candidates: each wave has new tokens of its own, all have the same candidates, 64 at a
// time in LDS. The products of 32 candidates with one tile of queries run beside the sums of those before.
// Norms of the rows, a tenth of the time where every workgroup works them out, are the request's, not a new
// token's: the workgroup that has its last new token of this step, which sees most, has them for all.
// 512 new tokens of 64 heads over 32768 keys: 253 to 284 us by the card, 0.97 to 1.09 PFLOP/s of products, three
// quarters to four fifths of the rate of a large matrix product; the rest is the weighted sum, 32 vector
// instructions to 16 MFMAs, which run beside each other only in part. (Measured: half of the waves moving candidates after their products instead of
// before, 2 % slower in all; a wave priority for them, no gain.)
template <int HEADS, int WAVES, int OCCUPANCY>
__global__ __launch_bounds__(64 * WAVES, OCCUPANCY) void score_keys_kernel(SelectArgs a) {
  constexpr int KIND = HISPARSE_INDEX_KEYS, T = 64 * WAVES;
  using R = Rows32<HEADS>;
  using St = Stage<KIND, T>;
  constexpr int ROWS = WAVES * R::TOKENS;
  __shared__ __align__(16) uint8_t s_mem[2 * St::BYTES];
  __shared__ uint32_t s_norm[WAVES], s_bits[WAVES];
  __shared__ float s_least[ROWS], s_most[ROWS];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t rest = blockIdx.x / (uint32_t)a.tiles;
  const int kt = (int)(blockIdx.x - rest * (uint32_t)a.tiles);
  const int row_tile = (int)(rest / (uint32_t)a.heads), h = (int)(rest - (uint32_t)row_tile * a.heads);
  const int row0 = a.row0 + row_tile * ROWS, row1 = min(row0 + ROWS, a.row0 + a.rows);
#pragma unroll 1
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
    const Tile<KIND> tile(a, q, h, kt, seen);
    if (r.n < kTeamChunk<KIND> || seen <= a.top_k || tile.first >= seen) continue;
    const int mine = wave * R::TOKENS;                     // this wave's first new token
    const int live = min(tokens - mine, (int)R::TOKENS);  // and how many it has (0 or less: none)
    R rows;
    rows.load(a, token0 + mine, live, h);
    const int64_t pitch = a.heads * a.row_pad;
    float* out = a.scores + ((int64_t)(token0 + mine - a.row0) * a.heads + h) * a.row_pad;
    float least[R::TOKENS], most[R::TOKENS];
#pragma unroll
    for (int n = 0; n < R::TOKENS; ++n) {
      least[n] = INFINITY;
      most[n] = -INFINITY;
    }
    // scores of the 64 candidates from `scored` on, not yet written down
    float scores[R::TOKENS] = {};
    int scored = tile.end;
    uint64_t scored_mask = 0;
    auto write_down = [&] {
#pragma unroll
      for (int n = 0; n < R::TOKENS; ++n)
        if (n < live && scored + lane < tile.end)
          put_score(scores[n], scored_mask >> lane & 1, out + n * pitch, scored + lane, least[n], most[n]);
    };
    St stage(tile, token0 + tokens == min(r.begin + r.n, a.row0 + a.rows));
    stage.start(s_mem);
    __syncthreads();
    int cur = 0;
#pragma unroll 1
    for (int base = tile.first; base < tile.end; base += 64) {
      const uint64_t mask = stage.ready;
      stage.move(base, s_mem + (cur ^ 1) * St::BYTES, write_down);
      if (live > 0) {
        float v[2][R::TOKENS] = {};
        u32x4_t y[2][R::STEPS];
        f32x16_t acc[2];
        auto read = [&](int g) {
          const int row = g * 32 + (lane & 31);
          const uint8_t* at = s_mem + cur * St::BYTES + row * kIndexRowBytes;
#pragma unroll
          for (int k = 0; k < R::STEPS; ++k)
            y[g][k] = *reinterpret_cast<const u32x4_t*>(at + (((k * 2 + (lane >> 5)) ^ (row & 15)) << 4));
        };
        read(0);
#pragma unroll
        for (int u = 0; u < 2 * R::TILES; ++u) {
          if (u == R::TILES - 1) read(1);
          acc[u & 1] = rows.multiply(u % R::TILES, y[u / R::TILES]);
          if (u > 0) rows.add_up((u - 1) % R::TILES, acc[(u - 1) & 1], v[(u - 1) / R::TILES]);
#pragma unroll
          for (int i = 0; i < R::STEPS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // an MFMA
            __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);  // four vector instructions
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        rows.add_up(R::TILES - 1, acc[1], v[1]);
#pragma unroll
        for (int n = 0; n < R::TOKENS; ++n) scores[n] = halves(v[0][n], v[1][n]);
      }
      scored = base;
      scored_mask = mask;
      cur ^= 1;
      __syncthreads();
    }
    write_down();
    const uint32_t nb = wave_reduce(__float_as_uint(stage.norm.largest), 0u, Largest());
    const uint32_t bits = wave_reduce(stage.norm.bits, 0u, Either());
    if (lane == 0) {
      s_norm[wave] = nb;
      s_bits[wave] = bits;
    }
#pragma unroll
    for (int n = 0; n < R::TOKENS; ++n) {
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        least[n] = fminf(least[n], __shfl_xor(least[n], d));
        most[n] = fmaxf(most[n], __shfl_xor(most[n], d));
      }
      if (lane == 0) {
        s_least[mine + n] = least[n];
        s_most[mine + n] = most[n];
      }
    }
    __syncthreads();
    put_facts<WAVES>(a, token0, tokens, h, kt, s_norm, s_bits, s_least[threadIdx.x % ROWS],
                     s_most[threadIdx.x % ROWS]);
    __syncthreads();
  }
}

// The same for bounds and means, four new tokens a wave. 1024 new tokens of 4 x 16 heads over 512 means: 17 us,
// of which 6 go into the sums over the heads (each of the two tiles of candidates reads all 17 MB of queries)
// and 4 into the scores: one round of workgroups, each a chain of loads. The last token_blocks workgroups are those of single
// tokens. (A launch of their own took 2.5 us where none were due.)
template <int KIND>
__global__ __launch_bounds__(256, 2) void score_rows_kernel(SelectArgs a, uint32_t token_blocks) {
  using S = Shape<KIND>;
  constexpr int WAVES = 4, T = 64 * WAVES, TOKENS = 4, ROWS = WAVES * TOKENS;
  using St = Stage<KIND, T>;
  constexpr int A_BYTES = 16 * WAVES * (S::DIMS + 8) * 2;
  __shared__ __align__(16) uint8_t s_mem[std::max(2 * St::BYTES, A_BYTES)];
  if (blockIdx.x >= gridDim.x - token_blocks)
    return score_token<KIND, 1>(a, blockIdx.x - (gridDim.x - token_blocks), reinterpret_cast<uint16_t*>(s_mem));
  __shared__ uint32_t s_norm[WAVES], s_bits[WAVES];
  __shared__ float s_least[ROWS], s_most[ROWS];
  const int lane = threadIdx.x & 63, col = lane & 15, group = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t rest = blockIdx.x / (uint32_t)a.tiles;
  const int kt = (int)(blockIdx.x - rest * (uint32_t)a.tiles);
  const int row_tile = (int)(rest / (uint32_t)a.heads), h = (int)(rest - (uint32_t)row_tile * a.heads);
  const int row0 = a.row0 + row_tile * ROWS, row1 = min(row0 + ROWS, a.row0 + a.rows);
#pragma unroll 1
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
    const Tile<KIND> tile(a, q, h, kt, seen);
    if (r.n < kTeamChunk<KIND> || seen <= a.top_k || tile.first >= seen) continue;
    Rows16<KIND, 1> rows;
    linear_rows<KIND, T>(a, token0, tokens, ROWS, h, reinterpret_cast<uint16_t*>(s_mem));
    __syncthreads();
    rows.load(reinterpret_cast<const uint16_t*>(s_mem), wave);
    __syncthreads();
    const int mine = wave * TOKENS + group;  // this lane's new token
    float* out = a.scores + ((int64_t)(token0 + mine - a.row0) * a.heads + h) * a.row_pad;
    float least = INFINITY, most = -INFINITY;
    // scores of the 64 candidates from `scored` on, not yet written down
    float scores[4] = {};
    int scored = tile.end;
    uint64_t scored_mask = 0;
    auto write_down = [&] {
#pragma unroll
      for (int sub = 0; sub < 4; ++sub) {
        const int at = sub * 16 + col;
        if (mine < tokens && scored + at < tile.end)
          put_score(scores[sub], scored_mask >> at & 1, out, scored + at, least, most);
      }
    };
    St stage(tile, token0 + tokens == min(r.begin + r.n, a.row0 + a.rows));
    stage.start(s_mem);
    __syncthreads();
    int cur = 0;
#pragma unroll 1
    for (int base = tile.first; base < tile.end; base += 64) {
      const uint64_t mask = stage.ready;
      stage.move(base, s_mem + (cur ^ 1) * St::BYTES, write_down);
#pragma unroll
      for (int sub = 0; sub < 4; ++sub) {
        u32x4_t y[S::STEPS];
        const uint8_t* row = s_mem + cur * St::BYTES + (sub * 16 + col) * (S::PIECES * 16);
#pragma unroll
        for (int k = 0; k < S::STEPS; ++k)
          y[k] = *reinterpret_cast<const u32x4_t*>(row + (((k * 4 + group) ^ col) << 4));
        scores[sub] = rows.score(y);
      }
      scored = base;
      scored_mask = mask;
      cur ^= 1;
      __syncthreads();
    }
    write_down();
    const uint32_t nb = wave_reduce(__float_as_uint(stage.norm.largest), 0u, Largest());
    const uint32_t bits = wave_reduce(stage.norm.bits, 0u, Either());
    least = least16(least);
    most = -least16(-most);
    if (lane == 0) {
      s_norm[wave] = nb;
      s_bits[wave] = bits;
    }
    if (col == 0) {
      s_least[mine] = least;
      s_most[mine] = most;
    }
    __syncthreads();
    put_facts<WAVES>(a, token0, tokens, h, kt, s_norm, s_bits, s_least[threadIdx.x % ROWS],
                     s_most[threadIdx.x % ROWS]);
    __syncthreads();
  }
}

// ---- host ------------------------------------------------------------------------------------

// New tokens of a workgroup that has a chunk's.
int team_rows(int kind, int q_heads) {
  if (kind != HISPARSE_INDEX_KEYS) return 16;
  return q_heads <= 16 ? 32 : q_heads <= 32 ? 16 : q_heads <= 64 ? 8 : 4;
}

struct SelectPlan {
  int64_t candidates, row_pad, tiles, parts;
  bool is_long;
  int64_t row_bytes;  // of a new token, all kv heads
  int64_t token_rows;  // workgroups of single tokens, for each tile
  int32_t tile_size;
  bool team;          // chunks of kTeamChunk or more new tokens can occur
  int32_t alone;      // the most new tokens of a request that are scored one by one
};

int64_t whole(int64_t n, int64_t of) { return (n + of - 1) / of; }

SelectPlan plan_select(const hisparse_index_desc_t& x, const hisparse_batch_desc_t& b,
                       const hisparse_select_desc_t& d) {
  SelectPlan p{};
  const bool keys = x.kind == HISPARSE_INDEX_KEYS;
  p.candidates = keys ? (int64_t)b.max_records * b.tokens_per_record : b.max_records;
  // The largest tiles of which there are enough: a workgroup first loads its queries. (64 heads, all of a call:
  // 128 new tokens over 32768 keys, 101 us with 512 workgroups, 114 with 1024, 98 with 256; a new token of 32
  // requests over 8192, 39, 45 and 38; means of 512 blocks for 1024 new tokens, 34.3 with 512, 36.1 with 256.)
  const int team = keys ? kTeamChunk<HISPARSE_INDEX_KEYS> : kTeamChunk<HISPARSE_INDEX_MEANS>;
  p.team = b.max_chunk >= team;
  p.alone = std::min(b.max_chunk, team - 1);
  const int64_t row_tiles =
      (p.team ? whole(b.total_tokens, team_rows(x.kind, d.q_heads))
              : std::min<int64_t>(b.total_tokens, (int64_t)b.num_requests * b.max_chunk)) * b.kv_heads;
  p.tile_size = !keys ? 9 : p.team ? 12 : 11;
  while (p.tile_size > kLeastTile &&
         row_tiles * whole(p.candidates, 1 << p.tile_size) < kWantedGroups)
    --p.tile_size;
  // (a launch's workgroups are counted in 32 bits, with all their threads)
  p.token_rows = (int64_t)b.num_requests * p.alone * b.kv_heads;
  while (p.tile_size < 30 && p.token_rows * whole(p.candidates, 1 << p.tile_size) > kMostGroups)
    ++p.tile_size;
  p.tiles = whole(p.candidates, 1 << p.tile_size);
  p.parts = whole(p.candidates, kPart);
  const bool big = p.candidates > kRegisterRow;
  p.is_long = big && p.parts <= kMaxParts;
  p.row_pad = whole(p.candidates, big ? kPart : kRowPad) * (big ? kPart : kRowPad);
  // (those of rows of too many parts too: a workspace serves smaller batches)
  const int64_t words =
      p.row_pad + 3 * whole(p.candidates, 1 << kLeastTile) + (big ? p.row_pad + kLongBins + p.parts + 3 : 0);
  p.row_bytes = words * 4 * b.kv_heads;
  return p;
}

template <int KIND, int MT, int OCCUPANCY>
void launch_tokens(const SelectArgs& a, const SelectPlan& p, hipStream_t s) {
  hipLaunchKernelGGL((score_token_kernel<KIND, MT, OCCUPANCY>), dim3((unsigned)(p.token_rows * p.tiles)),
                     dim3(256), 0, s, a);
}
template <int HEADS, int WAVES, int OCCUPANCY>
void launch_keys(const SelectArgs& a, hipStream_t s) {
  constexpr int ROWS = WAVES * Rows32<HEADS>::TOKENS;
  const unsigned row_tiles = (unsigned)((a.rows + ROWS - 1) / ROWS);
  hipLaunchKernelGGL((score_keys_kernel<HEADS, WAVES, OCCUPANCY>),
                     dim3(row_tiles * (unsigned)a.heads * (unsigned)a.tiles), dim3(64 * WAVES), 0, s, a);
}
template <int KIND>
void launch_rows(const SelectArgs& a, unsigned token_blocks, hipStream_t s) {
  const unsigned row_tiles = (unsigned)((a.rows + 15) / 16);
  hipLaunchKernelGGL(score_rows_kernel<KIND>,
                     dim3(row_tiles * (unsigned)a.heads * (unsigned)a.tiles + token_blocks), dim3(256), 0, s, a,
                     token_blocks);
}

hipError_t launch_select(const SelectArgs& a, int kind, const SelectPlan& p, hipStream_t s) {
  constexpr int K = HISPARSE_INDEX_KEYS, B = HISPARSE_INDEX_BOUNDS, M = HISPARSE_INDEX_MEANS;
  const bool tokens = a.start || !p.team;  // (without starts all chunks are max_chunk)
  if (tokens && (kind == K || !p.team)) {
    if (kind == B) launch_tokens<B, 1, 2>(a, p, s);
    else if (kind == M) launch_tokens<M, 1, 2>(a, p, s);
    else if (a.q_heads <= 16) launch_tokens<K, 1, 3>(a, p, s);
    else if (a.q_heads <= 32) launch_tokens<K, 2, 3>(a, p, s);
    else if (a.q_heads <= 64) launch_tokens<K, 4, 3>(a, p, s);
    else launch_tokens<K, 8, 1>(a, p, s);
  }
  if (p.team) {
    const unsigned token_blocks = tokens ? (unsigned)(p.token_rows * p.tiles) : 0u;
    if (kind == B) launch_rows<B>(a, token_blocks, s);
    else if (kind == M) launch_rows<M>(a, token_blocks, s);
    else if (a.q_heads <= 16) launch_keys<16, 8, 2>(a, s);
    else if (a.q_heads <= 32) launch_keys<32, 8, 2>(a, s);
    else if (a.q_heads <= 64) launch_keys<64, 8, 2>(a, s);
    else launch_keys<128, 4, 1>(a, s);
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
  const hisparse::SelectPlan p = hisparse::plan_select(*x, *b, *d);
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
  const SelectPlan p = plan_select(*x, *b, *d);
  const int64_t rows = b->total_tokens > 1 ? b->total_tokens : 1;
  size_t bytes = (size_t)rows <= kMostScoreBytes / (size_t)p.row_bytes ? (size_t)(rows * p.row_bytes)
                                                                      : kMostScoreBytes;
  if (bytes < (size_t)p.row_bytes) bytes = (size_t)p.row_bytes;
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
  const SelectPlan p = plan_select(*x, *b, *d);
  if (!d_index || !d_q || !d_sel || !d_workspace ||
      workspace_bytes < (size_t)p.row_bytes)
    return HISPARSE_ERR_INVALID_ARG;
  // rows of a step: what the workspace holds, and a launch's 2^32 threads
  int64_t step = (int64_t)(workspace_bytes / (size_t)p.row_bytes);
  const int64_t blocks_of_tile = p.tiles * b->kv_heads;
  const int64_t most = (int64_t)UINT32_MAX / 512 / blocks_of_tile;
  const int64_t most_chosen =
      (int64_t)UINT32_MAX / 1024 / ((p.is_long ? p.parts : 1) * b->kv_heads);
  if (step > most) step = most;
  if (step > most_chosen) step = most_chosen;
  if (step > b->total_tokens) step = b->total_tokens;
  if (step < 1 || p.token_rows * p.tiles > kMostGroups) return HISPARSE_ERR_UNSUPPORTED;
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
  a.tokens_of_request = p.alone;
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
