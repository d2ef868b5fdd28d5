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

constexpr int kRowPad = 256;          // a row of scores is a multiple of this
// New tokens of a request from which waves have new tokens of their own.
constexpr int kTeamChunk = 5;
// Workgroups that tiles of candidates are made small for, and the least tile (log2).
constexpr int kWantedGroups = 512, kLeastTile = 8;
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
// The totals over the four rows of 16 lanes of v0 .. v3: that of v_r in row r.
__device__ __forceinline__ float totals(float v0, float v1, float v2, float v3) {
  auto halves = [](float x, float y) {  // x's halves added in the lower half, y's in the upper
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
  };
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

// What a wave scores: keys, NT new tokens of MT tiles of 16 heads each; the others, 4 MT new tokens, four of
// three rows (and an empty one) to a tile.
template <int KIND, int MT, int NT>
struct Wave {
  using S = Shape<KIND>;
  static constexpr bool KEYS = S::KEYS;
  static constexpr int TILES = KEYS ? MT * NT : MT, TOKENS = KEYS ? NT : 4 * MT;
  // Sums of a lane: keys, of four values at a time (see `totals`) that are four new tokens, or fewer and
  // several 16 candidates; the others, of the new token 4 m + group.
  static constexpr int SETS = KEYS ? (NT + 3) / 4 : MT;
  static constexpr int SPAN = KEYS && NT < 4 ? 64 / NT : 16;  // candidates of a lane's new token at a time
  bf16x8_t A[TILES][S::STEPS];
  float w[KEYS ? TILES * 4 : 1];
  float least[SETS], most[SETS];

  __device__ __forceinline__ void start() {
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
      least[i] = INFINITY;
      most[i] = -INFINITY;
    }
  }
  // keys: the queries of tokens token0 .. of kv head h
  __device__ __forceinline__ void load(const SelectArgs& a, int token0, int tokens, int h) {
    const int lane = threadIdx.x & 63, col = lane & 15, group = lane >> 4;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int64_t token = token0 + n;
      const uint16_t* q = a.q + token * a.q_stride + (int64_t)h * a.q_heads * kIndexDims + group * 8;
      const float* wr = a.weights ? a.weights + (token * a.heads + h) * a.q_heads : nullptr;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int e = m * 16 + col;
#pragma unroll
        for (int k = 0; k < S::STEPS; ++k) {
          u32x4_t x = {};
          if (n < tokens && e < a.q_heads)
            x = *reinterpret_cast<const any_u32x4_t*>(q + e * kIndexDims + k * 32);
          A[n * MT + m][k] = __builtin_bit_cast(bf16x8_t, x);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int y = m * 16 + group * 4 + i;
          w[(n * MT + m) * 4 + i] = n < tokens && y < a.q_heads ? (wr ? wr[y] : 1.f) : 0.f;
        }
      }
    }
  }
  // the others: rows of s_a from token `first` of the workgroup's on
  __device__ __forceinline__ void load(const uint16_t* s_a, int first) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int k = 0; k < S::STEPS; ++k)
        A[m][k] = *reinterpret_cast<const bf16x8_t*>(
            s_a + (first * 4 + m * 16 + (lane & 15)) * (S::DIMS + 8) + k * 32 + (lane >> 4) * 8);
  }

  // Products with 16 candidates' rows.
  __device__ __forceinline__ void multiply(const u32x4_t (&x)[S::STEPS], f32x4_t (&acc)[TILES]) const {
#pragma unroll
    for (int t = 0; t < TILES; ++t) acc[t] = f32x4_t{};
#pragma unroll
    for (int k = 0; k < S::STEPS; ++k)
#pragma unroll
      for (int t = 0; t < TILES; ++t)
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(A[t][k], __builtin_bit_cast(bf16x8_t, x[k]),
                                                         acc[t], 0, 0, 0);
  }
  // Their scores: keys, this lane's share of each new token's; the others, whole.
  __device__ __forceinline__ void add_up(const f32x4_t (&acc)[TILES], float (&v)[KEYS ? NT : MT]) const {
    if constexpr (KEYS) {
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        v[n] = 0.f;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[n] += w[(n * MT + m) * 4 + i] * positive(acc[n * MT + m][i]);
        asm volatile("" : "+v"(v[n]));  // here, and not where it is used: the accumulators are free
      }
    } else {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        v[m] = acc[m][0] + acc[m][1] + acc[m][2];
        asm volatile("" : "+v"(v[m]));
      }
    }
  }

  // A set's scores to memory: this lane's is candidate j's, of its new token's row.
  __device__ __forceinline__ void put(float s, int set, float* row, int j, int end, bool valid, bool live) {
    if (j >= end || !live) return;
    if (s != s) s = __uint_as_float(kNan);
    if (valid) {
      least[set] = fminf(least[set], s);  // (NaN is passed over)
      most[set] = fmaxf(most[set], s);
    }
    row[j] = valid ? s : __uint_as_float(kPad);
  }
  // The workgroup's new token (from the wave's first) that this lane has in a set.
  __device__ __forceinline__ int token_of(int set) const {
    const int row = (threadIdx.x & 63) >> 4;
    if (!KEYS) return 4 * set + row;
    return NT >= 4 ? 4 * set + row : NT == 2 ? row >> 1 : 0;
  }
  // Scores of 64 candidates base .., v[sub] of each 16, written down. out: row of the wave's first token;
  // mask: which are not padding.
  __device__ __forceinline__ void put64(const float (&v)[4][KEYS ? NT : MT], float* out, int64_t pitch,
                                        int tokens, int base, int end, uint64_t mask) {
    const int lane = threadIdx.x & 63, col = lane & 15;
    auto one = [&](float s, int set, int at) {
      const int t = token_of(set);
      put(s, set, out + t * pitch, base + at, end, mask >> at & 1, t < tokens);
    };
    if constexpr (!KEYS) {
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int sub = 0; sub < 4; ++sub) one(v[sub][m], m, sub * 16 + col);
    } else if constexpr (NT == 1) {
      one(totals(v[0][0], v[1][0], v[2][0], v[3][0]), 0, lane);
    } else if constexpr (NT == 2) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
        one(totals(v[2 * x][0], v[2 * x + 1][0], v[2 * x][1], v[2 * x + 1][1]), 0, x * 32 + (lane & 31));
    } else {
#pragma unroll
      for (int set = 0; set < SETS; ++set)
#pragma unroll
        for (int sub = 0; sub < 4; ++sub)
          one(totals(v[sub][4 * set], v[sub][4 * set + 1], v[sub][4 * set + 2], v[sub][4 * set + 3]),
              set, sub * 16 + col);
    }
  }
};

// The table's entry for candidate j of [0, end), as it is; j past the end has the last one's.
template <bool KEYS>
__device__ __forceinline__ int entry_of(const SelectArgs& a, const int32_t* table, int j, int end) {
  j = min(j, end - 1);
  const int e = KEYS ? j >> a.tpr_shift : j;
  return table ? table[e] : e;
}

// ROWS new tokens of a workgroup (of one or more requests, one after the other), a tile of candidates.
//
// TEAM: the waves have new tokens of their own and the same candidates, 64 at a time by way of LDS, the next
// 64 on their way in registers meanwhile. Otherwise, and where there are no more new tokens than one wave
// has, each wave has a quarter of the candidates and loads them as operands.
template <int KIND, int MT, int NT, int WAVES, bool TEAM, int OCCUPANCY>
__global__ __launch_bounds__(64 * WAVES, OCCUPANCY) void score_kernel(SelectArgs a) {
  using S = Shape<KIND>;
  using W = Wave<KIND, MT, NT>;
  constexpr bool KEYS = S::KEYS;
  constexpr int T = 64 * WAVES, ROWS = TEAM ? WAVES * W::TOKENS : 1;
  constexpr int LOADS = 64 * S::PIECES / T;  // of a thread, for 64 rows
  constexpr int A_ROWS = KEYS ? 0 : MT * (TEAM ? WAVES : 1);  // tiles
  constexpr int TILE_BYTES = 64 * S::DIMS * 2, A_BYTES = 16 * A_ROWS * (S::DIMS + 8) * 2;
  __shared__ __align__(16) uint8_t s_mem[std::max(TEAM ? 2 * TILE_BYTES : 16, A_BYTES)];
  __shared__ uint32_t s_norm[WAVES], s_bits[WAVES];
  __shared__ float s_least[WAVES][W::TOKENS], s_most[WAVES][W::TOKENS];
  const int lane = threadIdx.x & 63, col = lane & 15, group = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t block = blockIdx.x, rest = block / (uint32_t)a.tiles;
  const int kt = (int)(block - rest * (uint32_t)a.tiles);
  const int tile = (int)(rest / (uint32_t)a.heads), h = (int)(rest - (uint32_t)tile * a.heads);
  const int row0 = a.row0 + tile * ROWS, row1 = min(row0 + ROWS, a.row0 + a.rows);
#pragma unroll 1
  for (int t = row0; t < row1;) {
    const int q = request_at(a, t);
    const RequestRows r = rows_of(a, q);
    if (t < r.begin || t >= r.begin + r.n) {
      if (ROWS == 1) return;
      ++t;
      continue;
    }
    const int token0 = t, tokens = min(row1, r.begin + r.n) - t;
    t += tokens;
    const int seen = seen_at(a, r.len - r.n + token0 + tokens - 1 - r.begin);
    const int first = kt << a.tile_size, end = min(first + (1 << a.tile_size), seen);
    if (seen <= a.top_k || first >= seen) {
      if (ROWS == 1) return;
      continue;
    }
    const bool team = TEAM && tokens > W::TOKENS;
    const int mine = team ? wave * W::TOKENS : 0;      // this wave's first new token
    const int live = min(tokens - mine, W::TOKENS);    // and how many it has (0 or less: none)
    const int32_t* table =
        a.table ? a.table + q * a.table_request_stride + h * a.table_head_stride : nullptr;
    const uint8_t* index = a.index + q * a.request_stride + h * a.head_stride;
    // Padding is loaded as record 0 is, and left out of everything.
    auto there = [&](int entry, int j, int stop) {
      return j < stop && entry >= 0 && entry < a.num_records;
    };
    auto row_of = [&](int entry, bool valid, int j) {
      return index + (uint64_t)(uint32_t)(valid ? entry : 0) * (uint32_t)a.record_stride +
             (KEYS ? (j & ((1 << a.tpr_shift) - 1)) * kIndexRowBytes : 0);
    };
    // 64 candidates from a multiple of 64 on that lie in one record, one behind the other
    const bool one_record = KEYS && a.tpr_shift >= 6;
    W wv;
    wv.start();
    if constexpr (KEYS) {
      wv.load(a, token0 + mine, live, h);
    } else {
      __syncthreads();  // what the last segment kept here is read
      linear_rows<KIND, T>(a, token0, tokens, 4 * A_ROWS, h, reinterpret_cast<uint16_t*>(s_mem));
      __syncthreads();
      wv.load(reinterpret_cast<const uint16_t*>(s_mem), mine);
      if (TEAM) __syncthreads();
    }
    const int64_t pitch = a.heads * a.row_pad;
    float* out = a.scores + ((int64_t)(token0 + mine - a.row0) * a.heads + h) * a.row_pad;
    float norm = 0.f;  // the largest sum of squares; NaN stays (its bits are above infinity's)
    uint32_t bits = 0;
    auto larger = [&](float sq) {
      norm = __uint_as_float(max(__float_as_uint(norm), __float_as_uint(sq)));
    };
    if (team) {
      // thread t: piece t % PIECES of rows t / PIECES + i * (T / PIECES); piece p of row r lies in slot
      // p ^ (r & 15), so that 16 rows' pieces p are in 16 slots of the banks
      constexpr int P = S::PIECES;
      const int piece = threadIdx.x % P, row_first = threadIdx.x / P;
      int entry = entry_of<KEYS>(a, table, first + lane, end);  // of candidate base + lane, one step ahead
      u32x4_t x[LOADS];
      uint64_t mask;  // which of 64 candidates are not padding
      auto fetch = [&](int base) {
        mask = __ballot(there(entry, base + lane, end));
        if (one_record) {
          const uint8_t* from = row_of(__builtin_amdgcn_readfirstlane(entry), mask & 1, base);
#pragma unroll
          for (int i = 0; i < LOADS; ++i)
            x[i] = *reinterpret_cast<const u32x4_t*>(from + (threadIdx.x + i * T) * 16);
        } else
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int row = row_first + i * (T / P), e = __shfl(entry, row);
          x[i] = *reinterpret_cast<const u32x4_t*>(row_of(e, mask >> row & 1, base + row) + piece * 16);
        }
        entry = entry_of<KEYS>(a, table, base + 64 + lane, end);
      };
      auto store = [&](uint8_t* buf) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int row = row_first + i * (T / P);
          const bool valid = mask >> row & 1;
          *reinterpret_cast<u32x4_t*>(buf + row * (P * 16) + ((piece ^ (row & 15)) << 4)) = x[i];
          // the largest of this piece; over the row's pieces they are added up at the end, which is no less
          // than the largest row
          bits |= valid ? (x[i][0] | x[i][1] | x[i][2] | x[i][3]) & 0x7fff7fffu : 0;
          larger(valid ? squares(x[i], 0.f) : 0.f);
          asm volatile("" : "+v"(bits), "+v"(norm));
        }
      };
      fetch(first);
      store(s_mem);
      __syncthreads();
      int cur = 0;
#pragma unroll 1
      for (int base = first; base < end; base += 64) {
        const uint64_t now = mask;
        if (base + 64 < end) fetch(base + 64);
        if (live > 0) {
          // the products of 16 candidates while those of the 16 before are added up
          float v[4][KEYS ? NT : MT];
          u32x4_t y[2][S::STEPS];
          f32x4_t acc[2][W::TILES];
          auto read = [&](int sub) {
            const uint8_t* row = s_mem + cur * TILE_BYTES + (sub * 16 + col) * (P * 16);
#pragma unroll
            for (int k = 0; k < S::STEPS; ++k)
              y[sub & 1][k] = *reinterpret_cast<const u32x4_t*>(row + (((k * 4 + group) ^ col) << 4));
          };
          read(0);
#pragma unroll
          for (int sub = 0; sub < 4; ++sub) {
            if (sub < 3) read(sub + 1);
            wv.multiply(y[sub & 1], acc[sub & 1]);
            if (sub > 0) wv.add_up(acc[(sub - 1) & 1], v[sub - 1]);
            if (KEYS)
#pragma unroll
              for (int i = 0; i < W::TILES * S::STEPS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // an MFMA
                __builtin_amdgcn_sched_group_barrier(0x002, 2, 0);  // two vector instructions
              }
            __builtin_amdgcn_sched_barrier(0);
          }
          wv.add_up(acc[1], v[3]);
          wv.put64(v, out, pitch, live, base, end, now);
        }
        cur ^= 1;
        if (base + 64 < end) store(s_mem + cur * TILE_BYTES);
        __syncthreads();
      }
    } else {
      const int share = (1 << a.tile_size) / WAVES;
      const int from = first + wave * share, to = min(from + share, end);
      u32x4_t x[2][S::STEPS];  // two times 16 candidates, the next ones on their way
      int entry = 0, next = 0;  // of candidate base + lane, and of the next step's
      auto fetch = [&](u32x4_t (&y)[S::STEPS], int entries, int base, int sub) {
        const uint8_t* row;
        if (one_record) {
          const int e = __builtin_amdgcn_readfirstlane(entries);
          row = row_of(e, there(e, base, to), base + sub * 16) + col * kIndexRowBytes + group * 16;
        } else {
          const int j = base + sub * 16 + col, e = __shfl(entries, sub * 16 + col);
          row = row_of(e, there(e, j, to), min(j, to - 1)) + group * 16;
        }
#pragma unroll
        for (int k = 0; k < S::STEPS; ++k) y[k] = *reinterpret_cast<const u32x4_t*>(row + k * 64);
      };
      if (from < to) {
        entry = entry_of<KEYS>(a, table, from + lane, to);
        next = entry_of<KEYS>(a, table, from + 64 + lane, to);
        fetch(x[0], entry, from, 0);
        fetch(x[1], entry, from, 1);
#pragma unroll 1
        for (int base = from; base < to; base += 64) {
          const uint64_t mask = __ballot(there(entry, base + lane, to));
          const int after = entry_of<KEYS>(a, table, base + 128 + lane, to);
          float v[4][KEYS ? NT : MT];
#pragma unroll
          for (int sub = 0; sub < 4; ++sub) {
            float sq = 0.f;
            uint32_t any = 0;
#pragma unroll
            for (int k = 0; k < S::STEPS; ++k) {
              const u32x4_t y = x[sub & 1][k];
              any |= (y[0] | y[1] | y[2] | y[3]) & 0x7fff7fffu;
              sq = squares(y, sq);
            }
            sq += __shfl_xor(sq, 16);
            sq += __shfl_xor(sq, 32);
            const bool valid = mask >> (sub * 16 + col) & 1;
            larger(valid ? sq : 0.f);
            bits |= valid ? any : 0;
            asm volatile("" : "+v"(bits), "+v"(norm));  // now: the operands' registers are loaded again
            f32x4_t acc[W::TILES];
            wv.multiply(x[sub & 1], acc);
            wv.add_up(acc, v[sub]);
            __builtin_amdgcn_sched_barrier(0);
            // (past the end: the last candidate again)
            if (sub < 2) fetch(x[sub & 1], entry, base, sub + 2);
            else fetch(x[sub & 1], next, base + 64, sub - 2);
          }
          wv.put64(v, out, pitch, live, base, to, mask);
          entry = next;
          next = after;
        }
      }
    }
    // The tile's facts. The largest norm is 0 only if all rows are zero; squares below the float range are
    // made up for.
    if (team) {
      norm = sum16(norm);
      if (S::PIECES == 32) norm += __shfl_xor(norm, 16);
    }
    const uint32_t nb = wave_reduce(__float_as_uint(norm), 0u, Largest());
    bits = wave_reduce(bits, 0u, Either());
    if (lane == 0) {
      s_norm[wave] = nb;
      s_bits[wave] = bits;
    }
#pragma unroll
    for (int set = 0; set < W::SETS; ++set) {  // over the lanes that have the same new token
      float lo = least16(wv.least[set]), hi = -least16(-wv.most[set]);
      if (KEYS && NT <= 2) {
        lo = fminf(lo, __shfl_xor(lo, 16));
        hi = fmaxf(hi, __shfl_xor(hi, 16));
      }
      if (KEYS && NT == 1) {
        lo = fminf(lo, __shfl_xor(lo, 32));
        hi = fmaxf(hi, __shfl_xor(hi, 32));
      }
      if (col == 0) {
        s_least[wave][wv.token_of(set)] = lo;
        s_most[wave][wv.token_of(set)] = hi;
      }
    }
    __syncthreads();
    if (threadIdx.x < (unsigned)tokens) {
      uint32_t n = 0, any = 0;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) {
        n = max(n, s_norm[i]);
        any |= s_bits[i];
      }
      float least = INFINITY, most = -INFINITY;
      if (team) {
        least = s_least[threadIdx.x / W::TOKENS][threadIdx.x % W::TOKENS];
        most = s_most[threadIdx.x / W::TOKENS][threadIdx.x % W::TOKENS];
      } else {
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
          least = fminf(least, s_least[i][threadIdx.x]);
          most = fmaxf(most, s_most[i][threadIdx.x]);
        }
      }
      a.facts[((int64_t)(token0 + (int)threadIdx.x - a.row0) * a.heads + h) * a.tiles + kt] =
          TileFacts{any ? sqrtf(__uint_as_float(n)) * 1.01f + 0x1p-58f : 0.f, least, most};
    }
    if (a.hist && kt == 0)  // added to by the next kernel
      for (int i = 0; i < tokens; ++i)
        for (int x = threadIdx.x; x < kLongBins; x += T)
          a.hist[((int64_t)(token0 + i - a.row0) * a.heads + h) * kLongBins + x] = 0;
    if (ROWS == 1) return;
    __syncthreads();
  }
}

// ---- host ------------------------------------------------------------------------------------

// New tokens of a workgroup of score_kernel.
int team_rows(int kind, int q_heads) {
  if (kind != HISPARSE_INDEX_KEYS) return 16;
  return q_heads <= 16 ? 32 : q_heads <= 32 ? 16 : q_heads <= 64 ? 8 : 4;
}

struct SelectPlan {
  int64_t candidates, row_pad, tiles, parts;
  bool is_long;
  int64_t row_bytes;  // of a new token, all kv heads
  int32_t tile_size;
};

int64_t whole(int64_t n, int64_t of) { return (n + of - 1) / of; }

SelectPlan plan_select(const hisparse_index_desc_t& x, const hisparse_batch_desc_t& b,
                       const hisparse_select_desc_t& d) {
  SelectPlan p{};
  const bool keys = x.kind == HISPARSE_INDEX_KEYS;
  p.candidates = keys ? (int64_t)b.max_records * b.tokens_per_record : b.max_records;
  // The largest tiles of which there are enough: a workgroup first loads its queries. (512 new tokens x 64
  // heads over 32768 keys: scores and choice in 321 us with 512 of them, 331 with 1024.)
  const bool team = b.max_chunk >= kTeamChunk;
  const int64_t row_tiles =
      whole(b.total_tokens, team ? team_rows(x.kind, d.q_heads) : 1) * b.kv_heads;
  p.tile_size = !keys ? 9 : team ? 12 : 11;
  while (p.tile_size > kLeastTile &&
         row_tiles * whole(p.candidates, 1 << p.tile_size) < kWantedGroups)
    --p.tile_size;
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

template <int KIND, int MT, int NT, int WAVES, bool TEAM, int OCCUPANCY>
void launch_score(const SelectArgs& a, hipStream_t s) {
  constexpr int ROWS = TEAM ? WAVES * Wave<KIND, MT, NT>::TOKENS : 1;
  const unsigned row_tiles = (unsigned)((a.rows + ROWS - 1) / ROWS);
  hipLaunchKernelGGL((score_kernel<KIND, MT, NT, WAVES, TEAM, OCCUPANCY>),
                     dim3(row_tiles * (unsigned)a.heads * (unsigned)a.tiles), dim3(64 * WAVES), 0, s, a);
}

hipError_t launch_select(const SelectArgs& a, int kind, const SelectPlan& p, hipStream_t s) {
  constexpr int K = HISPARSE_INDEX_KEYS, B = HISPARSE_INDEX_BOUNDS, M = HISPARSE_INDEX_MEANS;
  const bool team = a.max_chunk >= kTeamChunk;
  if (kind == B) {
    if (team) launch_score<B, 1, 1, 4, true, 2>(a, s);
    else launch_score<B, 1, 1, 4, false, 2>(a, s);
  } else if (kind == M) {
    if (team) launch_score<M, 1, 1, 4, true, 2>(a, s);
    else launch_score<M, 1, 1, 4, false, 2>(a, s);
  } else if (team) {
    if (a.q_heads <= 16) launch_score<K, 1, 4, 8, true, 2>(a, s);
    else if (a.q_heads <= 32) launch_score<K, 2, 2, 8, true, 2>(a, s);
    else if (a.q_heads <= 64) launch_score<K, 4, 1, 8, true, 2>(a, s);
    else launch_score<K, 8, 1, 4, true, 1>(a, s);
  } else {
    if (a.q_heads <= 16) launch_score<K, 1, 1, 4, false, 3>(a, s);
    else if (a.q_heads <= 32) launch_score<K, 2, 1, 4, false, 3>(a, s);
    else if (a.q_heads <= 64) launch_score<K, 4, 1, 4, false, 2>(a, s);
    else launch_score<K, 8, 1, 4, false, 1>(a, s);
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
