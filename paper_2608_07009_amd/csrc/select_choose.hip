// The choice of a selection (hisparse_select_records): which candidates have the largest scores.
//
// The choice is that of scores in 64 bits, which the fp32 scores of select.hip settle but for a few:
// with
//   |s_j - exact| <= eps = 1.25 c A N,  A = sum_e |w_e| |q_e|, N = the largest |k_j| seen
// (keys: sums of 128 products, each step off by at most 2^-23, and of the heads, 2^-24 a step and the
// weight's product: c = 2^-16 + (heads + 1) 2^-24; the others: c = 2^-15, 256 products, their three parts and
// what is left of q+ and q-, 2^-22, being less than the quarter added; and a term for what is lost below the
// normal range. Keys: none where a head's products may leave fp32, whatever its weight)
// and with the m-th largest s in [lo, hi], candidates above hi + 2 eps are among the best m, those below
// lo - 2 eps are not, and those between ("open") are scored again in 64 bits.
//
// [lo, hi] is a bin of a histogram between the least and the largest score. A row of up to 32768 scores
// is held in the registers of one workgroup, loaded once. Longer rows are cut down
// first: narrow_kernel's workgroups add up the row's histogram, keep_kernel's write down the candidates
// that its bin leaves in question or in, a part of the row each, and those few are chosen from. Rows
// that neither way settles (thousands of open candidates, no error bound) go over
// their scores in memory as often as it takes (Stream).
#include "select.h"

namespace hisparse {
namespace {

typedef double f64x4 __attribute__((ext_vector_type(4)));

constexpr int kQPitch = kIndexDims + 8;  // keys: a query's row in LDS (16-byte pieces, banks apart)
constexpr int kCUs = 256;
constexpr int kBatch = 128;              // open candidates scored at a time

// 64-bit scores in the order of the choice: NaN above everything, -0 as 0.
__device__ __forceinline__ uint64_t ordered(double x) {
  if (x != x) return ~0ull;
  const int64_t b = __double_as_longlong(x + 0.0);
  return b < 0 ? ~(uint64_t)b : (uint64_t)b | 0x8000000000000000ull;
}
__device__ __forceinline__ uint32_t ordered32(float x) {
  const uint32_t b = __float_as_uint(x);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered32(uint32_t b) {
  return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ double positive(double x) { return x > 0.0 ? x : x == x ? 0.0 : x; }

// T threads, of a kernel that chooses among up to CAP candidates at once.
template <int KIND, int T, int BINS, int LIST, int CAP>
struct alignas(16) Shared {
  static constexpr bool KEYS = KIND == HISPARSE_INDEX_KEYS;
  union {
    struct {
      union {
        uint32_t hist[BINS];
        double part[KEYS ? 8 * kBatch : 1];  // keys: 16 heads' share of open candidates' scores
      };
      uint64_t score[LIST];
      int list[LIST];        // open candidates, and each one's place among those looked at
      uint16_t where[LIST];
    };
    int out[CAP < kMaxTopK ? CAP : kMaxTopK];  // at the end, the chosen ones
  };
  uint32_t win[CAP < 8192 ? 256 : CAP / 32];  // chosen ones among the open, by place
  unsigned long long least, most;
  double q[KEYS ? 2 : 2 * kIndexDims];   // bounds and means: the sums over the heads
  uint32_t wave_a[T / 64], wave_b[T / 64], wave_c[T / 64];
  double wave_d[T / 64], wave_e[T / 64], wave_f[T / 64];
  int count, bin, above, in_bin;
};

struct Add {
  static constexpr uint32_t none = 0;
  __device__ __forceinline__ uint32_t operator()(uint32_t x, uint32_t y) const { return x + y; }
};
struct Most {
  static constexpr uint32_t none = 0;
  __device__ __forceinline__ uint32_t operator()(uint32_t x, uint32_t y) const { return max(x, y); }
};
struct Least {
  static constexpr uint32_t none = ~0u;
  __device__ __forceinline__ uint32_t operator()(uint32_t x, uint32_t y) const { return min(x, y); }
};
template <int T, class F>
__device__ __forceinline__ uint32_t group_reduce(uint32_t x, uint32_t* waves, F f) {
  x = wave_reduce(x, F::none, f);
  if constexpr (T == 64) return x;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = x;
  __syncthreads();
  x = waves[0];
#pragma unroll
  for (int i = 1; i < T / 64; ++i) x = f(x, waves[i]);
  return x;
}

// The bin in which the need-th from the top lies: s.bin, s.above, s.in_bin. Returns the number of all.
template <int T, int BINS, class S>
__device__ __forceinline__ int find_bin(S& s, const uint32_t* hist, int need) {
  constexpr int PER = BINS / T;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  uint32_t c[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) sum += c[i] = hist[BINS - 1 - (t * PER + i)];
  const int inc = wave_inclusive((int)sum);
  if (lane == 63) s.wave_a[wave] = (uint32_t)inc;
  __syncthreads();
  int before = inc - (int)sum, total = 0;
#pragma unroll
  for (int i = 0; i < T / 64; ++i) {
    before += i < wave ? (int)s.wave_a[i] : 0;
    total += (int)s.wave_a[i];
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (before < need && before + (int)c[i] >= need) {
      s.bin = BINS - 1 - (t * PER + i);
      s.above = before;
      s.in_bin = (int)c[i];
    }
    before += (int)c[i];
  }
  __syncthreads();
  return total;
}

// Bins between two scores, and the scores that bin b can hold: bin_of is off by three roundings of x - from,
// its ends by as many.
template <int BINS>
struct Division {
  float from, to, scale, width;
  __device__ __forceinline__ Division(float a, float b)
      : from(a), to(b), scale((float)BINS / (b - a)), width((b - a) * (1.f / BINS)) {}
  // The scale stays inside the float range.
  static __device__ __forceinline__ bool divides(float a, float b) {
    return b - a > 0x1p-100f && b - a < INFINITY;
  }
  __device__ __forceinline__ int of(float x) const { return min((int)((x - from) * scale), BINS - 1); }
  __device__ __forceinline__ float slack() const { return (fabsf(from) + fabsf(to)) * 0x1p-21f; }
  __device__ __forceinline__ float bottom(int b) const { return from + (float)b * width - slack(); }
  __device__ __forceinline__ float top(int b) const { return from + (float)(b + 1) * width + slack(); }
};

// One row of scores: a new token's, of one kv head.
template <int KIND, int T>
struct Row {
  static constexpr bool KEYS = KIND == HISPARSE_INDEX_KEYS;
  static constexpr int DIMS = IndexShape<KIND>::DIMS, WAVES = T / 64;
  const SelectArgs& a;
  uint16_t* s_q;        // keys: the queries, [q_heads] rows of kQPitch
  const float* wrow;    // and their weights, or null
  float* scores;
  const TileFacts *facts, *norms;  // (the tiles' largest norms are in the second)
  int token, q, h, p, seen, first, last0;  // forced: j < first, j >= last0
  int lane, wave;

  // Whether the block's row is one of a chunk.
  __device__ __forceinline__ bool find(int local, int kv_head) {
    token = a.row0 + local;
    h = kv_head;
    q = request_at(a, token);
    const RequestRows r = rows_of(a, q);
    if (token < r.begin || token >= r.begin + r.n) return false;
    p = r.len - r.n + token - r.begin;
    seen = seen_at(a, p);
    first = min(a.first, seen);
    last0 = max(seen - a.last, 0);
    const int64_t slot = (int64_t)local * a.heads + h;
    scores = a.scores + slot * a.row_pad;
    facts = a.facts + slot * a.tiles;
    const int last = min(r.begin + r.n, a.row0 + a.rows) - 1;
    norms = r.n < kTeamChunk<KIND> ? facts : a.facts + ((int64_t)(last - a.row0) * a.heads + h) * a.tiles;
    wrow = KEYS && a.weights ? a.weights + ((int64_t)token * a.heads + h) * a.q_heads : nullptr;
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    return true;
  }
  __device__ __forceinline__ bool forced(int j) const { return j < first || j >= last0; }
  __device__ __forceinline__ int own() const { return a.last > 0 ? seen - 1 : -1; }
  __device__ __forceinline__ int chosen() const { return min(seen, a.top_k); }

  // Places that forced candidates take; the newest one's is kept even if it is padding.
  template <class S>
  __device__ __forceinline__ int places(S& s) const {
    uint32_t n = 0;
    for (int i = threadIdx.x; i < a.first + a.last; i += T) {
      const int j = i < a.first ? i : seen - 1 - (i - a.first);
      n += __float_as_uint(scores[j]) != kPad || j == seen - 1;
    }
    return (int)group_reduce<T>(n, s.wave_a, Add());
  }

  // eps (0: every score is 0), the range of the scores, and the queries in LDS; or the range alone.
  template <class S>
  __device__ __forceinline__ float error_bound(S& s, float& from, float& to, bool range_only = false) const {
    double A = 0.0, W = 0.0, Q = 0.0;
    if (range_only) {
    } else if constexpr (KEYS) {  // 16 lanes a query
      const uint16_t* qrow = a.q + (int64_t)token * a.q_stride + (int64_t)h * a.q_heads * kIndexDims;
      const int c = threadIdx.x & 15;
      for (int e = threadIdx.x >> 4; e < a.q_heads; e += T / 16) {
        const u32x4_t x = *reinterpret_cast<const any_u32x4_t*>(qrow + e * kIndexDims + 8 * c);
        *reinterpret_cast<u32x4_t*>(s_q + e * kQPitch + 8 * c) = x;
        double sq = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const double lo = low_half(x[i]), hi = high_half(x[i]);
          sq = fma(lo, lo, fma(hi, hi, sq));
        }
        sq = sum16_64(sq);
        if (c == 0) {
          const double n = sqrt(sq), w = wrow ? fabs((double)wrow[e]) : 1.0;
          A += w * n;
          W += w;
          Q += n;
        }
      }
    } else {
      if (wave == 0) {  // 16 lanes a query
        double pos[8], neg[8];
        query_sums<KIND, 2>(a, token, h, lane & 15, lane >> 4, 4, pos, neg);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
          for (int d = 16; d < 64; d *= 2) {
            pos[i] += __shfl_xor(pos[i], d);
            if (KIND == HISPARSE_INDEX_BOUNDS) neg[i] += __shfl_xor(neg[i], d);
          }
          const int d = 8 * (lane & 15) + i;
          if (lane < 16) {
            if (KIND == HISPARSE_INDEX_BOUNDS) s.q[d] = neg[i];
            s.q[KIND == HISPARSE_INDEX_BOUNDS ? kIndexDims + d : d] = pos[i];
            A += fabs(pos[i]) + fabs(neg[i]);  // (0 only if all are)
            Q = fma(pos[i], pos[i], fma(neg[i], neg[i], Q));
          }
        }
      }
    }
    A = wave_sum64(A);
    W = wave_sum64(W);
    Q = wave_sum64(Q);
    uint32_t norm = 0, least = ~0u, most = 0;
    const int tiles = (seen + (1 << a.tile_size) - 1) >> a.tile_size;
    for (int i = threadIdx.x; i < tiles; i += T) {
      const TileFacts f = facts[i];
      norm = max(norm, __float_as_uint(norms[i].norm));
      least = min(least, ordered32(f.least));
      most = max(most, ordered32(f.most));
    }
    norm = wave_reduce(norm, Most::none, Most());
    least = wave_reduce(least, Least::none, Least());
    most = wave_reduce(most, Most::none, Most());
    __syncthreads();
    if (lane == 63) {
      s.wave_d[wave] = A;
      s.wave_e[wave] = W;
      s.wave_f[wave] = Q;
      s.wave_a[wave] = norm;
      s.wave_b[wave] = least;
      s.wave_c[wave] = most;
    }
    __syncthreads();
    A = W = Q = 0.0;
    for (int i = 0; i < WAVES; ++i) {
      A += s.wave_d[i];
      W += s.wave_e[i];
      Q += s.wave_f[i];
      norm = max(norm, s.wave_a[i]);
      least = min(least, s.wave_b[i]);
      most = max(most, s.wave_c[i]);
    }
    if (!KEYS) {  // one query, the sums, of weight 1; A == 0 tells that it is 0
      A = A == 0.0 ? 0.0 : sqrt(Q) + 0x1p-500;
      Q = A;
      W = 1.0;
    }
    from = unordered32(least);
    to = unordered32(most);
    const float N = __uint_as_float(norm);
    if (A == 0.0 && N < INFINITY) return 0.f;
    if (N == 0.f && A < INFINITY) return 0.f;
    // A head whose products may leave fp32 leaves no bound, however small its weight is (their sums are NaN,
    // or infinities that the weight does not bring back).
    if (KEYS && !((float)Q * 1.01f * N < INFINITY)) return INFINITY;
    // the last term: what inputs and sums below the normal range are off by, before the weights and after
    // (never 0: that every score is 0 has been told above)
    const float AN = (float)A * 1.01f * N;
    const float c = KEYS ? 0x1.4p-16f + (float)(a.q_heads + 1) * 0x1.4p-24f : 0x1.4p-15f;
    return AN * c + ((float)W * (N + (float)Q + 1.f) + 1.f) * 0x1p-118f;
  }

  // Writes candidate j (-1: none) to a place of the list.
  __device__ __forceinline__ void put(int place, int j) const {
    const uint8_t* x;
    int record = -1;
    const bool there = j >= 0 && find_row<KEYS>(a, q, h, j, x, record);
    const int64_t at = ((int64_t)token * a.heads + h) * a.top_k + place;
    a.sel[at] = there ? j : -1;
    if (a.records) a.records[at] = there ? record : -1;
  }
  // What follows the `total` chosen ones other than the newest, and the newest one's place.
  __device__ __forceinline__ void finish(int total) const {
    const int mine = own(), n = chosen();
    for (int i = total + (int)threadIdx.x; i < a.top_k; i += T)
      if (mine < 0 || i != n - 1) put(i, -1);
    if (threadIdx.x == 0) {
      if (mine >= 0) put(n - 1, mine);
      if (a.sel_len && h == 0) {
        const int t = 1 << a.cand_shift;
        a.sel_len[token] = n > 0 ? (n - 1) * t + (p & (t - 1)) + 1 : 0;
      }
    }
  }
};

// Scores of the open candidates s.list[0 .. n) in 64 bits, to s.score.
//
// Keys: fp64 MFMAs, 16 heads by 16 candidates: a wave has a tile of heads and 16 candidates; a lane holds
// dims 32 g .. 32 g + 31 of its head and of its candidate, g its quarter of the wave, which are the k index
// of 32 MFMAs. (With a candidate a wave and a head a lane, 50 candidates of 64 heads took 16 us.) The
// others: 16 lanes a candidate.
template <int KIND, int T, class S>
__device__ __forceinline__ void score_open(const Row<KIND, T>& r, S& s, int n) {
  if constexpr (KIND == HISPARSE_INDEX_KEYS) {
    const int col = r.lane & 15, g = r.lane >> 4, tiles = (r.a.q_heads + 15) >> 4;
    for (int from = 0; from < n; from += kBatch) {
      const int count = min(kBatch, n - from), tasks = ((count + 15) >> 4) * tiles;
      for (int task = r.wave; task < tasks; task += T / 64) {
        const int batch = task / tiles, tile = task - batch * tiles;
        const int i = batch * 16 + col, e = tile * 16 + col;
        const uint8_t* key = nullptr;
        int record;
        u32x4_t kx[4] = {}, qx[4] = {};
        if (i < count && find_row<true>(r.a, r.q, r.h, s.list[from + i], key, record)) {
#pragma unroll
          for (int x = 0; x < 4; ++x) kx[x] = reinterpret_cast<const u32x4_t*>(key + 64 * g)[x];
        }
        if (e < r.a.q_heads) {
#pragma unroll
          for (int x = 0; x < 4; ++x)
            qx[x] = reinterpret_cast<const u32x4_t*>(r.s_q + e * kQPitch + 32 * g)[x];
        }
        float w[4];  // a lane has heads g, g + 4, g + 8, g + 12 of the tile
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int head = tile * 16 + g + 4 * x;
          w[x] = r.wrow && head < r.a.q_heads ? r.wrow[head] : 1.f;
        }
        f64x4 acc = {};
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)low_half(qx[x][y]),
                                                       (double)low_half(kx[x][y]), acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f64_16x16x4f64((double)high_half(qx[x][y]),
                                                       (double)high_half(kx[x][y]), acc, 0, 0, 0);
          }
        double sum = 0.0;
#pragma unroll
        for (int x = 0; x < 4; ++x)
          if (tile * 16 + g + 4 * x < r.a.q_heads) sum = fma((double)w[x], positive(acc[x]), sum);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (g == 0) s.part[tile * kBatch + i] = sum;
      }
      __syncthreads();
      for (int i = threadIdx.x; i < count; i += T) {
        double sum = s.part[i];
        for (int x = 1; x < tiles; ++x) sum += s.part[x * kBatch + i];
        s.score[from + i] = ordered(sum);
      }
      __syncthreads();
    }
  } else {
    constexpr int PER = IndexShape<KIND>::DIMS / 16;
    const int c = r.lane & 15;
    for (int i = threadIdx.x >> 4; i < n; i += T / 16) {
      const uint8_t* key = nullptr;
      int record;
      find_row<false>(r.a, r.q, r.h, s.list[i], key, record);
      double sum = 0.0;
#pragma unroll
      for (int x = 0; x < PER / 8; ++x) {
        const u32x4_t y = reinterpret_cast<const u32x4_t*>(key + c * PER * 2)[x];
        const double* q = s.q + c * PER + 8 * x;
#pragma unroll
        for (int z = 0; z < 4; ++z)
          sum = fma((double)high_half(y[z]), q[2 * z + 1], fma((double)low_half(y[z]), q[2 * z], sum));
      }
      sum = sum16_64(sum);
      if (c == 0) s.score[i] = ordered(sum);
    }
    __syncthreads();
  }
}

// The choice from scores in memory, whatever they are: a few passes where 64 bits settle few candidates,
// and where they have to settle many, the scores worked out anew in each of up to nine passes.
template <int KIND, int T, int BINS, int LIST, class S>
struct Stream {
  static constexpr bool KEYS = KIND == HISPARSE_INDEX_KEYS;
  static constexpr int WAVES = T / 64;
  const Row<KIND, T>& r;
  S& s;
  int lo, hi;           // this wave's candidates
  bool all, zero;       // every candidate is open; every score is 0
  float sure, maybe;    // above sure: chosen; below maybe: not

  __device__ Stream(const Row<KIND, T>& row, S& shared) : r(row), s(shared) {
    const int span = (((r.seen + WAVES - 1) / WAVES) + 255) & ~255;
    lo = (int)min((int64_t)r.wave * span, (int64_t)r.seen);
    hi = (int)min((int64_t)(r.wave + 1) * span, (int64_t)r.seen);
    all = zero = false;
    sure = maybe = INFINITY;
  }
  __device__ __forceinline__ bool rankable(int j, float x) const {
    return __float_as_uint(x) != kPad && !r.forced(j);
  }
  __device__ __forceinline__ bool is_sure(float x) const { return !all && x > sure; }
  __device__ __forceinline__ bool is_open(float x) const { return all || (x >= maybe && !(x > sure)); }

  // f(j, score) for this wave's candidates, four in a row per lane.
  template <class F>
  __device__ __forceinline__ void each(F&& f) const {
    for (int base = lo + r.lane * 4; base < hi; base += 256) {
      const f32x4_t x = *reinterpret_cast<const f32x4_t*>(r.scores + base);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (base + i < hi) f(base + i, x[i]);
    }
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
      float from = unordered32(group_reduce<T>(least, s.wave_a, Least()));
      float to = unordered32(group_reduce<T>(most, s.wave_b, Most()));
      const int rankables = (int)group_reduce<T>(count, s.wave_a, Add());
      all = rankables <= m;  // nothing to choose
      int need = m;
      for (int round = 0; round < 4 && from < to && !all; ++round) {
        const float scale = (float)BINS / (to - from);
        auto bin_of = [&](float x) { return min((int)((x - from) * scale), BINS - 1); };
        for (int i = threadIdx.x; i < BINS; i += T) s.hist[i] = 0;
        __syncthreads();
        each([&](int j, float x) {
          if (rankable(j, x) && x >= from && x <= to) atomicAdd(&s.hist[bin_of(x)], 1u);
        });
        __syncthreads();
        find_bin<T, BINS>(s, s.hist, need);
        const int bin = s.bin, in_bin = s.in_bin;
        need -= s.above;
        least = ~0u;
        most = 0;
        each([&](int j, float x) {
          if (!rankable(j, x) || !(x >= from && x <= to) || bin_of(x) != bin) return;
          least = min(least, ordered32(x));
          most = max(most, ordered32(x));
        });
        from = unordered32(group_reduce<T>(least, s.wave_a, Least()));
        to = unordered32(group_reduce<T>(most, s.wave_b, Most()));
        if (in_bin <= LIST / 4) break;
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
        if (at < LIST) s.list[at] = j;
      }
    });
    const int need = m - (int)group_reduce<T>(n_sure, s.wave_a, Add());
    const int open = s.count;
    __syncthreads();
    if (need >= open) {  // (all of them: fewer rankable candidates than asked for)
      each([&](int j, float x) {
        if (rankable(j, x) && is_open(x)) r.scores[j] = __uint_as_float(kWin);
      });
    } else if (open <= LIST && !zero) {
      score_open<KIND, T>(r, s, open);
      for (int i = threadIdx.x; i < open; i += T) {
        const uint64_t x = s.score[i];
        const int j = s.list[i];
        int better = 0;
        for (int y = 0; y < open; ++y)
          better += s.score[y] > x || (s.score[y] == x && s.list[y] < j);
        if (better < need) r.scores[j] = __uint_as_float(kWin);
      }
    } else {
      choose_many(need);
    }
    __syncthreads();  // the marks are read by other waves
  }

  // f(n) for LIST candidates after the other, the n open ones among them in ascending order in s.list, and
  // unless every score is 0, their scores in s.score.
  template <class F>
  __device__ __forceinline__ void lists(F&& f) {
    constexpr int PER = LIST / T;
#pragma unroll 1
    for (int base = 0; base < r.seen; base += LIST) {
      const int j0 = base + (int)threadIdx.x * PER;
      uint32_t open = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (j0 + i < r.seen) {
          const float x = r.scores[j0 + i];
          open |= (uint32_t)(rankable(j0 + i, x) && is_open(x)) << i;
        }
      const int c = __popc(open), inc = wave_inclusive(c);
      __syncthreads();  // what the last list left has been read
      if (r.lane == 63) s.wave_a[r.wave] = (uint32_t)inc;
      __syncthreads();
      int at = inc - c, n = 0;
      for (int i = 0; i < WAVES; ++i) {
        at += i < r.wave ? (int)s.wave_a[i] : 0;
        n += (int)s.wave_a[i];
      }
#pragma unroll
      for (int i = 0; i < PER; ++i)
        if (open >> i & 1) s.list[at++] = j0 + i;
      __syncthreads();
      if (n == 0) continue;
      if (!zero) score_open<KIND, T>(r, s, n);
      f(n);
    }
    __syncthreads();
  }

  // More open candidates than the list holds (thousands of equal scores, or no error bound): the need-th
  // largest in 64 bits is found 8 bits at a time, the scores worked out anew each time, until those that
  // share its first bits are all equal or all wanted. (32768 equal keys of 64 heads: 6.5 ms; a candidate a wave
  // at a time took 115.)
  __device__ void choose_many(int need) {
    uint64_t prefix = 0;
    int shift = 0;
    if (!zero) {
      for (shift = 56;; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += T) s.win[i] = 0;
        if (threadIdx.x == 0) {
          s.least = ~0ull;
          s.most = 0;
        }
        uint64_t least = ~0ull, most = 0;
        lists([&](int n) {
          for (int i = threadIdx.x; i < n; i += T) {
            const uint64_t x = s.score[i];
            if (shift < 56 && x >> (shift + 8) != prefix) continue;
            atomicAdd(&s.win[(int)(x >> shift) & 255], 1u);
            least = min(least, x);
            most = max(most, x);
          }
        });
        atomicMin(&s.least, (unsigned long long)least);
        atomicMax(&s.most, (unsigned long long)most);
        __syncthreads();
        if (s.least == s.most) {
          prefix = s.least;
          shift = 0;
          break;
        }
        if (r.wave == 0) {  // four bins a lane, from the top
          uint32_t c[4], sum = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) sum += c[i] = s.win[255 - (r.lane * 4 + i)];
          int before = wave_inclusive((int)sum) - (int)sum;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (before < need && before + (int)c[i] >= need) {
              s.bin = 255 - (r.lane * 4 + i);
              s.above = before;
              s.in_bin = (int)c[i];
            }
            before += (int)c[i];
          }
        }
        __syncthreads();
        prefix = prefix << 8 | (uint64_t)s.bin;
        need -= s.above;
        const bool done = shift == 0 || s.in_bin == need;
        __syncthreads();
        if (done) break;
      }
    }
    // above the prefix: chosen; with it: the first ones
    int before = 0;
    lists([&](int n) {
      for (int i0 = 0; i0 < n; i0 += T) {
        const int i = i0 + (int)threadIdx.x;
        const uint64_t x = i < n && !zero ? s.score[i] >> shift : prefix;
        const uint64_t equal = __ballot(i < n && x == prefix);
        if (r.lane == 0) s.wave_b[r.wave] = (uint32_t)__popcll(equal);
        __syncthreads();
        int mine = before + (int)__popcll(equal & ((1ull << r.lane) - 1));
        for (int w = 0; w < WAVES; ++w) {
          mine += w < r.wave ? (int)s.wave_b[w] : 0;
          before += (int)s.wave_b[w];
        }
        __syncthreads();
        if (i < n && (x > prefix || (x == prefix && mine < need)))
          r.scores[s.list[i]] = __uint_as_float(kWin);
      }
    });
  }

  // The marked and the sure ones in ascending order (scored false: all that are not padding).
  __device__ __forceinline__ void write(bool scored) const {
    const int own = r.own();
    auto is_in = [&](int j) {
      if (j >= hi || j == own) return false;
      if (!scored) {
        const uint8_t* at;
        int record;
        return find_row<KEYS>(r.a, r.q, r.h, j, at, record);
      }
      const float x = r.scores[j];
      const uint32_t b = __float_as_uint(x);
      return b != kPad && (b == kWin || r.forced(j) || is_sure(x));
    };
    int mine = 0;
    for (int base = lo; base < hi; base += 64) mine += __popcll(__ballot(is_in(base + r.lane)));
    __syncthreads();
    if (r.lane == 0) s.wave_a[r.wave] = (uint32_t)mine;
    __syncthreads();
    int at = 0, total = 0;
    for (int i = 0; i < WAVES; ++i) {
      if (i < r.wave) at += (int)s.wave_a[i];
      total += (int)s.wave_a[i];
    }
    for (int base = lo; base < hi; base += 64) {
      const bool in = is_in(base + r.lane);
      const uint64_t mask = __ballot(in);
      const int place = at + (int)__popcll(mask & ((1ull << r.lane) - 1));
      if (in && place < r.a.top_k) r.put(place, base + r.lane);
      at += __popcll(mask);
    }
    r.finish(total);
  }
};

// eps, and the range of scores, that a long row's kernels agree on.
struct LongRow {
  float eps, from, to;
  __device__ __forceinline__ bool divisible() const {
    return eps > 0.f && eps < INFINITY && Division<kLongBins>::divides(from, to);
  }
};

// T threads hold the row's scores, 4 V each, or a long row's survivors. What bounds it is a chain of steps, each of
// them a trip to memory or a barrier or two: 30 us for a row of 32768, 16 for one of 8192, alone or with as many
// others as there are CUs. (512 threads: registers for two workgroups on a CU, so that one's steps run beside
// the other's: 512 rows of 32768 in 63 us, not 78.)
template <int KIND, int T, int V, int BINS, int LIST, bool LONG>
__global__ __launch_bounds__(T, T == 512 ? 4 : 1) void choose_kernel(SelectArgs a) {
  constexpr bool KEYS = KIND == HISPARSE_INDEX_KEYS;
  constexpr int WAVES = T / 64, CAP = T * V * 4;
  using S = Shared<KIND, T, BINS, LIST, CAP>;
  using Bits = std::conditional_t<V * 4 <= 32, uint32_t, uint64_t>;  // one for each of a thread's candidates
  static_assert(V * 4 <= 64 && CAP <= 65536, "bits; 16-bit places");
  static_assert(sizeof(S) + (KEYS ? 128 * kQPitch * 2 : 0) <= 65536, "LDS of a launch");
  extern __shared__ __align__(16) uint8_t s_mem[];
  S& s = *reinterpret_cast<S*>(s_mem);
  Row<KIND, T> r{a, reinterpret_cast<uint16_t*>(s_mem + sizeof(S))};
  const int local = (int)(blockIdx.x / (uint32_t)a.heads);
  if (!r.find(local, (int)(blockIdx.x - (uint32_t)local * a.heads))) return;
  using Slow = Stream<KIND, T, BINS, LIST, S>;
  if (r.seen <= a.top_k) {
    Slow(r, s).write(false);
    return;
  }
  LongRow row;
  row.eps = r.error_bound(s, row.from, row.to);
  auto slow = [&] {
    Slow c(r, s);
    const int places = r.places(s);
    if (a.top_k > places) c.choose(a.top_k - places, row.eps);
    c.write(true);
  };
  if (!(row.eps > 0.f && row.eps < INFINITY && row.to - row.from < INFINITY)) return slow();
  int n = r.seen;  // candidates that are looked at
  const int64_t slot = (int64_t)local * a.heads + r.h;
  const bool listed = LONG && r.seen > kRegisterRow;
  if (listed) {
    if (!a.hist || !row.divisible()) return slow();
    const int parts = (r.seen + kPart - 1) / kPart;  // at most kMaxParts, T
    // (held to what can be: where starts do not ascend, a row may not have been scored)
    const int mine = (int)threadIdx.x < parts
                         ? min(max(a.part_count[slot * a.parts + threadIdx.x], 0), kPart) : 0;
    const int inc = wave_inclusive(mine);
    if (r.lane == 63) s.wave_a[r.wave] = (uint32_t)inc;
    __syncthreads();
    int before = inc - mine;
    n = 0;
    for (int i = 0; i < WAVES; ++i) {
      before += i < r.wave ? (int)s.wave_a[i] : 0;
      n += (int)s.wave_a[i];
    }
    s.win[threadIdx.x] = (uint32_t)before;  // where each part's survivors begin
    __syncthreads();
  }
  if (n > CAP) return slow();

  // The candidates of this thread: v of span / 256 groups of four in a row, ascending over waves, v and lanes.
  // Those that are padding or forced are NaN here: no comparison holds.
  const int span = (((n + WAVES - 1) / WAVES) + 255) & ~255, groups = span >> 8;
  f32x4_t x[V];
  int pos[LONG ? V * 4 : 1];
  Bits in = 0;  // the chosen ones: bit 4 v + i
  const int own = r.own();
  const int e0 = r.wave * span + r.lane * 4;
  if (listed) {
    const int parts = (r.seen + kPart - 1) / kPart;
    const int32_t* survivors = a.survivors + slot * a.row_pad;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      int at[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[v][i] = __uint_as_float(kNan);
        pos[LONG ? 4 * v + i : 0] = -1;
      }
      if (v >= groups || e0 + v * 256 >= n) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // (past the last one: the last one, for four loads at a time)
        const int e = min(e0 + v * 256 + i, n - 1);
        int lo = 0, hi = parts;  // the last part that begins at or before e
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if ((int)s.win[mid] <= e) lo = mid;
          else hi = mid;
        }
        at[i] = lo * kPart + e - (int)s.win[lo];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) at[i] = survivors[at[i]];
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        at[i] = min(max(at[i], 0), r.seen - 1);
        y[i] = r.scores[at[i]];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (e0 + v * 256 + i < n) {
          pos[LONG ? 4 * v + i : 0] = at[i];
          if (r.forced(at[i])) in |= Bits(1) << (4 * v + i);
          else x[v][i] = y[i];
        }
    }
    __syncthreads();
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int base = e0 + v * 256;
      u32x4_t y = {kPad, kPad, kPad, kPad};
      if (v < groups && base < n) y = *reinterpret_cast<const u32x4_t*>(r.scores + base);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = base + i;
        const bool dead = j >= n || y[i] == kPad, kept = !dead && r.forced(j);
        if (kept && j != own) in |= Bits(1) << (4 * v + i);
        x[v][i] = dead || kept ? __uint_as_float(kNan) : __uint_as_float(y[i]);
        if (LONG) pos[LONG ? 4 * v + i : 0] = j;
      }
    }
  }
  for (int i = threadIdx.x; i < CAP / 32; i += T) s.win[i] = 0;
  if (threadIdx.x == 0) s.count = 0;
  auto each = [&](auto&& f) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v < groups)
#pragma unroll
        for (int i = 0; i < 4; ++i) f(4 * v + i, x[v][i]);
  };
  auto position = [&](int bit) {
    return LONG ? pos[LONG ? bit : 0] : e0 + (bit >> 2) * 256 + (bit & 3);
  };
  const int m = a.top_k - (a.last > 0) - (int)group_reduce<T>((uint32_t)__popcll(in), s.wave_b, Add());

  float sure = INFINITY, maybe = INFINITY;
  if (m > 0) {
    float from = row.from, to = row.to;
    bool any = false;  // nothing to choose: all of them
    for (int round = 0; round < 3 && Division<BINS>::divides(from, to); ++round) {
      const Division<BINS> d(from, to);
      for (int i = threadIdx.x; i < BINS; i += T) s.hist[i] = 0;
      __syncthreads();
      uint32_t above = 0;
      each([&](int, float y) {
        if (y >= from && y <= to) atomicAdd(&s.hist[d.of(y)], 1u);
        above += y > to;
      });
      if (round > 0) above = group_reduce<T>(above, s.wave_c, Add());
      else above = 0;
      __syncthreads();
      const int total = find_bin<T, BINS>(s, s.hist, m - (int)above);
      // (later rounds see a bin of the one before, whose last candidate may be the m-th)
      if (round == 0 && total <= m) {
        any = true;
        break;
      }
      from = fmaxf(from, d.bottom(s.bin));
      to = fminf(to, d.top(s.bin));
      const bool few = s.in_bin <= LIST / 4;
      __syncthreads();
      if (few) break;
    }
    // rounded outwards
    sure = any ? -INFINITY : nextafterf(to + 2.f * row.eps, INFINITY);
    maybe = any ? -INFINITY : nextafterf(from - 2.f * row.eps, -INFINITY);
    uint32_t n_sure = 0;
    Bits open_bits = 0;
    each([&](int bit, float y) {
      if (y > sure) {
        in |= Bits(1) << bit;
        ++n_sure;
      } else if (y >= maybe) {
        open_bits |= Bits(1) << bit;
        const int at = atomicAdd(&s.count, 1);
        if (at < LIST) {
          s.list[at] = position(bit);
          s.where[at] = (uint16_t)(e0 + (bit >> 2) * 256 + (bit & 3));
        }
      }
    });
    const int need = m - (int)group_reduce<T>(n_sure, s.wave_b, Add());
    const int open = s.count;
    if (need >= open) {
      in |= open_bits;
    } else if (need > 0) {
      if (open > LIST) {
        __syncthreads();
        return slow();
      }
      score_open<KIND, T>(r, s, open);
      for (int i = r.wave; i < open; i += WAVES) {  // a wave looks at 64 others at a time
        const uint64_t y = s.score[i];
        const int e = s.where[i];
        int better = 0;
        for (int z = r.lane; z - r.lane < open; z += 64) {
          const int at = min(z, open - 1);
          const uint64_t o = s.score[at];
          better += (int)__popcll(__ballot(z < open && (o > y || (o == y && s.where[at] < e))));
        }
        if (better < need && r.lane == 0) atomicOr(&s.win[e >> 5], 1u << (e & 31));
      }
      __syncthreads();
      if (open_bits)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int e = e0 + v * 256;
          if (v < groups) in |= (Bits)((s.win[e >> 5] >> (e & 31)) & 15u) << (4 * v);
        }
    }
  }

  // Written down in ascending order: this wave's, group by group.
  int places[V], mine = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    places[v] = 0;
    if (v < groups) {
      const int c = __popc((uint32_t)(in >> (4 * v)) & 15u), inc = wave_inclusive(c);
      places[v] = mine + inc - c;
      mine += last_lane(inc);
    }
  }
  __syncthreads();
  if (r.lane == 0) s.wave_a[r.wave] = (uint32_t)mine;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    before += i < r.wave ? (int)s.wave_a[i] : 0;
    total += (int)s.wave_a[i];
  }
  // by way of LDS: looked up and stored 64 at a time, and not where each lane finds its own
#pragma unroll
  for (int v = 0; v < V; ++v) {
    int at = before + places[v];
    if (v < groups)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (((uint32_t)(in >> (4 * v + i)) & 1) && at < a.top_k) s.out[at++] = position(4 * v + i);
  }
  __syncthreads();
#pragma unroll 4
  for (int i = threadIdx.x; i < min(total, a.top_k); i += T) r.put(i, s.out[i]);
  r.finish(total);
}

// ---- long rows -------------------------------------------------------------------------------

constexpr int kLongThreads = 1024, kLongGroups = kPart / kLongThreads / 4;

// The row's histogram, a part of it each; the first part's workgroup has the error bound too.
template <int KIND>
__global__ __launch_bounds__(kLongThreads) void narrow_kernel(SelectArgs a) {
  using S = Shared<KIND, kLongThreads, kLongBins, 64, 32>;
  extern __shared__ __align__(16) uint8_t s_mem[];
  S& s = *reinterpret_cast<S*>(s_mem);
  Row<KIND, kLongThreads> r{a, reinterpret_cast<uint16_t*>(s_mem + sizeof(S))};
  const int64_t slot = blockIdx.x / (uint32_t)a.parts;
  const int part = (int)(blockIdx.x - (uint32_t)slot * a.parts);
  const int local = (int)slot / a.heads;
  if (!r.find(local, (int)slot - local * a.heads)) return;
  if (r.seen <= kRegisterRow || part * kPart >= r.seen) return;
  LongRow row;
  row.eps = r.error_bound(s, row.from, row.to, part != 0);
  if (part == 0 && threadIdx.x == 0) reinterpret_cast<LongRow*>(a.bound)[slot] = row;
  if (!Division<kLongBins>::divides(row.from, row.to)) return;
  const Division<kLongBins> d(row.from, row.to);
  for (int i = threadIdx.x; i < kLongBins; i += kLongThreads) s.hist[i] = 0;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < kLongGroups; ++v) {
    const int base = part * kPart + v * kLongThreads * 4 + (int)threadIdx.x * 4;
    if (base >= r.seen) continue;
    const f32x4_t x = *reinterpret_cast<const f32x4_t*>(r.scores + base);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = base + i;
      if (j < r.seen && !r.forced(j) && x[i] >= row.from && x[i] <= row.to)
        atomicAdd(&s.hist[d.of(x[i])], 1u);
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < kLongBins; i += kLongThreads)
    if (s.hist[i]) atomicAdd(a.hist + slot * kLongBins + i, s.hist[i]);
}

// The part's candidates that may be among the top_k best, and the forced ones, in ascending order. (The
// top_k-th best lies at or below the last that is wanted, whatever places forced ones take.)
template <int KIND>
__global__ __launch_bounds__(kLongThreads) void keep_kernel(SelectArgs a) {
  using S = Shared<KIND, kLongThreads, kLongBins, 64, 32>;
  __shared__ S s;
  Row<KIND, kLongThreads> r{a, nullptr};
  const int64_t slot = blockIdx.x / (uint32_t)a.parts;
  const int part = (int)(blockIdx.x - (uint32_t)slot * a.parts);
  const int local = (int)slot / a.heads;
  if (!r.find(local, (int)slot - local * a.heads)) return;
  if (r.seen <= kRegisterRow || part * kPart >= r.seen) return;
  const LongRow row = reinterpret_cast<const LongRow*>(a.bound)[slot];
  if (!row.divisible()) return;
  const Division<kLongBins> d(row.from, row.to);
  const int total = find_bin<kLongThreads, kLongBins>(s, a.hist + slot * kLongBins, a.top_k);
  float maybe = -INFINITY;
  if (total > a.top_k) maybe = nextafterf(d.bottom(s.bin) - 2.f * row.eps, -INFINITY);
  const int own = r.own(), e0 = part * kPart + r.wave * (256 * kLongGroups) + r.lane * 4;
  uint32_t keep = 0;
  int places[kLongGroups], mine = 0;
#pragma unroll
  for (int v = 0; v < kLongGroups; ++v) {
    const int base = e0 + v * 256;
    u32x4_t x = {kPad, kPad, kPad, kPad};
    if (base < r.seen) x = *reinterpret_cast<const u32x4_t*>(r.scores + base);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int j = base + i;
      if (j < r.seen && x[i] != kPad && j != own && (r.forced(j) || __uint_as_float(x[i]) >= maybe))
        keep |= 1u << (4 * v + i);
    }
    const int c = __popc((keep >> (4 * v)) & 15u), inc = wave_inclusive(c);
    places[v] = mine + inc - c;
    mine += last_lane(inc);
  }
  __syncthreads();
  if (r.lane == 0) s.wave_a[r.wave] = (uint32_t)mine;
  __syncthreads();
  int before = 0, sum = 0;
  for (int i = 0; i < kLongThreads / 64; ++i) {
    before += i < r.wave ? (int)s.wave_a[i] : 0;
    sum += (int)s.wave_a[i];
  }
  if (threadIdx.x == 0) a.part_count[slot * a.parts + part] = sum;
  int32_t* out = a.survivors + slot * a.row_pad + (int64_t)part * kPart;
#pragma unroll
  for (int v = 0; v < kLongGroups; ++v) {
    int at = before + places[v];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (keep >> (4 * v + i) & 1) out[at++] = e0 + v * 256 + i;
  }
}

template <int KIND, int T, int V, int BINS, int LIST, bool LONG>
void launch(const SelectArgs& a, hipStream_t s) {
  constexpr bool KEYS = KIND == HISPARSE_INDEX_KEYS;
  const size_t queries = KEYS ? (size_t)a.q_heads * kQPitch * 2 : 0;
  const unsigned rows = (unsigned)(a.rows * a.heads);
  if (LONG && a.hist) {
    const dim3 grid(rows * (unsigned)a.parts);
    hipLaunchKernelGGL(narrow_kernel<KIND>, grid, dim3(kLongThreads),
                       sizeof(Shared<KIND, kLongThreads, kLongBins, 64, 32>) + queries, s, a);
    hipLaunchKernelGGL(keep_kernel<KIND>, grid, dim3(kLongThreads), 0, s, a);
  }
  hipLaunchKernelGGL((choose_kernel<KIND, T, V, BINS, LIST, LONG>), dim3(rows), dim3(T),
                     sizeof(Shared<KIND, T, BINS, LIST, T * V * 4>) + queries, s, a);
}

// The workgroups that hold a row, 16 to 64 scores a thread. Few threads have less to agree on, many get through
// their own sooner, and where rows are more than compute units, small workgroups share them. Keys of 64 heads
// and bounds, all of a call:
//   1 row of 8192     512 threads, not 1024: 23.4 us, not 26.2      21.1, not 22.9
//   600 rows of 8192  256, not 512:          130, not 138           63, not 71
//   600 rows of 16000 512, not 1024:         225, not 234           94, not 101
//   600 rows of 4096  256, not 1024:         85, not 105            41, not 58
//   4000 rows of 512  64, not 256:           (keys: always 256)     27, not 40 (means; 300 rows: 19.5, 18.4)
template <int KIND>
void launch_kind(const SelectArgs& a, int64_t candidates, hipStream_t s) {
  constexpr bool KEYS = KIND == HISPARSE_INDEX_KEYS;
  const int64_t rows = (int64_t)a.rows * a.heads;
  if constexpr (!KEYS) {
    if (candidates <= 1024 && rows > 8 * kCUs) return launch<KIND, 64, 4, 256, 256, false>(a, s);
  }
  if (candidates <= 4096) launch<KIND, 256, 4, 1024, 512, false>(a, s);
  else if (candidates <= 8192 && rows > kCUs) launch<KIND, 256, 8, 1024, 512, false>(a, s);
  else if (candidates <= 16384) launch<KIND, 512, 8, 2048, 1024, false>(a, s);
  else if (candidates <= kRegisterRow && rows > kCUs) launch<KIND, 512, 16, 2048, 1024, false>(a, s);
  else if (candidates <= kRegisterRow) launch<KIND, 1024, 8, 2048, 1024, false>(a, s);
  else launch<KIND, 1024, 8, 2048, 1024, true>(a, s);
}

}  // namespace

hipError_t launch_choose(const SelectArgs& a, int kind, int64_t candidates, hipStream_t s) {
  if (kind == HISPARSE_INDEX_KEYS) launch_kind<HISPARSE_INDEX_KEYS>(a, candidates, s);
  else if (kind == HISPARSE_INDEX_BOUNDS) launch_kind<HISPARSE_INDEX_BOUNDS>(a, candidates, s);
  else launch_kind<HISPARSE_INDEX_MEANS>(a, candidates, s);
  return hipGetLastError();
}

}  // namespace hisparse
