// Attention of chunks of new tokens over token records (hisparse_chunk_attention).
//
// For new token i of a request with n new and len cached tokens, and query head e on kv head h:
//   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j - m),  m the largest score,
// over the cached tokens j that it sees: j < len, j <= len - n + i (causal), j > len - n + i -
// window, and its record not padding.
#include <algorithm>

#include "attention_device.h"
#include "chunk_plan.h"
#include "fetch_device.h"
#include "tokens.h"

namespace hisparse {
namespace {

constexpr float kLn2 = 0.6931471805599453f;
// Exponentials are taken against a reference per row, the largest score of the first tile that it
// sees, which moves only when weights outgrow it: exact softmax arithmetic with another reference
// point, and no search for the largest score in the other tiles. (The score that the reference was
// taken from weighs 1, so that a row's sum is at least that.) What must stay inside the float range is
// the sums, and the output, which is up to them times the largest value.
// Grouped-query records: the weights that a lane has of a tile add up to this at most, 2^16, so that
// values up to 2^111 over the number of tokens seen leave the output finite. (With 2^64 values from 2^64
// on did not; a smaller limit moves the reference oftener where scores are sharp: the mixed batch of
// 8-bit pages with queries times 12 takes 242 us with 2^64, 280 with 2^16, 301 with 2^8; with its own
// queries 242 in all three.)
constexpr float kTileLimit = 65536.f;
// Latent ones, for which moving the reference costs two more passes: a row's weights add up to this
// at most (2^64, far inside the range of sums over 2^30 tokens), and where they add up to more than
// the number of tokens the output is looked at.
constexpr float kWeightLimit = 18446744073709551616.f;
// Up to this reference a weight comes from one fused multiply-add; beyond it the product is rounded
// first, as the reference was, or a weight could leave the float range.
constexpr float kFused = 16777216.f;

struct ChunkArgs : ChunkShape {
  const uint8_t* pool;
  const int32_t* table;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  float* part_o;    // unnormalised outputs of splits, 32 rows at a time (see part_quad)
  float2* part_ml;  // [part rows] (reference in log2 units, sum)
  int64_t record_stride, head_stride, request_stride;
  int64_t q_stride, out_stride, table_request_stride, table_head_stride;
  int64_t num_records;
  KvLayout l;
  int32_t causal;
  int32_t* n_split;             // where few row tiles are split: how many of a kv head, left for the
                                // merge by the last workgroup; or NULL
  FastDiv div_g;
  float scale_log2;
};

// The kernel's arguments (its only parameter) once more: what is read from here is loaded then, and
// not kept in scalar registers through a loop that is short of them.
__device__ __forceinline__ const ChunkArgs& arguments_again() {
  auto p = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const ChunkArgs*)p;
}

// ---- which piece of the call a workgroup does ------------------------------------------------

struct Work {
  Request q;
  int req, groups, tile, split, splits;
  int64_t part_row;  // first partial-result row of the tile's split 0
};

// Lane moves inside the vector unit (a shuffle by way of LDS takes about ten times as long).
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ int moved(int x) {  // 0 where nothing comes from
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
  x += moved<0x128>(x);  // 16 lanes: rotations by 8, 4, 2, 1
  x += moved<0x124>(x);
  x += moved<0x122>(x);
  x += moved<0x121>(x);
  auto of = [&](int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); };
  return (of(0) + of(16)) + (of(32) + of(48));
}
__device__ __forceinline__ int wave_prefix(int x) {  // inclusive
  x += moved<0x111>(x);  // 16 lanes: shifts by 1, 2, 4, 8
  x += moved<0x112>(x);
  x += moved<0x114>(x);
  x += moved<0x118>(x);
  x += moved<0x142, 0xa>(x);         // lane 15 of rows 0 and 2 to the row behind
  return x + moved<0x143, 0xc>(x);  // lane 31 to the upper half
}

// The length of parts (see choose_part). Wave-uniform.
template <bool LATENT>
__device__ __forceinline__ int part_of(const ChunkArgs& a, const Request& first) {
  if (!a.target || a.num_splits) return 0;
  const int lane = threadIdx.x & 63;
  uint64_t blocks = 0;
  uint32_t tiles = 0;
  for (int base = 0; base < a.requests; base += 64) {
    const int r = base + lane;
    uint64_t x = 0;
    int groups, t = 0;
    if (r < a.requests) {
      const Request q = base == 0 ? first : request_of(a, r);
      t = tiles_of(a, LATENT, q, groups);
      x = blocks_of(a, q, t);  // below 2^50
    }
    blocks += wave_sum((uint32_t)x & 0xffffff);
    if (__ballot(x >> 24)) blocks += (uint64_t)wave_sum((uint32_t)(x >> 24)) << 24;
    tiles += wave_sum((uint32_t)t);
  }
  return choose_part(blocks, (int)tiles, a.kv_heads, LATENT, [&](int part) {
    uint32_t items = 0;
    for (int base = 0; base < a.requests; base += 64) {
      const int r = base + lane;
      int groups, n = 0;
      if (r < a.requests) {
        const Request q = base == 0 ? first : request_of(a, r);
        n = tiles_of(a, LATENT, q, groups) * splits_of(a, q, part);
      }
      items += wave_sum((uint32_t)n);
    }
    return items;
  });
}
__device__ __forceinline__ Request first_request(const ChunkArgs& a) {
  const int lane = threadIdx.x & 63;
  return lane < a.requests ? request_of(a, lane) : Request{0, 0, 0};
}

// How many row tiles of a kv head are split. Wave-uniform.
template <bool LATENT>
__device__ __forceinline__ int split_tiles(const ChunkArgs& a) {
  const int lane = threadIdx.x & 63;
  const Request first = first_request(a);
  const int part = part_of<LATENT>(a, first);
  int n = 0;
  for (int base = 0; base < a.requests; base += 64) {
    const int r = base + lane;
    int groups, tiles = 0;
    if (r < a.requests) {
      const Request q = base == 0 ? first : request_of(a, r);
      if (splits_of(a, q, part) > 1) tiles = tiles_of(a, LATENT, q, groups);
    }
    n += __builtin_amdgcn_readlane(wave_prefix(tiles), 63);
  }
  return n;
}

template <bool LATENT>
__device__ __forceinline__ void leave_split_tiles(const ChunkArgs& a) {
  if (a.n_split && blockIdx.x == gridDim.x - 1) {
    const int n = split_tiles<LATENT>(a);
    if (threadIdx.x == 0) *a.n_split = n;
  }
}

// Item `item` of a kv head's work: MERGE: row tiles that are split, else (row tile, split)s, request
// by request, each request's tiles from the last (which see most) to the first.
// False if there are fewer items. Wave-uniform.
template <bool LATENT, bool MERGE>
__device__ __forceinline__ bool find_work(const ChunkArgs& a, int item, Work& w) {
  const int lane = threadIdx.x & 63;
  if (!a.start && !a.kv_len) {
    const int bm = 32 * row_groups(a.max_chunk * a.g, LATENT, a.split);
    const int per = MERGE ? a.uni_tiles : a.uni_tiles * a.uni_splits;
    w.req = item / per;
    if (w.req >= a.requests) return false;
    w.q = request_of(a, w.req);
    const int x = item - w.req * per;
    w.groups = bm / 32;
    w.splits = a.uni_splits;
    w.tile = MERGE ? x : x / w.splits;
    w.split = MERGE ? 0 : x - w.tile * w.splits;
    w.part_row = (int64_t)(w.req * a.uni_tiles + w.tile) * w.splits * bm;
    w.tile = a.uni_tiles - 1 - w.tile;
    return true;
  }
  const Request first = first_request(a);  // loaded once for both passes
  const int part = part_of<LATENT>(a, first);
  uint32_t items = 0;
  int64_t rows = 0;
  for (int base = 0; base < a.requests; base += 64) {
    const int r = base + lane;
    Request q{0, 0, 0};
    int groups = 1, tiles = 0, splits = 1;
    if (r < a.requests) {
      q = base == 0 ? first : request_of(a, r);
      tiles = tiles_of(a, LATENT, q, groups);
      splits = splits_of(a, q, part);
    }
    const uint32_t pieces = items_of(tiles, splits);
    const uint32_t mine = !MERGE ? pieces : splits > 1 ? (uint32_t)tiles : 0;
    const uint32_t mine_rows = splits > 1 ? pieces * (uint32_t)groups : 0;
    const uint32_t pi = wave_prefix((int)mine), pr = wave_prefix((int)mine_rows);
    const uint64_t hit = __ballot(items + pi > (uint32_t)item);
    if (hit) {
      const int src = __builtin_ctzll(hit);
      auto get = [&](int x) { return __builtin_amdgcn_readlane(x, src); };
      w.req = base + src;
      w.q = Request{get(q.begin), get(q.n), get(q.len)};
      w.groups = get(groups);
      w.splits = get(splits);
      const int x = item - (int)(items + (uint32_t)get((int)(pi - mine)));
      w.tile = MERGE ? x : x / w.splits;
      w.split = MERGE ? 0 : x - w.tile * w.splits;
      w.part_row = (rows + (uint32_t)get((int)(pr - mine_rows)) +
                    (int64_t)w.tile * w.splits * w.groups) * 32;
      w.tile = get(tiles) - 1 - w.tile;
      return partial_rows_fit(a, w.part_row, w.splits, w.groups);
    }
    items += (uint32_t)__builtin_amdgcn_readlane((int)pi, 63);
    rows += (uint32_t)__builtin_amdgcn_readlane((int)pr, 63);
  }
  return false;
}

  // 8 e4m3 values times the power of two s, in bf16.
  __device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi, float s) {
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s, true));
    return r;
  }
  // x with its non-finite bf16 values cleared; true if there was one.
  __device__ __forceinline__ bool clear_bad(u32x4& x) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool lo = (x[i] & 0x7f80u) == 0x7f80u, hi = (x[i] & 0x7f800000u) == 0x7f800000u;
      bad |= lo | hi;
      x[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
    }
    return bad;
  }

// x if it is an infinity or NaN, else 0 (in bit operations, for the reason given at mask_scores).
__device__ __forceinline__ float if_not_finite(float x) {
  const uint32_t b = __float_as_uint(x);
  return __uint_as_float(b & (uint32_t)((int32_t)((b & 0x7fffffffu) + 0x00800000u) >> 31));
}
// The same for e4m3 values (NaN is 0x7f, with either sign; there are no infinities).
__device__ __forceinline__ bool clear_bad8(u32x4& x) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t b = ((x[i] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    any |= b;
    x[i] &= ~((b >> 7) * 0xffu);
  }
  return any != 0;
}
// ln of a softmax's sum from its reference (log2 units) and the sum against it.
__device__ __forceinline__ float natural(float m, float l) {
  return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}
__device__ __forceinline__ bf16x8_t words(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8_t, u32x4{a, b, c, d});
}
typedef u32x4 any_u32x4 __attribute__((aligned(2)));  // queries and outputs start at any element
typedef u32x2 any_u32x2 __attribute__((aligned(2)));
__device__ __forceinline__ void store_bf16x4(uint16_t* to, f32x4 y) {
  const bf16x2_t b0 = __builtin_convertvector(f32x2{y[0], y[1]}, bf16x2_t);
  const bf16x2_t b1 = __builtin_convertvector(f32x2{y[2], y[3]}, bf16x2_t);
  *reinterpret_cast<any_u32x2*>(to) =
      u32x2{__builtin_bit_cast(uint32_t, b0), __builtin_bit_cast(uint32_t, b1)};
}

// Partial results are stored as the accumulators hold them, so that every lane writes 16 contiguous
// bytes of a wave's 1024: per 32 rows, quad 4n + x (dims 32n + 8x ..), lane (row lane & 31), dims +
// 4 (lane / 32) .. +3. (Row by row a store touched 32 rows, 32 bytes of each.)
__device__ __forceinline__ float* part_quad(float* part_o, int64_t part_row, int d_v, int quad,
                                            int lane) {
  return part_o + part_row * d_v + (quad * 64 + lane) * 4;
}

// The cached tokens [lo, hi) that new token i of a request sees (hi may be below lo).
__device__ __forceinline__ int seen_to(const ChunkArgs& a, const Request& q, int i) {
  return a.causal ? min(q.len, q.len - q.n + i + 1) : q.len;
}
__device__ __forceinline__ int seen_from(const ChunkArgs& a, const Request& q, int i) {
  return a.window ? max(0, q.len - q.n + i + 1 - a.window) : 0;
}

// Tokens that do not exist are read from here.
__device__ __attribute__((aligned(16))) uint8_t g_zero_row[1152];
// The address of g_zero_row, kept: left to itself the compiler loads it at every use, and waits for
// the LDS reads in flight on the way.
__device__ __forceinline__ const uint8_t* zero_row() {
  const uint8_t* p = g_zero_row;
  asm volatile("" : "+s"(p));
  return p;
}

// What the rows of a workgroup (ROWS of them from row0 on) and one of its groups of 32 see, where
// the cached tokens are, and this lane's row.
struct View {
  const int32_t* table;
  const uint8_t* pool;
  int t0, t1;          // this split's tokens [t0, t1)
  int hi_min, lo_max;  // tokens in [lo_max, hi_min) are seen by every row of the workgroup
  int w_lo, w_hi;      // and by every row of the group; none of which sees w_end or later ones
  int w_end;
  int row_lo, row_hi;  // what this lane's row sees
  int tok, head;       // its new token and query head (of all heads)
  bool live, group_live;  // this row, any row of the group exists; one past the end stands in for
                          // the last
};
template <int ROWS>
__device__ __forceinline__ View view_of(const ChunkArgs& a, const Work& w, int h, int group,
                                        int col) {
  View v;
  const Request& q = w.q;
  const int n_rows = q.n * a.g, row0 = w.tile * ROWS;
  const int first = (int)fastdiv(row0, a.div_g);
  const int last = (int)fastdiv(min(n_rows, row0 + ROWS) - 1, a.div_g);
  const int lo = seen_from(a, q, first), hi = max(seen_to(a, q, last), 0);
  v.hi_min = seen_to(a, q, first);
  v.lo_max = seen_from(a, q, last);
  v.table = a.table + w.req * a.table_request_stride + h * a.table_head_stride;
  v.pool = a.pool + w.req * a.request_stride + h * a.head_stride;
  const int base = lo & ~63, blocks = max(0, hi - base + 63) >> 6;
  const int c = (blocks + w.splits - 1) / w.splits;
  v.t0 = base + w.split * c * 64;
  v.t1 = min(hi, v.t0 + c * 64);
  const int row_w = row0 + 32 * group, row = min(row_w + col, n_rows - 1);
  v.group_live = row_w < n_rows;
  v.live = row_w + col < n_rows;
  v.tok = (int)fastdiv(row, a.div_g);
  v.head = h * a.g + row - v.tok * a.g;
  v.row_hi = seen_to(a, q, v.tok);
  v.row_lo = seen_from(a, q, v.tok);
  const int g_first = (int)fastdiv(min(row_w, n_rows - 1), a.div_g);
  const int g_last = (int)fastdiv(min(row_w + 31, n_rows - 1), a.div_g);
  v.w_hi = __builtin_amdgcn_readfirstlane(seen_to(a, q, g_first));
  v.w_lo = __builtin_amdgcn_readfirstlane(seen_from(a, q, g_last));
  v.w_end = __builtin_amdgcn_readfirstlane(seen_to(a, q, g_last));
  return v;
}

// The token of a 32-token group that register i of half 0 of a lane's S^T accumulator holds (half
// 1: one more).
__device__ constexpr int score_token(int i) {
  return 16 * (i >> 3) + 4 * (i & 3) + 2 * ((i >> 2) & 1);
}

// Bits of the tokens base .. base + 31 that lie in [lo, hi) and in `exist`, moved down by `half`: bit
// score_token(i) is register i's.
__device__ __forceinline__ uint32_t seen_bits(uint32_t exist, int lo, int hi, int base, int half) {
  lo = max(lo - base, 0);
  hi = min(hi - base, 32);
  const uint32_t range = lo < hi ? (0xffffffffu >> (32 - hi + lo)) << lo : 0u;
  return (range & exist) >> half;
}
// A score whose token is not seen weighs nothing. (Bit operations on the score itself: compares
// would hold a pair of scalar registers for each of 16 lane masks.)
__device__ __forceinline__ void mask_scores(f32x16& s, uint32_t seen) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t m = (uint32_t)((int32_t)(seen << (31 - score_token(i))) >> 31);
    s[i] = __uint_as_float((__float_as_uint(s[i]) & m) | (0xff800000u & ~m));
  }
}
// Softmax weights of 16 N scores (raw products) of this lane's row against a reference, in pairs
// rounded to bf16 (times their tokens' value scales, if given: powers of two, which round nothing);
// returns their unrounded sum. The rounding is the MFMA operand's: 2^-8 of a weight at most, each token's
// its own, so that results are off by 0.0019 to 0.0024 of their norm, and by 0.0017 from their own
// rounding to bf16 alone. A weight in two bf16 terms would double the MFMAs with V.
template <int N>
__device__ __forceinline__ float weights_of(uint32_t (&pw)[N][8], const f32x16 (&s)[N],
                                            float scale, float ref,
                                            const u32x4* value_scale = nullptr) {
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      f32x2 p = {__builtin_amdgcn_exp2f(__builtin_fmaf(s[j][i], scale, -ref)),
                 __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][i + 1], scale, -ref))};
      sum[i & 2] += p[0];
      sum[(i & 2) + 1] += p[1];
      if (value_scale) {
        p[0] *= __uint_as_float(value_scale[4 * j + (i >> 2)][i & 3]);
        p[1] *= __uint_as_float(value_scale[4 * j + (i >> 2)][(i & 3) + 1]);
      }
      pw[j][i >> 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2_t));
    }
  return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}
// The largest of a row's 16 N scores on its two lanes, times the scale.
template <int N>
__device__ __forceinline__ float largest(const f32x16 (&s)[N], float scale) {
  float c = s[0][0];
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) c = fmaxf(c, s[j][i]);
  c *= scale;
  return fmaxf(c, __shfl_xor(c, 32, 64));
}
// Weights against a reference whose products would not stay in range unrounded, or none (-inf).
template <int N>
__device__ __forceinline__ float weights_rounded(uint32_t (&pw)[N][8], f32x16 (&s)[N],
                                                 float scale, float ref,
                                                 const u32x4* value_scale = nullptr) {
  if (ref == -INFINITY) ref = 0.f;
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[j][i] = over_reference(s[j][i], scale, ref);
  return weights_of<N>(pw, s, 1.f, 0.f, value_scale);
}
// The rare cases: rows without a reference, rows that outgrew theirs (both get the largest of these
// scores, sum and output following), and references whose products would not stay in range
// unrounded.
template <int N, int NO>
__device__ __forceinline__ float weights_moved(uint32_t (&pw)[N][8], f32x16 (&s)[N], float scale,
                                               float& m_run, float& l_run, f32x16 (&o)[NO]) {
  const float m_new = fmaxf(m_run, largest<N>(s, scale));
  // without a reference, sum and output are zero
  const float alpha = m_run == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
  m_run = m_new;
  l_run *= alpha;
#pragma unroll
  for (int n = 0; n < NO; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[n][i] *= alpha;
  return weights_rounded<N>(pw, s, scale, m_new);
}
// The weights of a row's next 16 N scores; its sum, and where need be its reference and output,
// follow.
template <int N, int NO>
__device__ __forceinline__ void next_weights(uint32_t (&pw)[N][8], f32x16 (&s)[N], float scale,
                                             float& m_run, float& l_run, f32x16 (&o)[NO]) {
  float sum = 0.f;
  bool rare = __ballot(!(__builtin_fabsf(m_run) <= kFused)) != 0;  // -inf: none yet
  if (__builtin_expect(!rare, 1)) {
    sum = weights_of<N>(pw, s, scale, m_run);
    rare = __ballot(!(sum <= kTileLimit)) != 0;
  }
  if (__builtin_expect(rare, 0)) sum = weights_moved<N, NO>(pw, s, scale, m_run, l_run, o);
  l_run += sum;
}

// ---- grouped-query records -------------------------------------------------------------------
//
// A workgroup is eight waves, RW row waves of 32 rows each in TG = 8 / RW token groups; a group's
// waves share tiles of CT tokens (K | V in bf16) in LDS, staged by way of registers: the next
// tile's loads are in flight while one is computed on, 8-bit rows are widened on their way to LDS
// (exact: the scale is a power of two), and tokens that nobody may see are stored as zeros. (16-bit
// tiles of 256 rows: by direct loads.)
//   S^T[token][row] = K[token][:] . Q^T[:][row]    v_mfma_f32_32x32x16_bf16, Q in registers
//   O^T[dim][row]  += V^T[dim][token] P^T[token][row]   the same, V by LDS transpose reads
// A lane holds one row: 16 of a tile's 32 scores (lane ^ 32 holds the others), which in the token
// order of mla_row are its P operands, and the row's reference, sum and limits are one register
// each.
//
// Many rows are bound by the issue of MFMAs and of the softmax (6 other vector instructions for each
// MFMA): 2048 tokens x 64 heads on 4 kv heads over 16384 tokens in 1030 us, 1.00 PFLOP/s (other cards up
// to 1060). Few rows are bound by HBM: one token of 64 requests x 8 kv heads x 4 over 4096 8-bit tokens
// in 111 us, 5.0 TB/s.

using GTile = Tile<32>;  // 32 tokens of 32 pieces: K 0..15, V 16..31

// LDS of a workgroup, whichever its path: tiles, bad-token marks, the groups' (max, sum) pairs.
constexpr int kGroupedMarks = 8 * GTile::BYTES;
constexpr int kGroupedMl = kGroupedMarks + 8 * 2 * 65 * 4;
constexpr int kGroupedLds = kGroupedMl + 8 * 32 * 8;

template <bool FP8, int RW, int TG, int CT>
struct Grouped {
  static constexpr int NB = RW == 8 ? 3 : RW == 1 ? 1 : 2;  // tile buffers
  static constexpr int NS = CT / 32;
  static constexpr int TILE = NS * GTile::BYTES;
  static constexpr int RGW = CT / 8 / RW;  // groups of eight rows that a wave stages
  static constexpr int NLD = FP8 ? 2 : 4;  // 16-byte loads of a lane's row
  static constexpr int LDS_TILES = TG * NB * TILE;
  static_assert(LDS_TILES <= kGroupedMarks && TG * NB * (CT + 1) * 4 <= kGroupedMl - kGroupedMarks,
                "LDS");
  static_assert(RW * TG == 8 && CT % (8 * RW) == 0 && CT <= 64, "shape");

  // 16-bit tiles of the widest path go to LDS directly
  static constexpr bool DIRECT = RW == 8 && !FP8;

  struct Staged {
    u32x4 x[RGW][NLD];
    f32x2 sc[RGW];
  };

  static __device__ __forceinline__ void run(const ChunkArgs& a, const Work& w, int h,
                                             uint8_t* s_mem) {
    const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hg = wave % RW, tg = wave / RW;
    uint8_t* s_tiles = s_mem + tg * NB * TILE;
    // tokens whose V is not finite in a tile that not every row sees: the tile's number + 1
    int* s_bad = reinterpret_cast<int*>(s_mem + kGroupedMarks) + tg * NB * (CT + 1);

    const View v = view_of<32 * RW>(a, w, h, hg, col);

    // ---- staging ----
    const int n_it = max(0, v.t1 - v.t0 + TG * CT - 1) / (TG * CT);
    auto tile_base = [&](int it) { return v.t0 + (it * TG + tg) * CT; };
    int32_t e[RGW];  // table entries of this lane's rows of the tile to load next
    int32_t ev;      // and of token `lane` of the tile whose scores come next
    auto entry = [&](int t) { return t < v.t1 ? v.table[t >> a.l.tpr_shift] : -1; };
    auto load_entries = [&](int it) {
      const int base = tile_base(it);
#pragma unroll
      for (int i = 0; i < RGW; ++i) e[i] = entry(base + 8 * (hg * RGW + i) + (lane >> 3));
    };
    auto mask_entry = [&](int it) { return entry(tile_base(it) + (lane & (CT - 1))); };
    Staged st;
    auto ok_entry = [&](int32_t r) { return r >= 0 && r < a.num_records; };
    auto issue = [&](int it) {
      const int base = tile_base(it);
#pragma unroll
      for (int i = 0; i < RGW; ++i) {
        const int t = base + 8 * (hg * RGW + i) + (lane >> 3);
        const int in = t & ((1 << a.l.tpr_shift) - 1);
        const uint8_t* rec = v.pool + (uint64_t)(uint32_t)e[i] * (uint32_t)a.record_stride;
        const uint8_t* src = rec + __umul24(in, a.l.row_bytes) + 16 * (lane & 7);
        if (ok_entry(e[i])) {
#pragma unroll
          for (int x = 0; x < NLD; ++x)
            st.x[i][x] = *reinterpret_cast<const u32x4*>(src + 128 * x);
          if constexpr (FP8)
            st.sc[i] = *reinterpret_cast<const f32x2*>(rec + a.l.scale_offset + 8 * in);
        } else {
#pragma unroll
          for (int x = 0; x < NLD; ++x) st.x[i][x] = u32x4{};
          if constexpr (FP8) st.sc[i] = f32x2{1.f, 1.f};
        }
      }
    };
    auto partial = [&](int base) { return base + CT > v.hi_min || base < v.lo_max; };
    auto mark_bad = [&](int it, int r) {
      s_bad[(it % NB) * (CT + 1) + 1 + r] = it + 1;
      s_bad[(it % NB) * (CT + 1)] = it + 1;
    };
    const uint8_t* const zero = zero_row();
    auto direct = [&](int it) {
      static_assert(!DIRECT || RGW == 1, "a wave stages eight rows");
      const int t = tile_base(it) + 8 * hg + (lane >> 3);
      const int in = t & ((1 << a.l.tpr_shift) - 1);
      const uint8_t* row = v.pool + (uint64_t)(uint32_t)e[0] * (uint32_t)a.record_stride +
                           __umul24(in, a.l.row_bytes);
      stage_rows<32>(s_tiles + (it % NB) * TILE + (hg >> 2) * GTile::BYTES, hg & 3,
                     (ok_entry(e[0]) ? row : zero) + stage_piece(lane, hg));
    };
    // this wave's rows of a tile that was stored directly
    auto scrub = [&](int it) {
      const int r = 8 * hg + (lane >> 3);
      bool bad = false;
#pragma unroll
      for (int x = 2; x < 4; ++x) {
        u32x4* at = reinterpret_cast<u32x4*>(s_tiles + (it % NB) * TILE + (r >> 5) * GTile::BYTES +
                                             GTile::row(r & 31) + x * 1024) + (lane & 7);
        u32x4 p = *at;
        if (clear_bad(p)) {
          bad = true;
          *at = p;
        }
      }
      if (bad) mark_bad(it, r);
    };
    auto store = [&](int it) {
      uint8_t* tile = s_tiles + (it % NB) * TILE;
      const bool part = partial(tile_base(it));
#pragma unroll
      for (int i = 0; i < RGW; ++i) {
        const int r = 8 * (hg * RGW + i) + (lane >> 3);
        uint8_t* dst = tile + (r >> 5) * GTile::BYTES + GTile::row(r & 31);
        const int sw = tile_swizzle(r);
        bool bad = false;
        if constexpr (FP8) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {  // K, V
            u32x4 p0 = widen(st.x[i][x][0], st.x[i][x][1], st.sc[i][x]);
            u32x4 p1 = widen(st.x[i][x][2], st.x[i][x][3], st.sc[i][x]);
            if (x == 1 && part) {
              bad |= clear_bad(p0);
              bad |= clear_bad(p1);
            }
            uint8_t* seg = dst + (2 * x + ((lane & 7) >> 2)) * 1024;
            const int p = 2 * (lane & 3);
            *reinterpret_cast<u32x4*>(seg + ((p ^ sw) << 4)) = p0;
            *reinterpret_cast<u32x4*>(seg + (((p + 1) ^ sw) << 4)) = p1;
          }
        } else {
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            u32x4 p = st.x[i][x];
            if (x >= 2 && part) bad |= clear_bad(p);
            *reinterpret_cast<u32x4*>(dst + x * 1024 + (((lane & 7) ^ sw) << 4)) = p;
          }
        }
        if (part && bad) mark_bad(it, r);
      }
    };

    load_entries(0);
    ev = mask_entry(0);
    for (int i = lane + 64 * hg; i < NB * (CT + 1); i += 64 * RW) s_bad[i] = 0;
    // Q^T operand: this lane's row, dims 16 kk + 8 half .. +7
    bf16x8_t qreg[8];
    {
      const uint16_t* q = a.q + (int64_t)(w.q.begin + v.tok) * a.q_stride + (int64_t)v.head * 128;
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
        qreg[kk] = __builtin_bit_cast(
            bf16x8_t, (u32x4)*reinterpret_cast<const any_u32x4*>(q + 16 * kk + 8 * half));
    }
    f32x16 o[4];
#pragma unroll
    for (int n = 0; n < 4; ++n) o[n] = f32x16{};
    float m_run = -INFINITY, l_run = 0.f;

    // ---- one tile's steps ----
    auto busy = [&](int it) { return v.group_live && tile_base(it) < v.w_end; };
    // S^T of a tile: K reads KD k-steps ahead of the MFMAs (see lds_read_b128)
    auto scores = [&](int it, f32x16 (&s)[NS]) {
      const int kr = mla_row(col), sw = tile_swizzle(kr);
      const uint32_t krow = lds_addr(s_tiles + (it % NB) * TILE + GTile::row(kr));
      uint32_t ka[4];  // piece 2 kk + half of k-steps kk, kk + 4
#pragma unroll
      for (int i = 0; i < 4; ++i) ka[i] = krow + (((2 * i + half) ^ sw) << 4);
      constexpr int N = 8 * NS, KD = 8;  // read x: k-step x / NS of tokens 32 (x % NS) ..
      u32x4 kb[KD];
      auto kread = [&](auto x) {
        constexpr int kk = x / NS, j = x % NS;
        kb[x % KD] = lds_read_b128<j * GTile::BYTES + (kk / 4) * 1024>(ka[kk & 3]);
      };
      static_for<KD>(kread);
      static_for<N>([&](auto x) {
        constexpr int later = N - 1 - x < KD - 1 ? N - 1 - x : KD - 1;
        constexpr int kk = x / NS, j = x % NS;
        lgkm_wait1<later>(kb[x % KD]);
        s[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, kb[x % KD]),
                                                      qreg[kk], kk == 0 ? f32x16{} : s[j], 0, 0,
                                                      0);
        if constexpr (x + KD < N) kread(std::integral_constant<int, x + KD>{});
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    auto softmax = [&](int it, f32x16 (&s)[NS], uint64_t exist, uint32_t (&pw)[NS][8]) {
      const int base = tile_base(it);
      constexpr uint64_t kFull = CT == 64 ? ~0ull : 0xffffffffull;
      if (base + CT > v.w_hi || base < v.w_lo || (exist & kFull) != kFull) {
#pragma unroll
        for (int j = 0; j < NS; ++j)
          mask_scores(s[j], seen_bits((uint32_t)(exist >> (32 * j)), v.row_lo, v.row_hi,
                                      base + 32 * j, half));
      }
      next_weights<NS, 4>(pw, s, a.scale_log2, m_run, l_run, o);
    };
    // O^T += V^T P^T. V by transpose reads: in each 16-lane group lane 4s + q addresses row 16 kb +
    // 4s + half (+ 2 for the second read), dims 32 n + 16 (col >> 4) + 4q .. +3; lane t of the
    // group then holds those rows of dim 32 n + 16 (col >> 4) + t, in P's token order.
    auto pv = [&](int it, const uint32_t (&pw)[NS][8]) {
      const int vr = 4 * ((lane & 15) >> 2) + half;
      const int vp = 2 * (col >> 4) + ((lane & 3) >> 1);
      const uint8_t* tile = s_tiles + (it % NB) * TILE;
      uint32_t va[2][2];  // [n & 1][first / second read]
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int y = 0; y < 2; ++y)
          va[n][y] = lds_addr(tile + GTile::row(vr + 2 * y) + 8 * (lane & 1) +
                              (((vp + 4 * n) ^ tile_swizzle(vr + 2 * y)) << 4));
      constexpr int N = 8 * NS, VD = 6;  // MFMA x: tokens 16 (x / 4) .., dims 32 (x % 4) ..
      v4i16 lo[VD], hi[VD];
      auto vread = [&](auto x) {
        constexpr int j = x / 8, kb = x / 4 % 2, n = x % 4;
        constexpr int OFF = j * GTile::BYTES + kb * 2 * GTile::NSEG * 1024 + (2 + n / 2) * 1024;
        lo[x % VD] = lds_read_tr16_b64<OFF>(va[n & 1][0]);
        hi[x % VD] = lds_read_tr16_b64<OFF>(va[n & 1][1]);
      };
      static_for<VD>(vread);
      static_for<N>([&](auto x) {
        constexpr int later = N - 1 - x < VD - 1 ? N - 1 - x : VD - 1;
        constexpr int j = x / 8, kb = x / 4 % 2, n = x % 4;
        lgkm_wait2<2 * later>(lo[x % VD], hi[x % VD]);
        const bf16x8_t vt = __builtin_bit_cast(
            bf16x8_t, __builtin_shufflevector(lo[x % VD], hi[x % VD], 0, 1, 2, 3, 4, 5, 6, 7));
        o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            vt, words(pw[j][4 * kb], pw[j][4 * kb + 1], pw[j][4 * kb + 2], pw[j][4 * kb + 3]),
            o[n], 0, 0, 0);
        if constexpr (x + VD < N) vread(std::integral_constant<int, x + VD>{});
        __builtin_amdgcn_sched_barrier(0);
      });
      // Infinities and NaN in V of a tile that only some rows see were stored as zeros (zero
      // weights would have made NaN of them): they go to the rows that see them here.
      const int base = tile_base(it);
      if (partial(base) &&
          __builtin_amdgcn_readfirstlane(s_bad[(it % NB) * (CT + 1)]) == it + 1) {
        for (int t = 0; t < CT; ++t) {
          if (s_bad[(it % NB) * (CT + 1) + 1 + t] != it + 1) continue;
          const int tk = base + t;
          if (tk >= v.row_hi || tk < v.row_lo) continue;
          const uint8_t* rec = v.pool + (int64_t)v.table[tk >> a.l.tpr_shift] * a.record_stride;
          const int in = tk & ((1 << a.l.tpr_shift) - 1);
          const uint8_t* vrow = rec + (int64_t)in * a.l.row_bytes + (FP8 ? 128 : 256);
          float sc = 1.f;
          if constexpr (FP8)
            sc = reinterpret_cast<const float*>(rec + a.l.scale_offset)[2 * in + 1];
#pragma unroll
          for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int d = 32 * n + 8 * (i >> 2) + 4 * half + (i & 3);
              float x;
              if constexpr (FP8) x = __builtin_amdgcn_cvt_f32_fp8(vrow[d], 0) * sc;
              else x = bf16_to_f32(reinterpret_cast<const uint16_t*>(vrow)[d]);
              o[n][i] += if_not_finite(x);
              if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // few loads at a time
            }
        }
      }
    };
    f32x16 s[NS];
    uint32_t pw[NS][8];

    if constexpr (RW == 8) {
      // The two waves of a SIMD (w and w + 4) take turns: while one's MFMAs run (V of tile i - 1,
      // scores of tile i) the other works out its softmax and stages, a barrier apart. Waves 4..7
      // are half a tile behind, so they stage a tile further ahead. Tile t is read until the
      // second MFMA phase of t + 1; three buffers.
      // By way of registers, tile t is stored in the softmax phase before its first reader's
      // MFMAs. Directly, it is sent for in the slot in which its buffer comes free: by waves 0..3
      // as their MFMA phase begins, by 4..7 a softmax phase earlier.
      const int lead = wave >= 4 ? 2 : 1;
      if (n_it > 0) {
        if constexpr (DIRECT) {
          direct(0);
          load_entries(1);
          if (lead == 2) {
            if (n_it > 1) direct(1);
            load_entries(2);
          }
          wait_loads_and_barrier<0>();
          // the query too: a wait for it inside the loop would drain the tiles in flight
#pragma unroll
          for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+v"(qreg[kk]));
          if (lead == 2 && partial(tile_base(0))) scrub(0);
        } else {
          issue(0);
          load_entries(1);
          lds_barrier();  // s_bad is clear
          store(0);
          if (lead == 2 && n_it > 1) {
            issue(1);
            load_entries(2);
            store(1);
          }
          if (lead < n_it) issue(lead);
          load_entries(lead + 1);
          lds_barrier();  // tile 0 is stored
        }
        if (lead == 2) lds_barrier();
        for (int i = 0; i <= n_it; ++i) {
          if (DIRECT && lead == 1) {
            if (i + 1 < n_it) direct(i + 1);
            load_entries(i + 2);
          }
          if (i > 0 && busy(i - 1)) pv(i - 1, pw);
          if (i < n_it && busy(i)) scores(i, s);
          if (DIRECT && lead == 2) wait_loads_and_barrier<0>();  // tile i + 1 is here
          else lds_barrier();
          if (i < n_it) {
            const uint64_t exist = __ballot(ok_entry(ev));
            if constexpr (DIRECT) {
              if (lead == 2) {
                if (i + 2 < n_it) direct(i + 2);
                load_entries(i + 3);
              }
              const int t = i + lead - 1;
              if (t < n_it && partial(tile_base(t))) scrub(t);
            }
            ev = mask_entry(i + 1);
            if (busy(i)) softmax(i, s, exist, pw);
            if constexpr (!DIRECT) {
              if (i + lead < n_it) {
                store(i + lead);
                if (i + lead + 1 < n_it) issue(i + lead + 1);
                load_entries(i + lead + 2);
              }
            }
          }
          if (DIRECT && lead == 1) wait_loads_and_barrier<0>();
          else lds_barrier();
        }
        if (lead == 1) lds_barrier();
      }
    } else {
      if (n_it > 0) {
        issue(0);
        load_entries(1);
        lds_barrier();  // s_bad is clear
        store(0);
      }
      for (int it = 0; it < n_it; ++it) {
        // tile `it` is stored, tile it - 1 read by all (one wave alone: in its own order)
        if constexpr (RW > 1) lds_barrier();
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const uint64_t exist = __ballot(ok_entry(ev));
        ev = mask_entry(it + 1);
        if (it + 1 < n_it) {
          issue(it + 1);
          load_entries(it + 2);
        }
        if (busy(it)) {
          scores(it, s);
          softmax(it, s, exist, pw);
          pv(it, pw);
        }
        asm volatile("" ::: "memory");
        if (it + 1 < n_it) store(it + 1);
      }
    }
    l_run += __shfl_xor(l_run, 32, 64);

    // ---- the token groups' results merged through LDS, in group order ----
    float m = m_run, l = l_run;
    if constexpr (TG > 1) {
      float2* s_ml = reinterpret_cast<float2*>(s_mem + kGroupedMl);
      __syncthreads();
      f32x4* s_o = reinterpret_cast<f32x4*>(s_mem);  // [TG][RW][16 quads][64 lanes]
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          s_o[(wave * 16 + n * 4 + x) * 64 + lane] =
              f32x4{o[n][4 * x], o[n][4 * x + 1], o[n][4 * x + 2], o[n][4 * x + 3]};
      if (half == 0) s_ml[wave * 32 + col] = make_float2(m_run, l_run);
      __syncthreads();
      m = -INFINITY;
      float2 ml[TG];
#pragma unroll
      for (int t = 0; t < TG; ++t) {
        ml[t] = s_ml[(t * RW + hg) * 32 + col];
        m = fmaxf(m, ml[t].x);
      }
      l = 0.f;
      float wt[TG];
#pragma unroll
      for (int t = 0; t < TG; ++t) {
        wt[t] = ml[t].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml[t].x - m);
        l += ml[t].y * wt[t];
      }
      // this wave finishes 16 / TG quads of its rows
      constexpr int NQ = 16 / TG;
      f32x4 r[NQ];
#pragma unroll
      for (int x = 0; x < NQ; ++x) {
        r[x] = f32x4{};
#pragma unroll
        for (int t = 0; t < TG; ++t)
          r[x] += s_o[((t * RW + hg) * 16 + tg * NQ + x) * 64 + lane] * wt[t];
      }
      if (v.live) finish<NQ>(arguments_again(), w, v, h, r, tg * NQ, hg * 32 + col, m, l, half);
    } else {
      f32x4 r[16];
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          r[4 * n + x] = f32x4{o[n][4 * x], o[n][4 * x + 1], o[n][4 * x + 2], o[n][4 * x + 3]};
      if (v.live) finish<16>(arguments_again(), w, v, h, r, 0, hg * 32 + col, m, l, half);
    }
  }

  // NQ quads of a row's result from quad q0 on (quad 4n + x: dims 32n + 8x + 4 half .. +3).
  template <int NQ>
  static __device__ __forceinline__ void finish(const ChunkArgs& a, const Work& w,
                                                const View& v, int h, const f32x4* r, int q0,
                                                int tile_row, float m, float l, int half) {
    const bool first = q0 == 0 && half == 0;
    if (w.splits > 1) {
      const int64_t pr = h * a.head_part_rows + w.part_row + (w.split * RW + (tile_row >> 5)) * 32;
#pragma unroll
      for (int x = 0; x < NQ; ++x)
        *reinterpret_cast<f32x4*>(part_quad(a.part_o, pr, 128, q0 + x, threadIdx.x & 63)) = r[x];
      if (first) a.part_ml[pr + (tile_row & 31)] = make_float2(m, l);
      return;
    }
    const float inv = l > 0.f ? 1.f / l : l;
    uint16_t* out =
        a.out + (int64_t)(w.q.begin + v.tok) * a.out_stride + (int64_t)v.head * 128;
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
      const int q = q0 + x;
      store_bf16x4(out + 32 * (q >> 2) + 8 * (q & 3) + 4 * half, r[x] * inv);
    }
    if (a.lse && first)
      a.lse[(int64_t)(w.q.begin + v.tok) * (a.kv_heads * a.g) + v.head] = natural(m, l);
  }
};

template <bool FP8>
__global__ __launch_bounds__(512, 2) void chunk_grouped_kernel(ChunkArgs a) {
  __shared__ __align__(1024) uint8_t s_mem[kGroupedLds];
  leave_split_tiles<false>(a);
  const int item = blockIdx.x / a.kv_heads, h = blockIdx.x - item * a.kv_heads;
  Work w;
  if (!find_work<false, false>(a, item, w)) return;
  if (w.groups == 1) Grouped<FP8, 1, 8, 32>::run(a, w, h, s_mem);
  else if (w.groups == 2) Grouped<FP8, 2, 4, 32>::run(a, w, h, s_mem);
  else if (w.groups == 4) Grouped<FP8, 4, 2, 64>::run(a, w, h, s_mem);
  else Grouped<FP8, 8, 1, 64>::run(a, w, h, s_mem);
}

// ---- latent records --------------------------------------------------------------------------
//
// Four waves, one per SIMD with all of its registers, in TG token groups of RG row waves: 128 rows on
// one tile, or 64 rows (a second row wave without rows only stages) on two tiles at once. A tile is
// 32 tokens of 1152 bytes (512 latent and 64 rotary dims in bf16; the value is the latent part).
// A wave keeps its 32 rows' query (144 registers a lane) and output (256 accumulators; the score
// MFMAs are assembly so that theirs are not, see mfma_qk). Nothing but MFMAs touches the output: a
// row's reference stays the largest score of the first tile that it sees. If some row's weights, or
// their products with its values, outgrow the range (kWeightLimit), the workgroup goes over its tokens
// twice more: for every row's largest score, then for the result against those.
// Tiles are stored by direct loads NB - 1 tiles ahead, sent in the shadow of the MFMAs. 8-bit
// tiles stay so in LDS (half the traffic) and are widened by the wave that reads an operand, exactly:
// e4m3 fits bf16. Their scales join where they cost least: the latent part of a score is multiplied
// by its token's (the rotary part, a chain of MFMAs of its own, is not), and so is the weight that
// goes with the token's value.
// Bound by the issue of one wave a SIMD (a vector instruction costs it about 8 cycles, an MFMA 32): 512
// tokens of 128 heads over 8192 16-bit tokens in 1021 us (other cards up to 1060), 1.11 PFLOP/s; 8-bit
// 1240, 0.91, for 256 widening instructions a tile. One token of 32 requests over 2048 8-bit tokens: 41 us
// and 9 for the merge, of which start 6, eight rounds of two tiles 26, results 4.5. 59 vector registers
// are spilled (8-bit; 16-bit 20), around the tiles' MFMAs, not between them.

using LTile = Tile<72>;  // 16-bit rows
using PTile = Tile<32>;  // 8-bit latent rows of 512 bytes
using RTile = Tile<8>;   // and their rotary dims

template <bool FP8, int TG>
struct Latent {
  static constexpr int CT = 32;
  static constexpr int RG = 4 / TG;            // row waves of a token group
  static constexpr int NB = (FP8 ? 6 : 4) / TG;  // tile buffers of a token group
  static constexpr int AHEAD = NB - 1;         // tiles between a load and its tile's scores
  // direct loads of a wave per tile: TG groups of eight rows; 8-bit, and the scales
  static constexpr int LOADS = FP8 ? 5 * TG + 1 : 9 * TG;
  static constexpr int TILE = FP8 ? PTile::BYTES + RTile::BYTES + RG * 256 : LTile::BYTES;
  // LDS: tiles (8-bit: latent rows, rotary dims, a copy of the 32 scales per wave), at whose end the
  // query passes first and in whose place the token groups' outputs are last; where WINDOW tokens
  // are (8-bit: also their rotary dims and scales) and which of them exist; bad-token marks; the
  // token groups' (reference, sum) pairs
  static constexpr int WINDOW = 512;
  static constexpr int ENTRIES = std::max(TG * NB * TILE, 4 * LTile::BYTES);
  static constexpr int QUERY = ENTRIES - RG * LTile::BYTES;
  // the first tiles, clear of the query: sent for before it is here
  static constexpr int EARLY = QUERY / (TG * TILE) < 1 ? 0 : 1;
  static constexpr int EXIST = ENTRIES + WINDOW * (FP8 ? 24 : 8);
  static constexpr int MARKS = EXIST + WINDOW / 8;
  static constexpr int N_MARKS = TG * NB * (CT + 1) + 1;  // the last: a row outgrew its reference
  static constexpr int ML = (MARKS + N_MARKS * 4 + 15) / 16 * 16;
  static constexpr int LDS = ML + 4 * 32 * 8;
  static_assert((AHEAD + 1) * TG * CT <= 256 && LDS <= 160 * 1024, "window and LDS");

  static __device__ __forceinline__ void run(const ChunkArgs& a, const Work& w, int h,
                                             uint8_t* s_mem) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tg = TG == 1 ? 0 : wave / RG, rg = TG == 1 ? wave : wave % RG;
    // What the loop derives from the lane is worked out anew in every tile: kept, it would spill,
    // and a reload waits for the direct loads in flight.
    auto lane_now = []() {
      int x = threadIdx.x & 63;
      asm volatile("" : "+v"(x));
      return x;
    };
    uint64_t* s_where = reinterpret_cast<uint64_t*>(s_mem + ENTRIES);
    uint64_t* s_exist = reinterpret_cast<uint64_t*>(s_mem + EXIST);
    int* s_marks = reinterpret_cast<int*>(s_mem + MARKS);
    int* s_outgrown = s_marks + N_MARKS - 1;
    const View v = view_of<32 * RG>(a, w, h, rg, threadIdx.x & 31);
    const int n_it = max(0, v.t1 - v.t0 + TG * CT - 1) / (TG * CT);
    auto first_token = [&](int it) { return (it * TG + tg) * CT; };  // from t0 on
    auto tile_base = [&](int it) { return v.t0 + first_token(it); };
    auto tile_at = [&](int it) { return s_mem + (it % NB * TG + tg) * TILE; };
    auto scales_at = [&](int it) { return tile_at(it) + PTile::BYTES + RTile::BYTES + rg * 256; };
    // a tile's marks: its number + 1 if a token has some, then per token the same
    auto marks_at = [&](int it) { return s_marks + (tg * NB + it % NB) * (CT + 1); };
    auto partial = [&](int base) { return base + CT > v.hi_min || base < v.lo_max; };

    // ---- where tokens are, worked out once per token, of WINDOW tokens from the current 256 on, so
    // that nothing in the loop waits for a load younger than the tiles': offsets from the pool, of
    // tokens that do not exist those of g_zero_row ----
    const uint8_t* const zero = zero_row();
    auto load_entry = [&](int block) {  // this thread's of 256 tokens
      const int t = v.t0 + block * 256 + (int)threadIdx.x;
      return t < v.t1 ? v.table[t >> a.l.tpr_shift] : -1;
    };
    auto store_entry = [&](int block, int32_t r) {
      const int at = (block & 1) * 256 + threadIdx.x;
      const bool ok = r >= 0 && r < a.num_records;
      const uint64_t rec = (uint64_t)(uint32_t)r * (uint32_t)a.record_stride;
      const uint64_t none = (uint64_t)(uintptr_t)zero - (uint64_t)(uintptr_t)v.pool;
      const int in = (v.t0 + block * 256 + (int)threadIdx.x) & ((1 << a.l.tpr_shift) - 1);
      s_where[at] = ok ? rec + __umul24(in, a.l.row_bytes) : none;
      if constexpr (FP8) {
        s_where[WINDOW + at] = ok ? rec + a.l.rope_offset + 128 * in : none;
        // scales lie in the order of the scores: token t's at its place in that order
        const int t = at & 31, p = 16 * (t & 1) + 8 * (t >> 4) + 4 * ((t >> 1) & 1) + ((t >> 2) & 3);
        s_where[2 * WINDOW + (at & ~31) + p] = ok ? rec + a.l.scale_offset + 4 * in : none;
      }
      const uint64_t mask = __ballot(ok);
      if ((threadIdx.x & 63) == 0) s_exist[at >> 6] = mask;
    };
    int32_t e_first, e_next;  // of the window's first 256 tokens; of the 256 after the window
    auto load_window = [&]() {
      e_first = load_entry(0);
      e_next = load_entry(1);
    };

    // ---- staging: a wave stages TG groups of eight rows of its token group's tiles ----
    auto scale_token = [](int place) { return score_token(place & 15) + (place >> 4); };
    // offset `which` (0 row, 1 rotary dims, 2 scale) of token t (from t0 on)
    auto where = [&](int which, int t) {
      const uint32_t at = lds_addr(s_where + which * WINDOW + (t & (WINDOW - 1)));
      uint64_t x;
      asm volatile("ds_read_b64 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(x) : "v"(at) : "memory");
      return v.pool + x;
    };
    const uint8_t* src;  // this lane's row (or its rotary dims) of the group at hand
    // load x of tile `it`: the segments of a group's rows, then the next group's; 8-bit: segment 4 is
    // the rotary dims, the last load the scales
    auto direct = [&](auto x, int it) {
      constexpr int SEGS = FP8 ? 5 : 9, y = x / SEGS, seg = x % SEGS;
      const int group = TG * rg + y;
      if constexpr (x == SEGS * TG) {
        load_lds4(where(2, first_token(it) + (lane_now() & 31)), scales_at(it));
      } else {
        if constexpr (seg == 0 || (FP8 && seg == 4)) {
          const int lane = lane_now();
          src = where(seg == 0 ? 0 : 1, first_token(it) + 8 * group + (lane >> 3)) +
                stage_piece(lane, group);
        }
        if constexpr (!FP8) stage_block<72, seg>(tile_at(it), group, src);
        else if constexpr (seg < 4) stage_block<32, seg>(tile_at(it), group, src);
        else stage_block<8, 0>(tile_at(it) + PTile::BYTES, group, src);
      }
    };
    // What is not finite in this wave's rows of a tile, and in its copy of the scales, is cleared.
    auto scrub = [&](int it) {
      const int lane = lane_now();
      int* marks = marks_at(it);
      for (int y = 0; y < TG; ++y) {
        const int r = 8 * (TG * rg + y) + (lane >> 3);
        bool bad = false;
        for (int x = 0; x < (FP8 ? 4 : 8); ++x) {
          u32x4* at = reinterpret_cast<u32x4*>(
                          tile_at(it) + (FP8 ? PTile::row(r) : LTile::row(r)) + x * 1024) +
                      (lane & 7);
          u32x4 p = *at;
          if (FP8 ? clear_bad8(p) : clear_bad(p)) {
            bad = true;
            *at = p;
          }
        }
        if (bad) marks[0] = marks[1 + r] = it + 1;
      }
      if constexpr (FP8) {
        float* at = reinterpret_cast<float*>(scales_at(it)) + (lane & 31);
        if (!(__builtin_fabsf(*at) <= 3.4028235e38f)) {
          marks[0] = marks[1 + scale_token(lane & 31)] = it + 1;
          *at = 0.f;
        }
      }
    };
    // A wait leaves the direct loads of `younger` later tiles in flight.
    auto wait_tiles = [&](int younger) {
      static_for<AHEAD>([&](auto x) {
        if (younger == x) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(x * LOADS) : "memory");
      });
    };
    // the window's entries in place, and tiles [from, to) on their way
    auto begin_entries = [&]() {
      store_entry(0, e_first);
      store_entry(1, e_next);
      e_next = load_entry(2);
      lds_barrier();
    };
    auto begin_tiles = [&](int from, int to) {
      for (int t = from; t < min(to, n_it); ++t)
        static_for<LOADS>([&](auto x) { direct(x, t); });
    };
    // The start of an iteration: tile `it` is stored, and tile it - 1 read, by every wave. `exist`:
    // its tokens.
    auto next_tile = [&](int it) {
      wait_tiles(min(n_it - 1 - it, AHEAD - 1));
      if (partial(tile_base(it))) scrub(it);
      lds_barrier();
      // the window moves on by 256 tokens
      constexpr int EVERY = 256 / (TG * CT);
      if (it % EVERY == 0 && it > 0) {
        store_entry(it / EVERY + 1, e_next);
        e_next = load_entry(it / EVERY + 2);
      }
      // word (tokens / 32) of the masks
      uint32_t exist;
      asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)"
                   : "=v"(exist)
                   : "v"(lds_addr(s_exist) + ((first_token(it) & (WINDOW - 1)) >> 3))
                   : "memory");
      return (uint32_t)__builtin_amdgcn_readfirstlane(exist);
    };

    load_window();
    for (int i = threadIdx.x; i < N_MARKS; i += 256) s_marks[i] = 0;
    if (!v.group_live) {  // no rows: stages only
      begin_entries();
      begin_tiles(0, EARLY);
      lds_barrier();  // the query's two (below)
      lds_barrier();
      for (int attempt = 0;; ++attempt) {
        begin_tiles(attempt == 0 ? EARLY : 0, AHEAD);
        for (int it = 0; it < n_it; ++it) {
          next_tile(it);
          if (it + AHEAD < n_it) static_for<LOADS>([&](auto x) { direct(x, it + AHEAD); });
        }
        lds_barrier();
        if (attempt == 2 || (attempt == 0 && *s_outgrown == 0)) break;
        load_window();
        begin_entries();
      }
      if constexpr (TG > 1) lds_barrier();
      return;
    }

    // ---- Q^T operands, by way of LDS (read in operand order, each load would touch 64 rows): the 32
    // rows of row wave rg as one tile, staged by the wave rg of every token group, then from k-step
    // kk dims 16 kk + 8 half .. +7; 8-bit: two k-steps from each 32 dims, 16 half + 0 .. 7 and 8 ..
    // 15 of them, as K's pieces lie. (A row wave without rows is not waited for: all of the token
    // groups' waves rg have rows, or none.) ----
    bf16x8_t qreg[36];
    {
      uint8_t* tile = s_mem + QUERY + rg * LTile::BYTES;
      const int lane = lane_now();
      const uint16_t* q = a.q + (int64_t)w.q.begin * a.q_stride + (int64_t)h * a.g * 576;
      const int row0 = (w.tile * RG + rg) * 32, last = w.q.n * a.g - 1;
      const bool aligned = (((uintptr_t)q | (uintptr_t)(a.q_stride * 2)) & 15) == 0;
#pragma unroll
      for (int i = 0; i < 4 / TG; ++i) {
        const int y = tg * (4 / TG) + i;
        const int row = min(row0 + 8 * y + (lane >> 3), last);
        const int tok = (int)fastdiv(row, a.div_g);
        const uint8_t* from = reinterpret_cast<const uint8_t*>(q + tok * a.q_stride +
                                                               (row - tok * a.g) * 576) +
                              stage_piece(lane, y);
        if (aligned) {
          stage_rows<72>(tile, y, from);
        } else {
          u32x4* to = reinterpret_cast<u32x4*>(tile + y * LTile::NSEG * 1024) + lane;
#pragma unroll
          for (int seg = 0; seg < 9; ++seg)
            to[seg * 64] = *reinterpret_cast<const any_u32x4*>(from + seg * 128);
        }
      }
      begin_entries();
      begin_tiles(0, EARLY);
      // (loads of entries in between make the wait a little stricter than need be)
      if (n_it > 0 && EARLY) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LOADS) : "memory");
      else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      lds_barrier();  // the query is stored
      const int half = lane >> 5, col = lane & 31, sw = tile_swizzle(col);
      const uint32_t at = lds_addr(tile + LTile::row(col));
      static_for<9>([&](auto i) {  // four reads and their wait in one block
        uint32_t p[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int piece = FP8 && i < 8 ? 4 * (x >> 1) + 2 * half + (x & 1) : 2 * x + half;
          p[x] = at + ((piece ^ sw) << 4);
        }
        u32x4 r0, r1, r2, r3;
        asm volatile(
            "ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%8\n\t"
            "ds_read_b128 %2, %6 offset:%8\n\tds_read_b128 %3, %7 offset:%8\n\t"
            "s_waitcnt lgkmcnt(0)"
            : "=&v"(r0), "=&v"(r1), "=&v"(r2), "=&v"(r3)
            : "v"(p[0]), "v"(p[1]), "v"(p[2]), "v"(p[3]), "n"(i * 1024)
            : "memory");
        qreg[4 * i] = __builtin_bit_cast(bf16x8_t, r0);
        qreg[4 * i + 1] = __builtin_bit_cast(bf16x8_t, r1);
        qreg[4 * i + 2] = __builtin_bit_cast(bf16x8_t, r2);
        qreg[4 * i + 3] = __builtin_bit_cast(bf16x8_t, r3);
      });
      lds_barrier();  // every wave has its query: the other tiles may come
    }

    // The scales of this lane's 16 scores.
    auto read_scales = [&](int it, u32x4 (&sc)[4]) {
      const uint32_t at = lds_addr(scales_at(it)) + 64 * (lane_now() >> 5);
      asm volatile(
          "ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:16\n\tds_read_b128 %2, %4 offset:32\n\t"
          "ds_read_b128 %3, %4 offset:48\n\ts_waitcnt lgkmcnt(0)"
          : "=&v"(sc[0]), "=&v"(sc[1]), "=&v"(sc[2]), "=&v"(sc[3])
          : "v"(at));
    };
    // The loads of the tile AHEAD of the one at hand go out between its MFMAs, SOON of them between
    // the scores', the others between the output's.
    constexpr int SOON = LOADS / 2;
    auto send = [&](auto from, auto to, int it) {
      if constexpr (from < to) {
        if (it < n_it)
          static_for<to - from>([&](auto y) {
            direct(std::integral_constant<int, from + y>{}, it);
          });
      }
    };
    // Scores of tile `it`, those of tokens that a row does not see -inf.
    auto scores = [&](int it, f32x16& sum, u32x4 (&sc)[4]) {
      const uint32_t exist = next_tile(it);
      const int ahead = it + AHEAD;
      const int lane = lane_now(), half = lane >> 5;
      const int kr = mla_row(lane & 31), sw = tile_swizzle(kr);
      const uint32_t krow = lds_addr(tile_at(it)) + (FP8 ? PTile::row(kr) : LTile::row(kr));
      uint32_t ka[4];  // pieces 2 x + half of a segment
#pragma unroll
      for (int x = 0; x < 4; ++x) ka[x] = krow + (((2 * x + half) ^ sw) << 4);
      f32x16 even, odd;  // two chains of MFMAs; 8-bit: the latent and the rotary part
      constexpr int NR = FP8 ? 20 : 36, KD = FP8 ? 3 : 4;  // reads, of which in flight
      u32x4 kb[KD];
      // 8-bit: 16 reads of two k-steps each, then the rotary four
      const uint32_t rope = lds_addr(tile_at(it) + PTile::BYTES) + RTile::row(kr) - krow;
      auto kread = [&](auto x) {
        if constexpr (FP8 && x >= 16) kb[x % KD] = lds_read_b128<0>(ka[x & 3] + rope);
        else kb[x % KD] = lds_read_b128<(x / 4) * 1024>(ka[x & 3]);
      };
      static_for<KD>(kread);
      static_for<NR>([&](auto x) {
        constexpr int later = NR - 1 - x < KD - 1 ? NR - 1 - x : KD - 1;
        if constexpr (!FP8) {
          mfma_qk<later, (x < 2)>((x & 1) ? odd : even, kb[x % KD], qreg[x]);
        } else if constexpr (x < 16) {
          lgkm_wait1<later>(kb[x % KD]);
          const u32x4 k = kb[x % KD];
          mfma_qk<15, (x == 0)>(even, widen(k[0], k[1], 1.f), qreg[2 * x]);
          mfma_qk<15, false>(even, widen(k[2], k[3], 1.f), qreg[2 * x + 1]);
        } else {
          mfma_qk<later, (x == 16)>(odd, kb[x % KD], qreg[16 + x]);
        }
        send(std::integral_constant<int, x * SOON / NR>{},
             std::integral_constant<int, (x + 1) * SOON / NR>{}, ahead);
        if constexpr (x + KD < NR) kread(std::integral_constant<int, x + KD>{});
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (FP8) read_scales(it, sc);
      asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" : "+v"(even), "+v"(odd));
      if constexpr (FP8) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          sum[i] = __builtin_fmaf(even[i], __uint_as_float(sc[i >> 2][i & 3]), odd[i]);
      } else {
        sum = even + odd;
      }
      const int base = tile_base(it);
      if (base + CT > v.w_hi || base < v.w_lo || exist != 0xffffffffu)
        mask_scores(sum, seen_bits(exist, v.row_lo, v.row_hi, base, lane_now() >> 5));
    };

    // Accumulator tile n holds dims 32 n .. of token group 0's output and dims 32 ((n + 8) % 16) ..
    // of group 1's, so that at the end each group finishes its tiles 0..7 and leaves the other group
    // tiles 8..15 with the same code (registers cannot be chosen at run time).
    f32x16 o[16];
    // They are read one by one (arithmetic on them would move all of them to vector registers); the
    // wait states after the last MFMA are given here.
    auto accumulated = []() { asm volatile("s_nop 7\n\ts_nop 7\n\ts_nop 7" ::: "memory"); };
    auto quad = [&](int n, int x) {
      f32x4 r;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y;
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(y) : "a"(o[n][4 * x + i]));
        r[i] = y;
      }
      return r;
    };
    float m_run = -INFINITY, l_run = 0.f;
    begin_tiles(EARLY, AHEAD);
    for (int attempt = 0;; ++attempt) {
#pragma unroll
      for (int n = 0; n < 16; ++n) {
        o[n] = f32x16{};
        asm volatile("" : "+a"(o[n]));
      }
      l_run = 0.f;
      for (int it = 0; it < n_it; ++it) {
        f32x16 s[1];
        u32x4 sc[4];
        scores(it, s[0], sc);
        const int lane = lane_now();
        constexpr int VD = 4;  // MFMA x: tokens 16 (x / 16) .., accumulator tile x % 16
        uint32_t pw[1][8];
        auto weights = [&]() {
          if (__builtin_expect(__ballot(!(__builtin_fabsf(m_run) <= kFused)) != 0, 0)) {
            if (m_run == -INFINITY) m_run = largest<1>(s, a.scale_log2);
            l_run += weights_rounded<1>(pw, s, a.scale_log2, m_run, FP8 ? sc : nullptr);
          } else {
            l_run += weights_of<1>(pw, s, a.scale_log2, m_run, FP8 ? sc : nullptr);
          }
        };
        auto multiply = [&](auto x, const bf16x8_t& vt) {
          constexpr int kb = x / 16, n = x % 16;
          o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              vt, words(pw[0][4 * kb], pw[0][4 * kb + 1], pw[0][4 * kb + 2], pw[0][4 * kb + 3]),
              o[n], 0, 0, 0);
          send(std::integral_constant<int, SOON + x * (LOADS - SOON) / 32>{},
               std::integral_constant<int, SOON + (x + 1) * (LOADS - SOON) / 32>{}, it + AHEAD);
        };
        if constexpr (FP8) {
          // V^T operand by byte transposes: in each 16-lane group, lane 2s + q addresses 8 bytes of
          // the token that is s-th in P's order, 16 kb + 4 (s & 3) + 2 (s >> 2) + half; dims 32 n +
          // 16 (lane / 16 & 1) are piece 2n + (lane / 16 & 1)
          const int sr = (lane & 15) >> 1, vr = 4 * (sr & 3) + 2 * (sr >> 2) + (lane >> 5);
          const int vp = (lane >> 4) & 1;
          uint32_t va[4];  // n & 3
#pragma unroll
          for (int n = 0; n < 4; ++n)
            va[n] = lds_addr(tile_at(it) + PTile::row(vr) + 8 * (lane & 1) +
                             (((2 * n + vp) ^ tile_swizzle(vr)) << 4));
          u32x2 vb[VD];
          const uint32_t turn = tg * 2048;
          auto vread = [&](auto x) {
            constexpr int OFF = (x / 16) * 2 * PTile::NSEG * 1024 + (x % 16) / 4 * 1024;
            vb[x % VD] =
                lds_read_tr8_b64<OFF>(x % 16 < 8 ? va[x & 3] + turn : va[x & 3] - turn);
          };
          static_for<VD>(vread);  // in flight while the weights are worked out
          weights();
          static_for<32>([&](auto x) {
            constexpr int later = 31 - x < VD - 1 ? 31 - x : VD - 1;
            lgkm_wait1<later>(vb[x % VD]);
            const u32x4 vt = widen(vb[x % VD][0], vb[x % VD][1], 1.f);
            if constexpr (x + VD < 32) vread(std::integral_constant<int, x + VD>{});
            multiply(x, __builtin_bit_cast(bf16x8_t, vt));
            __builtin_amdgcn_sched_barrier(0);
          });
        } else {
          // V^T operand by transpose reads, as in Grouped; dims 32 n .. are pieces 4 n .., segment
          // n / 2
          const int vr = 4 * ((lane & 15) >> 2) + (lane >> 5);
          const int vp = 2 * ((lane & 31) >> 4) + ((lane & 3) >> 1);
          uint32_t va[2][2];  // [n & 1][first / second read]
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int y = 0; y < 2; ++y)
              va[n][y] = lds_addr(tile_at(it) + LTile::row(vr + 2 * y) + 8 * (lane & 1) +
                                  (((vp + 4 * n) ^ tile_swizzle(vr + 2 * y)) << 4));
          v4i16 lo[VD], hi[VD];
          const uint32_t turn = tg * 4096;
          auto vread = [&](auto x) {
            constexpr int OFF = (x / 16) * 2 * LTile::NSEG * 1024 + (x % 16) / 2 * 1024;
            const uint32_t t = x % 16 < 8 ? turn : 0u - turn;
            lo[x % VD] = lds_read_tr16_b64<OFF>(va[x & 1][0] + t);
            hi[x % VD] = lds_read_tr16_b64<OFF>(va[x & 1][1] + t);
          };
          static_for<VD>(vread);
          weights();
          static_for<32>([&](auto x) {
            constexpr int later = 31 - x < VD - 1 ? 31 - x : VD - 1;
            lgkm_wait2<2 * later>(lo[x % VD], hi[x % VD]);
            multiply(x, __builtin_bit_cast(bf16x8_t,
                                           __builtin_shufflevector(lo[x % VD], hi[x % VD], 0, 1, 2,
                                                                   3, 4, 5, 6, 7)));
            if constexpr (x + VD < 32) vread(std::integral_constant<int, x + VD>{});
            __builtin_amdgcn_sched_barrier(0);
          });
        }
        // A latent that is not finite, in a tile that only some rows see, was stored as zeros
        // (zero weights would have made NaN of it). It is key and value at once: what a row that
        // sees it becomes is NaN.
        const int base = tile_base(it);
        const int* marks = marks_at(it);
        if (partial(base) && __builtin_amdgcn_readfirstlane(marks[0]) == it + 1) {
          const uint32_t bad = (uint32_t)__ballot(marks[1 + (threadIdx.x & 31)] == it + 1);
          if (bad & seen_bits(0xffffffffu, v.row_lo, v.row_hi, base, 0)) l_run = NAN;
        }
      }
      // some row's weights outgrew its reference? (A sum that is NaN is no reason: it stays so.)
      if (attempt == 0 && __ballot(l_run > (float)(v.t1 - v.t0))) {  // some weigh more than 1: 1 us
        float x = 0.f;
        accumulated();
#pragma unroll
        for (int n = 0; n < 16; ++n)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const f32x4 r = quad(n, y);
#pragma unroll
            for (int i = 0; i < 4; ++i) x = __builtin_fmaf(r[i], 0.f, x);  // NaN if not finite
          }
        if (__ballot(x != 0.f || l_run > kWeightLimit) && (threadIdx.x & 63) == 0) *s_outgrown = 1;
      }
      lds_barrier();  // every wave is past its tiles
      if (attempt == 1 || __builtin_amdgcn_readfirstlane(*s_outgrown) == 0) break;
      auto again = [&]() {
        load_window();
        begin_entries();
        begin_tiles(0, AHEAD);
      };
      again();
      m_run = -INFINITY;
      for (int it = 0; it < n_it; ++it) {
        f32x16 s[1];
        u32x4 sc[4];
        scores(it, s[0], sc);
        send(std::integral_constant<int, SOON>{}, std::integral_constant<int, LOADS>{}, it + AHEAD);
        m_run = fmaxf(m_run, largest<1>(s, a.scale_log2));
      }
      lds_barrier();  // the last tiles are read
      again();
    }
    l_run += __shfl_xor(l_run, 32, 64);

    // ---- results ----
    accumulated();
    const int lane = lane_now(), half = lane >> 5, col = lane & 31;
    float m = m_run, l = l_run, mine = 1.f, other = 0.f;
    f32x4* s_o = reinterpret_cast<f32x4*>(s_mem);  // [wave][8 tiles][4 quads][64 lanes]
    if constexpr (TG > 1) {
      float2* s_ml = reinterpret_cast<float2*>(s_mem + ML);
#pragma unroll
      for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) s_o[(wave * 32 + 4 * n + x) * 64 + lane] = quad(8 + n, x);
      if (half == 0) s_ml[wave * 32 + col] = make_float2(m_run, l_run);
      lds_barrier();
      const float2 g = s_ml[(wave ^ RG) * 32 + col];
      m = fmaxf(m_run, g.x);
      mine = m_run == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m);
      other = g.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(g.x - m);
      // in the groups' order, so that both halves of a row have one sum
      l = tg == 0 ? l_run * mine + g.y * other : g.y * other + l_run * mine;
    }
    const ChunkArgs& b = arguments_again();
    const View u = view_of<32 * RG>(b, w, h, rg, col);  // again, rather than kept
    const float inv = l > 0.f ? 1.f / l : l;
    const int64_t pr = h * b.head_part_rows + w.part_row + (w.split * RG + rg) * 32;
    uint16_t* out =
        b.out + (int64_t)(w.q.begin + u.tok) * b.out_stride + (int64_t)u.head * 512 + 4 * half;
    // token groups: two accumulator tiles at a time, for the branches between them would make each
    // read of the other group's wait for itself
    constexpr int NX = 4 * TG;
    static_for<64 / TG / NX>([&](auto i) {
      f32x4 r[NX];
      if constexpr (TG > 1) {
        const f32x4* theirs = s_o + ((wave ^ RG) * 32 + NX * i) * 64 + lane;
#pragma unroll
        for (int x = 0; x < NX; ++x) r[x] = theirs[x * 64];
      }
#pragma unroll
      for (int x = 0; x < NX; ++x) {
        const f32x4 y = quad((NX * i + x) >> 2, x & 3);
        if constexpr (TG == 1) r[x] = y;
        else r[x] = tg == 0 ? y * mine + r[x] * other : r[x] * other + y * mine;
      }
      const int first = (NX * i + 32 * tg) & 63;  // the quad of dims of the first
      if (w.splits > 1) {
#pragma unroll
        for (int x = 0; x < NX; ++x)
          *reinterpret_cast<f32x4*>(part_quad(b.part_o, pr, 512, first + x, lane)) = r[x];
      } else if (u.live) {
#pragma unroll
        for (int x = 0; x < NX; ++x) store_bf16x4(out + 8 * (first + x), r[x] * inv);
      }
    });
    if (u.live && tg == 0 && half == 0) {
      if (w.splits > 1) b.part_ml[pr + col] = make_float2(m, l);
      else if (b.lse)
        b.lse[(int64_t)(w.q.begin + u.tok) * (b.kv_heads * b.g) + u.head] = natural(m, l);
    }
  }
};

template <bool FP8>
__global__ __launch_bounds__(256, 1) void chunk_latent_kernel(ChunkArgs a) {
  __shared__ __align__(1024) uint8_t s_mem[std::max(Latent<FP8, 1>::LDS, Latent<FP8, 2>::LDS)];
  leave_split_tiles<true>(a);
  const int item = blockIdx.x / a.kv_heads, h = blockIdx.x - item * a.kv_heads;
  Work w;
  if (!find_work<true, false>(a, item, w)) return;
  if (w.groups == 2) Latent<FP8, 2>::run(a, w, h, s_mem);
  else Latent<FP8, 1>::run(a, w, h, s_mem);
}

// Merge of the splits' partial results of 32 rows and 128 dims: SG sets of four waves, each with
// every SG-th split, wave x of a set with quads 4x .. 4x + 3; the sets' sums are joined in LDS in
// their order, and rows written out whole from there.
template <int DV, int SG>
__global__ __launch_bounds__(256 * SG) void chunk_merge_kernel(ChunkArgs a) {
  constexpr int NT = 256 * SG;
  __shared__ float s_w[kMaxSplits][32];  // a split's weight in each row's result
  __shared__ float s_m[32], s_l[32], s_red[SG * 8][32];
  __shared__ f32x4 s_o[SG][16][64];
  const int item = blockIdx.x / a.kv_heads, h = blockIdx.x - item * a.kv_heads;
  if (a.n_split && item >= *a.n_split) return;  // 512 latent row tiles, none split: 5 us, not 17
  Work w;
  if (!find_work<(DV == 512), true>(a, item, w)) return;
  const int group = blockIdx.y / (DV / 128), block = blockIdx.y % (DV / 128);
  const int n_rows = w.q.n * a.g, row0 = (w.tile * w.groups + group) * 32;
  if (group >= w.groups || row0 >= n_rows) return;
  const int live = min(32, n_rows - row0);
  // rows pr + s * step .. + 31 hold split s
  const int64_t pr = h * a.head_part_rows + w.part_row + group * 32, step = w.groups * 32;
  const int t = threadIdx.x, lane = t & 63, row = t & 31, part = t >> 5;
  float m = -INFINITY;
  if (row < live)
    for (int s = part; s < w.splits; s += SG * 8) m = fmaxf(m, a.part_ml[pr + s * step + row].x);
  s_red[part][row] = m;
  __syncthreads();
  if (part == 0) {
#pragma unroll
    for (int i = 1; i < SG * 8; ++i) m = fmaxf(m, s_red[i][row]);
    s_m[row] = m;
  }
  __syncthreads();
  m = s_m[row];
  float l = 0.f;
  if (row < live)
    for (int s = part; s < w.splits; s += SG * 8) {
      const float2 ml = a.part_ml[pr + s * step + row];
      // a split that sees nothing has reference -inf, and sum and output 0
      const float wt = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
      s_w[s][row] = wt;
      l += ml.y * wt;
    }
  s_red[part][row] = l;
  __syncthreads();
  if (part == 0) {
    l = 0.f;
#pragma unroll
    for (int i = 0; i < SG * 8; ++i) l += s_red[i][row];
    s_l[row] = l;
  }
  const int set = t >> 8, q0 = (t >> 6 & 3) * 4;
  f32x4 r[4] = {};
  if (row < live) {
#pragma unroll 4
    for (int s = set; s < w.splits; s += SG) {
      const float wt = s_w[s][row];
#pragma unroll
      for (int x = 0; x < 4; ++x)
        r[x] += *reinterpret_cast<const f32x4*>(
                    part_quad(a.part_o, pr + s * step, DV, block * 16 + q0 + x, lane)) * wt;
    }
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) s_o[set][q0 + x][lane] = r[x];
  __syncthreads();
  // a row's 128 dims by 32 threads, four dims each: dims 4c .. are quad c / 2, half c & 1
  for (int y = t >> 5; y < live; y += NT / 32) {
    const int c = t & 31, at = (c & 1) * 32 + y;
    f32x4 o = s_o[0][c >> 1][at];
#pragma unroll
    for (int i = 1; i < SG; ++i) o += s_o[i][c >> 1][at];
    l = s_l[y];
    const float inv = l > 0.f ? 1.f / l : l;
    const int tok = (int)fastdiv(row0 + y, a.div_g), head = h * a.g + row0 + y - tok * a.g;
    store_bf16x4(a.out + (int64_t)(w.q.begin + tok) * a.out_stride + (int64_t)head * DV +
                     block * 128 + 4 * c,
                 o * inv);
    if (a.lse && c == 0 && block == 0)
      a.lse[(int64_t)(w.q.begin + tok) * (a.kv_heads * a.g) + head] = natural(s_m[y], l);
  }
}

// ---- host ------------------------------------------------------------------------------------

// Every workgroup goes over the chunk starts and lengths of its launch, which is quadratic in its
// requests: more than these are given to several launches, one after the other in the same workspace.
// (16384 decoding requests of 1024 8-bit tokens, one kv head x 4, 13.0 ms in one launch, 4.4 with 4096 in
// each, 2.9 with 2048, 2.2 with 1024, 1.9 with 512, which would divide the work of long requests worse.)
constexpr int32_t kRequestsOfALaunch = 1024;

void launch_chunk(const ChunkArgs& a, const ChunkPlan& p, bool latent, bool fp8, bool merges,
                  hipStream_t s) {
  const dim3 grid((unsigned)(p.items * a.kv_heads));
  if (latent) {
    if (fp8) hipLaunchKernelGGL(chunk_latent_kernel<true>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(chunk_latent_kernel<false>, grid, dim3(256), 0, s, a);
  } else {
    if (fp8) hipLaunchKernelGGL(chunk_grouped_kernel<true>, grid, dim3(512), 0, s, a);
    else hipLaunchKernelGGL(chunk_grouped_kernel<false>, grid, dim3(512), 0, s, a);
  }
  if (!merges) return;
  // few workgroups with many splits each: four times the threads
  const dim3 merge((unsigned)(p.tiles * a.kv_heads), p.groups * (latent ? 4 : 1));
  const bool deep = p.max_splits > 8 && (int64_t)merge.x * merge.y <= kTargetWorkgroups;
  if (latent && deep)
    hipLaunchKernelGGL((chunk_merge_kernel<512, 4>), merge, dim3(1024), 0, s, a);
  else if (latent)
    hipLaunchKernelGGL((chunk_merge_kernel<512, 1>), merge, dim3(256), 0, s, a);
  else if (deep)
    hipLaunchKernelGGL((chunk_merge_kernel<128, 4>), merge, dim3(1024), 0, s, a);
  else
    hipLaunchKernelGGL((chunk_merge_kernel<128, 1>), merge, dim3(256), 0, s, a);
}

}  // namespace
}  // namespace hisparse

extern "C" {

hisparse_status_t hisparse_validate_chunk(const hisparse_kv_desc_t* kv,
                                          const hisparse_chunk_desc_t* c) {
  const hisparse_status_t st = hisparse_validate_kv(kv);
  if (st != HISPARSE_OK) return st;
  if (!c || c->num_requests < 1 || c->kv_heads < 1 || c->q_heads < 1 || c->q_heads > 256 ||
      (int64_t)c->num_requests * c->kv_heads > (1 << 20))
    return HISPARSE_ERR_INVALID_ARG;
  if (c->total_tokens < 0 || c->max_chunk < 1 || c->max_records < 1 ||
      (int64_t)c->max_records * kv->tokens_per_record > (1 << 30))
    return HISPARSE_ERR_INVALID_ARG;
  const int64_t H = (int64_t)c->kv_heads * c->q_heads;
  const int64_t d_v = kv->layout == HISPARSE_KV_GROUPED ? 128 : 512;
  if (c->q_token_stride < 0 || c->out_token_stride < H * d_v || c->table_request_stride < 0 ||
      c->table_head_stride < 0)
    return HISPARSE_ERR_INVALID_ARG;
  if ((c->flags & ~HISPARSE_CHUNK_CAUSAL) != 0 || c->window < 0 ||
      (c->window > 0 && !(c->flags & HISPARSE_CHUNK_CAUSAL)) || c->num_splits < 0 ||
      c->num_splits > 64)
    return HISPARSE_ERR_INVALID_ARG;
  if (!(c->scale > 0.f) || c->scale > 1e6f) return HISPARSE_ERR_INVALID_ARG;
  if (c->total_tokens * H > (int64_t)INT32_MAX) return HISPARSE_ERR_UNSUPPORTED;
  // a launch's threads are counted in 32 bits
  if (hisparse::plan_chunk(*kv, *c).items * c->kv_heads * 512 > (int64_t)UINT32_MAX)
    return HISPARSE_ERR_UNSUPPORTED;
  return HISPARSE_OK;
}

size_t hisparse_chunk_workspace_bytes(const hisparse_kv_desc_t* kv,
                                      const hisparse_chunk_desc_t* c) {
  if (hisparse_validate_chunk(kv, c) != HISPARSE_OK) return 0;
  return hisparse::plan_chunk(*kv, *c).serves_bytes;
}

hisparse_status_t hisparse_chunk_attention(const hisparse_kv_desc_t* kv,
                                           const hisparse_chunk_desc_t* c, const void* d_pool,
                                           const int32_t* d_table, const int32_t* d_chunk_start,
                                           const int32_t* d_kv_len, const void* d_q, void* d_out,
                                           float* d_lse, void* d_workspace,
                                           size_t workspace_bytes, void* stream) {
  using namespace hisparse;
  const hisparse_status_t st = hisparse_validate_chunk(kv, c);
  if (st != HISPARSE_OK) return st;
  if (!d_chunk_start && (int64_t)c->num_requests * c->max_chunk > c->total_tokens)
    return HISPARSE_ERR_INVALID_ARG;
  if (c->total_tokens == 0) return HISPARSE_OK;
  if (!d_pool || !d_table || !d_q || !d_out || (uintptr_t)d_pool % 16 != 0 ||
      (uintptr_t)d_table % 4 != 0 || (uintptr_t)d_chunk_start % 4 != 0 ||
      (uintptr_t)d_kv_len % 4 != 0 || (uintptr_t)d_q % 2 != 0 || (uintptr_t)d_out % 2 != 0 ||
      (uintptr_t)d_lse % 4 != 0)
    return HISPARSE_ERR_INVALID_ARG;
  const bool ragged = d_chunk_start || d_kv_len;
  const int32_t step = ragged ? kRequestsOfALaunch : c->num_requests;
  auto piece_of = [&](int32_t first) {
    hisparse_chunk_desc_t d = *c;
    d.num_requests = std::min(step, c->num_requests - first);
    if (!d_chunk_start) d.total_tokens -= first * c->max_chunk;
    return d;
  };
  for (int64_t first = 0; first < c->num_requests; first += step) {
    const size_t need = plan_chunk(*kv, piece_of((int32_t)first)).workspace_bytes;
    if (need > 0 &&
        (!d_workspace || (uintptr_t)d_workspace % 16 != 0 || workspace_bytes < need))
      return HISPARSE_ERR_INVALID_ARG;
  }
  ChunkArgs a{};
  a.part_o = reinterpret_cast<float*>(d_workspace);
  a.record_stride = kv->record_stride;
  a.head_stride = kv->head_stride;
  a.request_stride = kv->request_stride;
  a.q_stride = c->q_token_stride;
  a.out_stride = c->out_token_stride;
  a.table_request_stride = c->table_request_stride;
  a.table_head_stride = c->table_head_stride;
  a.num_records = kv->num_records;
  a.l = kv_layout(*kv);
  a.causal = (c->flags & HISPARSE_CHUNK_CAUSAL) != 0;
  a.div_g = make_fastdiv((uint32_t)c->q_heads);
  a.scale_log2 = c->scale * 1.4426950408889634f;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const StreamDevice device(s);
  for (int64_t first = 0; first < c->num_requests; first += step) {
    const hisparse_chunk_desc_t d = piece_of((int32_t)first);
    const ChunkPlan p = plan_chunk(*kv, d);
    static_cast<ChunkShape&>(a) = chunk_shape(*kv, d, p, d_chunk_start ? d_chunk_start + first : nullptr,
                                              d_kv_len ? d_kv_len + first : nullptr);
    const int64_t row = d_chunk_start ? 0 : first * c->max_chunk;  // starts count from row 0
    a.pool = reinterpret_cast<const uint8_t*>(d_pool) + first * kv->request_stride;
    a.table = d_table + first * c->table_request_stride;
    a.q = reinterpret_cast<const uint16_t*>(d_q) + row * c->q_token_stride;
    a.out = reinterpret_cast<uint16_t*>(d_out) + row * c->out_token_stride;
    a.lse = d_lse ? d_lse + row * (c->kv_heads * c->q_heads) : nullptr;
    a.part_ml = reinterpret_cast<float2*>(a.part_o + p.part_rows * p.d_v);
    const bool merges = p.max_splits > 1 && (ragged || p.uni_splits > 1);
    a.n_split = merges && p.target && !p.split
                    ? reinterpret_cast<int32_t*>(a.part_ml + p.part_rows) : nullptr;
    launch_chunk(a, p, kv->layout == HISPARSE_KV_LATENT, kv->type == HISPARSE_KV_FP8, merges, s);
  }
  return hipGetLastError() == hipSuccess ? HISPARSE_OK : HISPARSE_ERR_HIP;
}

}  // extern "C"
