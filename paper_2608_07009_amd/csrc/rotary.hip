// Rotary positions (hisparse_rotate_tokens).
//
// Pair (a, b) of token t: (a c - b s, b c + a s), c, s = cos, sin of position * frequency, times the
// magnitude. Angles are taken in turns, in 64 bits: position * (frequency / 2 pi) less the nearest whole
// number is good to 2^-53 of the turns made (2^-23 turns at position 2^31), where a product in fp32 is
// off by whole turns from position 2^24 on. The fraction is at most half a turn and goes on in fp32.
//
// Cosines and sines are the token's, for all heads of all arrays: a workgroup works them out once, in LDS
// ([token][pair]), and turns its tokens' rows with them. HBM-bound, each row read and written once: 16384
// tokens of 32 + 8 heads of 128, 336 MB in 61 us, 5.5 TB/s. A step's rows are a launch: 32 tokens, 3.2 us.
#include <math.h>

#include <algorithm>

#include "fetch_device.h"
#include "tokens.h"

namespace hisparse {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 any_u32x4 __attribute__((aligned(2)));  // rows may start at any element
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

constexpr int kMaxPairs = 128;
constexpr int kThreads = 256;
constexpr int kTableBytes = 16384;  // cosines and sines of a workgroup's tokens

struct RowSet {
  const uint16_t* in;
  uint16_t* out;
  const int64_t* out_rows;
  int64_t num_out_rows, in_token, in_head, out_token, out_head;
  uint32_t items;      // pieces of a token: heads * per_head
  uint32_t per_head;   // pieces of a head
  FastDiv div_per_head;
  int32_t first;
};

struct RotaryArgs {
  const int32_t* positions;
  double turns[kMaxPairs];  // of a pair, a position
  RowSet set[HISPARSE_ROTARY_MAX_ROWS];
  float magnitude, sign;
  int32_t tokens, pairs;
  uint32_t items;           // of a token, all sets
  int32_t group_tokens;     // tokens of a workgroup
  uint32_t slice;           // items of a workgroup (of each of its tokens)
  FastDiv div_slice;
};

__device__ __forceinline__ float low(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float high(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2_t));
}
// The same roundings wherever it is used, so that results do not depend on the pieces taken.
__device__ __forceinline__ f32x2 turned(float a, float b, f32x2 cs) {
#pragma clang fp contract(off)
  const float x = b * cs[1], y = a * cs[1];
  return f32x2{__builtin_fmaf(a, cs[0], -x), __builtin_fmaf(b, cs[0], y)};
}

// Piece `piece` of a head, WIDE: 16 elements at a time. The rotated dims come first: HALF, 8 elements of
// the lower half and 8 of the upper; interleaved, 16 in a row. Then the other dims, 16 in a row (none
// where rows are turned in place).
template <bool HALF>
__device__ __forceinline__ void wide_piece(const RowSet& r, const uint16_t* in, uint16_t* out,
                                           uint32_t piece, int pairs, const f32x2* cs) {
  const uint32_t turning = (uint32_t)pairs >> 3;
  const int second = HALF && piece < turning ? pairs : 8;
  int at;
  if (piece < turning) {
    at = r.first + (int)piece * (HALF ? 8 : 16);
  } else {
    at = (int)(piece - turning) * 16;  // of the other dims
    if (at >= r.first) at += 2 * pairs;
  }
  u32x4 x = *reinterpret_cast<const any_u32x4*>(in + at);
  u32x4 y = *reinterpret_cast<const any_u32x4*>(in + at + second);
  if (piece < turning) {
    cs += piece * 8;
    if (HALF) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 p = turned(low(x[i]), low(y[i]), cs[2 * i]);
        const f32x2 q = turned(high(x[i]), high(y[i]), cs[2 * i + 1]);
        x[i] = pack(p[0], q[0]);
        y[i] = pack(p[1], q[1]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 p = turned(low(x[i]), high(x[i]), cs[i]);
        const f32x2 q = turned(low(y[i]), high(y[i]), cs[4 + i]);
        x[i] = pack(p[0], p[1]);
        y[i] = pack(q[0], q[1]);
      }
    }
  }
  *reinterpret_cast<any_u32x4*>(out + at) = x;
  *reinterpret_cast<any_u32x4*>(out + at + second) = y;
}

// One pair, or one of the other dims: rows whose parts are not whole pieces. (16384 tokens of 40 heads of 126
// dims: 212 us; of 128, in wide pieces, 65.)
template <bool HALF>
__device__ __forceinline__ void narrow_piece(const RowSet& r, const uint16_t* in, uint16_t* out,
                                             uint32_t piece, int pairs, const f32x2* cs) {
  if (piece < (uint32_t)pairs) {
    const int a = r.first + (HALF ? (int)piece : 2 * (int)piece), b = a + (HALF ? pairs : 1);
    const f32x2 p = turned(low(in[a]), low(in[b]), cs[piece]);
    const uint32_t w = pack(p[0], p[1]);
    out[a] = (uint16_t)w;
    out[b] = (uint16_t)(w >> 16);
  } else {
    int at = (int)piece - pairs;
    if (at >= r.first) at += 2 * pairs;
    out[at] = in[at];
  }
}

template <bool HALF, bool WIDE>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotaryArgs a) {
  __shared__ __align__(16) f32x2 s_cs[kTableBytes / sizeof(f32x2)];
  const int token0 = blockIdx.x * a.group_tokens;
  const int n = min(a.group_tokens, a.tokens - token0);
  for (int i = threadIdx.x; i < n * a.pairs; i += kThreads) {
    const int t = i / a.pairs, p = i - t * a.pairs;
    const double turns = (double)a.positions[token0 + t] * a.turns[p];
    float sn, c;
    sincospif(2.f * (float)(turns - rint(turns)), &sn, &c);
    s_cs[i] = f32x2{c * a.magnitude, sn * a.sign};
  }
  __syncthreads();
  const uint32_t item0 = blockIdx.y * a.slice;
  const uint32_t width = min(a.slice, a.items - item0);
  for (uint32_t i = threadIdx.x; i < width * (uint32_t)n; i += kThreads) {
    const uint32_t t = width == a.slice ? fastdiv(i, a.div_slice) : i / width;
    uint32_t item = item0 + i - t * width;
    int set = 0;
    while (item >= a.set[set].items) item -= a.set[set++].items;
    const RowSet& r = a.set[set];
    const uint32_t head = fastdiv(item, r.div_per_head), piece = item - head * r.per_head;
    const int64_t token = token0 + (int)t;
    int64_t row = token;
    if (r.out_rows) {
      row = r.out_rows[token];
      if (row < 0 || row >= r.num_out_rows) continue;
    }
    const uint16_t* in = r.in + token * r.in_token + head * r.in_head;
    uint16_t* out = r.out + row * r.out_token + head * r.out_head;
    if (WIDE) wide_piece<HALF>(r, in, out, piece, a.pairs, s_cs + t * a.pairs);
    else narrow_piece<HALF>(r, in, out, piece, a.pairs, s_cs + t * a.pairs);
  }
}

bool finite(double x) { return x - x == 0.0; }

// Pieces of a token that one launch turns: 65535 workgroups of it, four pieces a thread.
constexpr int kItems = 4 * kThreads;
constexpr int64_t kMostItems = 65535ll * kItems;

// The rows of the first `sets` of a.set, in as many launches as the tokens take (of 2^32 threads).
bool launch_rows(RotaryArgs& a, int sets, const int32_t* positions, int32_t num_tokens, bool wide, bool half,
                 hipStream_t s) {
  // Four items a thread where there is enough to fill the chip, one workgroup of a token otherwise. (16384
  // tokens of 32 + 8 heads of 128: 61.0 us; with one item a thread 71.4, two 61.6, eight 63.5.)
  const int64_t items = a.items;
  a.slice = (uint32_t)std::min<int64_t>(items, kItems);
  a.group_tokens = 1;
  const int most = std::min<int>(kItems / (int)a.slice, kTableBytes / 8 / a.pairs);
  while (a.group_tokens * 2 <= most && (int64_t)num_tokens * items / (a.group_tokens * a.slice) > 2048)
    a.group_tokens *= 2;
  while (a.group_tokens == 1 && a.slice > (uint32_t)kThreads &&
         (int64_t)num_tokens * items / a.slice < 1024)
    a.slice = (a.slice + 1) / 2;
  a.div_slice = make_fastdiv(a.slice);
  const int64_t slices = (items + a.slice - 1) / a.slice;
  const int64_t step = (int64_t)UINT32_MAX / kThreads / slices * a.group_tokens;
  for (int64_t token0 = 0; token0 < num_tokens; token0 += step) {
    a.positions = positions + token0;
    a.tokens = (int32_t)std::min<int64_t>(step, num_tokens - token0);
    const dim3 grid((unsigned)((a.tokens + (int64_t)a.group_tokens - 1) / a.group_tokens), (unsigned)slices);
    if (wide && half) hipLaunchKernelGGL((rotate_kernel<true, true>), grid, dim3(kThreads), 0, s, a);
    else if (wide) hipLaunchKernelGGL((rotate_kernel<false, true>), grid, dim3(kThreads), 0, s, a);
    else if (half) hipLaunchKernelGGL((rotate_kernel<true, false>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((rotate_kernel<false, false>), grid, dim3(kThreads), 0, s, a);
    if (hipGetLastError() != hipSuccess) return false;
    for (int i = 0; i < sets; ++i) {
      RowSet& x = a.set[i];
      x.in += a.tokens * x.in_token;
      if (x.out_rows) x.out_rows += a.tokens;
      else x.out += a.tokens * x.out_token;
    }
  }
  return true;
}

}  // namespace
}  // namespace hisparse

extern "C" {

hisparse_status_t hisparse_validate_rotary(const hisparse_rotary_desc_t* d) {
  using hisparse::finite;
  if (!d || d->dims < 2 || d->dims > 2 * hisparse::kMaxPairs || d->dims % 2 != 0 ||
      d->layout < HISPARSE_ROTARY_HALF || d->layout > HISPARSE_ROTARY_INTERLEAVED ||
      d->scaling < HISPARSE_ROTARY_PLAIN || d->scaling > HISPARSE_ROTARY_BY_PARTS ||
      (d->flags & ~HISPARSE_ROTARY_BACK) != 0)
    return HISPARSE_ERR_INVALID_ARG;
  if (!(d->theta > 0.0) || !finite(d->theta) || !finite(d->magnitude))
    return HISPARSE_ERR_INVALID_ARG;
  if (d->scaling != HISPARSE_ROTARY_PLAIN && (!(d->factor > 0.0) || !finite(d->factor)))
    return HISPARSE_ERR_INVALID_ARG;
  if (d->scaling == HISPARSE_ROTARY_BY_PARTS &&
      (!(d->original_tokens > 0.0) || !finite(d->original_tokens) || !finite(d->low_turns) ||
       !finite(d->high_turns) || !(d->low_turns < d->high_turns)))
    return HISPARSE_ERR_INVALID_ARG;
  return HISPARSE_OK;
}

hisparse_status_t hisparse_rotary_frequencies(const hisparse_rotary_desc_t* d, double* out) {
  const hisparse_status_t st = hisparse_validate_rotary(d);
  if (st != HISPARSE_OK) return st;
  if (!out) return HISPARSE_ERR_INVALID_ARG;
  for (int i = 0; i < d->dims / 2; ++i) {
    double f = pow(d->theta, -2.0 * i / d->dims);
    if (d->scaling == HISPARSE_ROTARY_LINEAR) {
      f /= d->factor;
    } else if (d->scaling == HISPARSE_ROTARY_BY_PARTS) {
      const double r = d->original_tokens * f / (2.0 * M_PI);
      const double s = fmin(fmax((r - d->low_turns) / (d->high_turns - d->low_turns), 0.0), 1.0);
      f *= s + (1.0 - s) / d->factor;
    }
    out[i] = f;
  }
  return HISPARSE_OK;
}

hisparse_status_t hisparse_rotate_tokens(const hisparse_rotary_desc_t* d, int32_t num_tokens,
                                         const int32_t* d_positions,
                                         const hisparse_rotary_rows_t* rows, int32_t num_rows,
                                         void* stream) {
  using namespace hisparse;
  RotaryArgs a{};
  const hisparse_status_t st = hisparse_rotary_frequencies(d, a.turns);
  if (st != HISPARSE_OK) return st;
  if (num_tokens < 0 || num_rows < 1 || num_rows > HISPARSE_ROTARY_MAX_ROWS || !rows)
    return HISPARSE_ERR_INVALID_ARG;
  bool wide = d->dims % 16 == 0;
  int64_t elements = 0;
  for (int i = 0; i < num_rows; ++i) {
    const hisparse_rotary_rows_t& r = rows[i];
    if (r.heads < 1 || r.first < 0 || r.dims > 65536 || r.dims < (int64_t)r.first + d->dims ||
        r.in_token_stride < 0 || r.in_head_stride < 0 || r.out_token_stride < 0 ||
        r.out_head_stride < 0 || (r.heads > 1 && r.out_head_stride < r.dims) ||
        (num_tokens > 1 && r.out_token_stride < r.dims) || (r.d_out_rows && r.num_out_rows < 0))
      return HISPARSE_ERR_INVALID_ARG;
    if ((uintptr_t)r.d_in % 2 != 0 || (uintptr_t)r.d_out % 2 != 0 || (uintptr_t)r.d_out_rows % 8 != 0)
      return HISPARSE_ERR_INVALID_ARG;
    const bool in_place = r.d_in == r.d_out;
    if (num_tokens > 0 &&
        (!r.d_in || !r.d_out ||
         (in_place && (r.d_out_rows || r.in_token_stride != r.out_token_stride ||
                       r.in_head_stride != r.out_head_stride))))
      return HISPARSE_ERR_INVALID_ARG;
    elements += (int64_t)r.heads * r.dims;
    if (!in_place) wide = wide && r.first % 16 == 0 && r.dims % 16 == 0;
  }
  if ((uintptr_t)d_positions % 4 != 0 || (num_tokens > 0 && !d_positions))
    return HISPARSE_ERR_INVALID_ARG;
  if (num_tokens == 0) return HISPARSE_OK;
  // (elements first: at most 4 * 2^47)
  if (elements >= (1ll << 38) || elements > ((1ll << 38) - 1) / num_tokens)
    return HISPARSE_ERR_UNSUPPORTED;
  a.pairs = d->dims / 2;
  a.magnitude = (float)d->magnitude;
  a.sign = d->flags & HISPARSE_ROTARY_BACK ? -a.magnitude : a.magnitude;
  for (int i = 0; i < a.pairs; ++i) a.turns[i] /= 2.0 * M_PI;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const StreamDevice device(s);
  // Arrays, and heads of the last one, until a launch has as many pieces of a token as its grid takes: almost
  // always all of them. (A head has 65536 pieces at most.)
  int32_t head0 = 0;
  for (int i = 0; i < num_rows;) {
    int sets = 0;
    int64_t items = 0;
    while (i < num_rows) {
      const hisparse_rotary_rows_t& r = rows[i];
      const int others = r.d_in == r.d_out ? 0 : r.dims - d->dims;
      const uint32_t per_head = (uint32_t)(wide ? d->dims / 16 + others / 16 : a.pairs + others);
      const int32_t heads = (int32_t)std::min<int64_t>(r.heads - head0, (kMostItems - items) / per_head);
      if (heads == 0) break;
      RowSet& x = a.set[sets++];
      x.in = reinterpret_cast<const uint16_t*>(r.d_in) + head0 * r.in_head_stride;
      x.out = reinterpret_cast<uint16_t*>(r.d_out) + head0 * r.out_head_stride;
      x.out_rows = r.d_out_rows;
      x.num_out_rows = r.num_out_rows;
      x.in_token = r.in_token_stride;
      x.in_head = r.in_head_stride;
      x.out_token = r.out_token_stride;
      x.out_head = r.out_head_stride;
      x.per_head = per_head;
      x.div_per_head = make_fastdiv(per_head);
      x.first = r.first;
      x.items = (uint32_t)heads * per_head;
      items += x.items;
      head0 += heads;
      if (head0 < r.heads) break;
      head0 = 0;
      ++i;
    }
    a.items = (uint32_t)items;
    if (!launch_rows(a, sets, d_positions, num_tokens, wide, d->layout == HISPARSE_ROTARY_HALF, s))
      return HISPARSE_ERR_HIP;
  }
  return HISPARSE_OK;
}

}  // extern "C"
