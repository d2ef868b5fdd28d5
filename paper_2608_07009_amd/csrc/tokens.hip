// K and V rows written into token records, and read back (hisparse_write_tokens,
// hisparse_read_tokens).
//
// 8-bit records hold e4m3 values q and, per token and part, a power of two s = 2^e:
//   e = the least exponent with amax <= 448 2^e (amax over the part's finite elements),
//   q = round(x / s) to nearest even, at most 448;   read back: q s.
// Dividing and multiplying by s only moves exponents, so e4m3's own rounding (half of 2^-3 of the
// value) is the only one, and reading back rounds nothing in bf16 (4 significant bits of 8, exponents
// from 2^-126 on: e >= -117, q >= 2^-9; but for q from 256 on at e = 120, which become infinities).
//
// A group of lanes owns one (token, head): 16 lanes for grouped records (K and V rows of 256
// bytes, 16 bytes of each per lane), 64 for latent ones (1024 bytes and, from 8 lanes, the 128
// rotary bytes). Rows are read and written in whole 16-byte pieces, runs of 128 to 1024 bytes, each
// byte once; the amax is a reduction over the group's lanes in registers. Bound by HBM: 32768 tokens of
// 8 kv heads written to 8-bit pages in 34 us on the device (204 MB), 65536 latent tokens read back in 21
// (118 MB). Both are above the 5.2 TB/s of a 1 GiB copy, for part of what they move stays in the
// last-level cache. Call after call, in TB/s: 32768 tokens of 8 kv heads written 5.1 (16-bit) and 4.7 (8-bit),
// read 5.2 and 4.8; 65536 latent tokens written 4.5 and 4.4, read 4.0 and 3.9. 32 tokens: 2.9 us.
#include "fetch_device.h"
#include "tokens.h"

namespace hisparse {
namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 any_u32x4 __attribute__((aligned(2)));  // rows may start at any element
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

struct TokenArgs {
  uint8_t* pool;
  uint16_t *k, *v;
  const int64_t* slots;  // null: token t is slot t
  int64_t k_stride, v_stride;  // elements
  int64_t num_records, record_stride, head_stride;
  KvLayout l;
  uint32_t items;  // tokens * heads
  int32_t heads;
  FastDiv div_heads;
};

template <int CTRL>
__device__ inline uint32_t max_dpp(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false));
}
// The largest of the 16 lanes of a row, in all of them (rotations by 8, 4, 2, 1).
__device__ inline uint32_t max16(uint32_t x) {
  x = max_dpp<0x128>(x);
  x = max_dpp<0x124>(x);
  x = max_dpp<0x122>(x);
  return max_dpp<0x121>(x);
}
__device__ inline uint32_t max64(uint32_t x) {
  x = max16(x);
  const uint32_t a = __builtin_amdgcn_readlane(x, 0), b = __builtin_amdgcn_readlane(x, 16);
  const uint32_t c = __builtin_amdgcn_readlane(x, 32), d = __builtin_amdgcn_readlane(x, 48);
  return max(max(a, b), max(c, d));
}

// The largest finite magnitude of 8 bf16 values, as float bits.
__device__ inline uint32_t finite_max(u32x4 x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = (x[i] << 16) & 0x7fffffffu, hi = x[i] & 0x7fff0000u;
    m = max(m, lo < 0x7f800000u ? lo : 0u);
    m = max(m, hi < 0x7f800000u ? hi : 0u);
  }
  return m;
}

// e of the scale 2^e for a largest magnitude given as float bits: 448 = 1.75 * 2^8, so the
// exponent less 8, and one more where the significand is above 1.75.
__device__ inline int scale_exponent(uint32_t amax) {
  const int e = (int)((amax + 0x1fffffu) >> 23) - 127 - 8;
  return amax == 0 ? 0 : max(e, -117);
}
__device__ inline float pow2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }

__device__ inline float to_e4m3_range(float x) {
  return x != x ? x : fminf(fmaxf(x, -448.f), 448.f);
}
// 8 bf16 values times 2^-e as e4m3 bytes.
__device__ inline u32x2 quantise8(u32x4 x, int e) {
  const float inv = pow2(-e);
  u32x2 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float f[4];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      f[2 * j] = to_e4m3_range(__uint_as_float(x[2 * i + j] << 16) * inv);
      f[2 * j + 1] = to_e4m3_range(__uint_as_float(x[2 * i + j] & 0xffff0000u) * inv);
    }
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w, true);
    r[i] = (uint32_t)w;
  }
  return r;
}
// 8 e4m3 bytes times the power of two s, in bf16 (exact).
__device__ inline u32x4 dequantise8(u32x2 q, float s) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], false) * s;
    const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], true) * s;
    r[2 * i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(a, bf16x2_t));
    r[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(b, bf16x2_t));
  }
  return r;
}

// The token slot of item i = token * heads + head: its record's address and the token's place in
// it; null for padding.
struct Slot {
  uint8_t* rec;
  int tok;
};
__device__ inline Slot slot_of(const TokenArgs& a, uint32_t t, uint32_t h) {
  const int64_t s = a.slots ? a.slots[t] : (int64_t)t;
  const int64_t r = s >> a.l.tpr_shift;
  if (s < 0 || r >= a.num_records) return Slot{nullptr, 0};
  return Slot{a.pool + r * a.record_stride + (int64_t)h * a.head_stride,
              (int)(s & ((1 << a.l.tpr_shift) - 1))};
}

// LANES 16: grouped records, LANES 64: latent ones.
template <int LANES, bool FP8>
__global__ __launch_bounds__(256) void write_tokens_kernel(TokenArgs a) {
  const int lane = threadIdx.x & (LANES - 1);
  const uint32_t i = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (i >= a.items) return;  // whole groups, and whole waves of 64
  const uint32_t t = fastdiv(i, a.div_heads), h = i - t * a.heads;
  const uint16_t* krow = a.k + (int64_t)t * a.k_stride + (int64_t)h * (LANES * 8);
  const u32x4 k = *reinterpret_cast<const any_u32x4*>(krow + 8 * lane);
  const Slot s = slot_of(a, t, h);
  uint8_t* row = s.rec + (int64_t)s.tok * a.l.row_bytes;
  if constexpr (LANES == 16) {
    const uint16_t* vrow = a.v + (int64_t)t * a.v_stride + (int64_t)h * 128;
    const u32x4 v = *reinterpret_cast<const any_u32x4*>(vrow + 8 * lane);
    if constexpr (FP8) {
      const int ek = scale_exponent(max16(finite_max(k)));
      const int ev = scale_exponent(max16(finite_max(v)));
      if (!s.rec) return;
      reinterpret_cast<u32x2*>(row)[lane] = quantise8(k, ek);
      reinterpret_cast<u32x2*>(row + 128)[lane] = quantise8(v, ev);
      if (lane == 0)
        reinterpret_cast<f32x2*>(s.rec + a.l.scale_offset)[s.tok] = f32x2{pow2(ek), pow2(ev)};
    } else {
      if (!s.rec) return;
      reinterpret_cast<u32x4*>(row)[lane] = k;
      reinterpret_cast<u32x4*>(row + 256)[lane] = v;
    }
  } else {
    const uint16_t* vrow = a.v + (int64_t)t * a.v_stride + (int64_t)h * 64;
    u32x4 v = {};
    if (lane < 8) v = *reinterpret_cast<const any_u32x4*>(vrow + 8 * lane);
    if constexpr (FP8) {
      const int e = scale_exponent(max64(finite_max(k)));
      if (!s.rec) return;
      reinterpret_cast<u32x2*>(row)[lane] = quantise8(k, e);
      if (lane < 8) reinterpret_cast<u32x4*>(s.rec + a.l.rope_offset + s.tok * 128)[lane] = v;
      if (lane == 0) reinterpret_cast<float*>(s.rec + a.l.scale_offset)[s.tok] = pow2(e);
    } else {
      if (!s.rec) return;
      reinterpret_cast<u32x4*>(row)[lane] = k;
      if (lane < 8) reinterpret_cast<u32x4*>(row + 1024)[lane] = v;
    }
  }
}

template <int LANES, bool FP8>
__global__ __launch_bounds__(256) void read_tokens_kernel(TokenArgs a) {
  const int lane = threadIdx.x & (LANES - 1);
  const uint32_t i = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (i >= a.items) return;
  const uint32_t t = fastdiv(i, a.div_heads), h = i - t * a.heads;
  const Slot s = slot_of(a, t, h);
  const uint8_t* row = s.rec + (int64_t)s.tok * a.l.row_bytes;
  u32x4 k = {}, v = {};
  const bool rope = LANES == 64 && lane < 8;
  if (s.rec) {
    if constexpr (FP8) {
      const u32x2 kq = reinterpret_cast<const u32x2*>(row)[lane];
      if constexpr (LANES == 16) {
        const u32x2 vq = reinterpret_cast<const u32x2*>(row + 128)[lane];
        const f32x2 sc = reinterpret_cast<const f32x2*>(s.rec + a.l.scale_offset)[s.tok];
        k = dequantise8(kq, sc[0]);
        v = dequantise8(vq, sc[1]);
      } else {
        const float sc = reinterpret_cast<const float*>(s.rec + a.l.scale_offset)[s.tok];
        if (rope) v = reinterpret_cast<const u32x4*>(s.rec + a.l.rope_offset + s.tok * 128)[lane];
        k = dequantise8(kq, sc);
      }
    } else {
      k = reinterpret_cast<const u32x4*>(row)[lane];
      if (LANES == 16 || rope)
        v = reinterpret_cast<const u32x4*>(row + LANES * 16)[lane];
    }
  }
  uint16_t* krow = a.k + (int64_t)t * a.k_stride + (int64_t)h * (LANES * 8);
  uint16_t* vrow = a.v + (int64_t)t * a.v_stride + (int64_t)h * (LANES == 16 ? 128 : 64);
  *reinterpret_cast<any_u32x4*>(krow + 8 * lane) = k;
  if (LANES == 16 || rope) *reinterpret_cast<any_u32x4*>(vrow + 8 * lane) = v;
}

hisparse_status_t token_args(const hisparse_kv_desc_t* kv, int32_t heads, int32_t tokens,
                             const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                             const int64_t* slots, const void* pool, TokenArgs* a) {
  const hisparse_status_t st = hisparse_validate_kv(kv);
  if (st != HISPARSE_OK) return st;
  if (heads < 1 || tokens < 0 || k_stride < 0 || v_stride < 0) return HISPARSE_ERR_INVALID_ARG;
  if (tokens == 0) return HISPARSE_OK;  // an empty batch's arrays have no address
  if (!k || !v || !pool || (uintptr_t)pool % 16 != 0 || (uintptr_t)k % 2 != 0 ||
      (uintptr_t)v % 2 != 0 || (uintptr_t)slots % 8 != 0)
    return HISPARSE_ERR_INVALID_ARG;
  if (heads > 1 && kv->head_stride < kv->record_bytes) return HISPARSE_ERR_INVALID_ARG;
  // a launch's threads are counted in 32 bits
  const int64_t lanes = kv->layout == HISPARSE_KV_GROUPED ? 16 : 64;
  if ((int64_t)tokens * heads > ((int64_t)UINT32_MAX - 255) / lanes) return HISPARSE_ERR_UNSUPPORTED;
  a->pool = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(pool));
  a->k = const_cast<uint16_t*>(reinterpret_cast<const uint16_t*>(k));
  a->v = const_cast<uint16_t*>(reinterpret_cast<const uint16_t*>(v));
  a->slots = slots;
  a->k_stride = k_stride;
  a->v_stride = v_stride;
  a->num_records = kv->num_records;
  a->record_stride = kv->record_stride;
  a->head_stride = kv->head_stride;
  a->l = kv_layout(*kv);
  a->items = (uint32_t)(tokens * heads);
  a->heads = heads;
  a->div_heads = make_fastdiv((uint32_t)heads);
  return HISPARSE_OK;
}

}  // namespace
}  // namespace hisparse

extern "C" {

int32_t hisparse_kv_record_bytes(int32_t layout, int32_t type, int32_t n) {
  if (n < 1 || n > 4096 || (n & (n - 1)) != 0) return 0;
  if (layout != HISPARSE_KV_GROUPED && layout != HISPARSE_KV_LATENT) return 0;
  const bool grouped = layout == HISPARSE_KV_GROUPED;
  int32_t per = 0;
  if (type == HISPARSE_KV_BF16) per = grouped ? 512 : 1152;
  else if (type == HISPARSE_KV_FP8) per = grouped ? 264 : 644;
  return (n * per + 15) / 16 * 16;
}

hisparse_status_t hisparse_validate_kv(const hisparse_kv_desc_t* d) {
  if (!d) return HISPARSE_ERR_INVALID_ARG;
  const int32_t least = hisparse_kv_record_bytes(d->layout, d->type, d->tokens_per_record);
  if (least == 0) return HISPARSE_ERR_INVALID_ARG;
  if (d->record_bytes < least || d->record_bytes > hisparse::kMaxTokenRecordBytes ||
      d->record_bytes % 16 != 0)
    return HISPARSE_ERR_INVALID_ARG;
  if (d->type == HISPARSE_KV_BF16 && d->record_bytes % (16 * d->tokens_per_record) != 0)
    return HISPARSE_ERR_INVALID_ARG;
  if (d->num_records < 1 || d->num_records > 0x7FFFFFFFLL) return HISPARSE_ERR_INVALID_ARG;
  if (d->record_stride < d->record_bytes || d->record_stride > INT32_MAX ||
      d->record_stride % 16 != 0 || d->head_stride < 0 ||
      d->head_stride % 16 != 0 || d->request_stride < 0 || d->request_stride % 16 != 0)
    return HISPARSE_ERR_INVALID_ARG;
  return HISPARSE_OK;
}

hisparse_status_t hisparse_write_tokens(const hisparse_kv_desc_t* kv, int32_t heads,
                                        int32_t num_tokens, const void* d_k,
                                        int64_t k_token_stride, const void* d_v,
                                        int64_t v_token_stride, const int64_t* d_slots,
                                        void* d_pool, void* stream) {
  using namespace hisparse;
  TokenArgs a{};
  const hisparse_status_t st = token_args(kv, heads, num_tokens, d_k, k_token_stride, d_v,
                                          v_token_stride, d_slots, d_pool, &a);
  if (st != HISPARSE_OK) return st;
  if (num_tokens == 0) return HISPARSE_OK;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const StreamDevice device(s);
  const bool fp8 = kv->type == HISPARSE_KV_FP8;
  if (kv->layout == HISPARSE_KV_GROUPED) {
    const dim3 grid((a.items + 15) / 16);
    if (fp8) hipLaunchKernelGGL((write_tokens_kernel<16, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((write_tokens_kernel<16, false>), grid, dim3(256), 0, s, a);
  } else {
    const dim3 grid((a.items + 3) / 4);
    if (fp8) hipLaunchKernelGGL((write_tokens_kernel<64, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((write_tokens_kernel<64, false>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError() == hipSuccess ? HISPARSE_OK : HISPARSE_ERR_HIP;
}

hisparse_status_t hisparse_read_tokens(const hisparse_kv_desc_t* kv, int32_t heads,
                                       int32_t num_tokens, const void* d_pool,
                                       const int64_t* d_slots, void* d_k, int64_t k_token_stride,
                                       void* d_v, int64_t v_token_stride, void* stream) {
  using namespace hisparse;
  TokenArgs a{};
  const hisparse_status_t st = token_args(kv, heads, num_tokens, d_k, k_token_stride, d_v,
                                          v_token_stride, d_slots, d_pool, &a);
  if (st != HISPARSE_OK) return st;
  const bool grouped = kv->layout == HISPARSE_KV_GROUPED;
  if (num_tokens > 1 && (k_token_stride < (int64_t)heads * (grouped ? 128 : 512) ||
                         v_token_stride < (int64_t)heads * (grouped ? 128 : 64)))
    return HISPARSE_ERR_INVALID_ARG;
  if (num_tokens == 0) return HISPARSE_OK;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const StreamDevice device(s);
  const bool fp8 = kv->type == HISPARSE_KV_FP8;
  if (grouped) {
    const dim3 grid((a.items + 15) / 16);
    if (fp8) hipLaunchKernelGGL((read_tokens_kernel<16, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((read_tokens_kernel<16, false>), grid, dim3(256), 0, s, a);
  } else {
    const dim3 grid((a.items + 3) / 4);
    if (fp8) hipLaunchKernelGGL((read_tokens_kernel<64, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((read_tokens_kernel<64, false>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError() == hipSuccess ? HISPARSE_OK : HISPARSE_ERR_HIP;
}

}  // extern "C"
