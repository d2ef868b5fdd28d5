// Device building blocks shared by the attention kernels: MFMA operand types, LDS reads and waits
// that stay out of the compiler's sight, the tile of 32 token rows, softmax weights.
#pragma once

#include <math.h>

#include <type_traits>

#include "internal.h"

namespace hisparse {
namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 32;            // tokens per wave per iteration

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Two softmax weights 2^e0, 2^e1 rounded to bf16 (nearest even, one packed v_cvt_pk_bf16_f32), the
// first in the low half. The exponential is the hardware v_exp_f32: weights below 2^-126 flush to
// zero.
__device__ inline uint32_t weights_bf16x2(float e0, float e1) {
  const f32x2 e = {__builtin_amdgcn_exp2f(e0), __builtin_amdgcn_exp2f(e1)};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(e, bf16x2_t));
}
// s * scale - m with the product rounded first, as the products that references are taken from are:
// 0 for the score that m is.
__device__ inline float over_reference(float s, float scale, float m) {
#pragma clang fp contract(off)
  return s * scale - m;
}
__device__ inline float bf16_to_f32(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
typedef __attribute__((address_space(3))) void lds_void;

// LDS reads that the compiler does not see as memory accesses. In the latent-attention loop the
// next chunk's direct-to-LDS loads are in flight while the current chunk is read from another
// buffer; before a compiler-visible LDS read the compiler would wait for those loads (it cannot
// tell the buffers apart), which takes the load of chunk it+1 out from under the compute of
// chunk it. The caller waits for these reads itself, with s_waitcnt lgkmcnt(N), N = the number
// of its own reads issued after the one it needs: LDS reads complete in order, so any other
// LGKM operation in flight can only lengthen that wait.
__device__ inline uint32_t lds_addr(const void* p) {
  return (uint32_t)(uintptr_t)(const lds_void*)p;
}
template <int OFF>
__device__ __forceinline__ u32x4 lds_read_b128(uint32_t addr) {
  static_assert(OFF >= 0 && OFF < 65536, "immediate offset");
  u32x4 v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
  return v;
}
template <int OFF>
__device__ __forceinline__ v4i16 lds_read_tr16_b64(uint32_t addr) {
  static_assert(OFF >= 0 && OFF < 65536, "immediate offset");
  v4i16 v;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
  return v;
}
// The same for bytes: in each group of 16 lanes, lane 2s + q addresses 8 bytes, columns 8q .., of row
// s; lane t then holds column t of the eight rows.
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
template <int OFF>
__device__ __forceinline__ u32x2 lds_read_tr8_b64(uint32_t addr) {
  static_assert(OFF >= 0 && OFF < 65536, "immediate offset");
  u32x2 v;
  asm volatile("ds_read_b64_tr_b8 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
  return v;
}
// f(0), f(1), ..., f(N - 1) with the index as a compile-time constant (immediate offsets).
template <int N, int I = 0, class F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<N, I + 1>(f);
  }
}
// Wait until at most N LGKM operations are outstanding; a and b are the registers of the reads
// waited for (tied, so that their users stay after the wait).
template <int N>
__device__ __forceinline__ void lgkm_wait2(v4i16& a, v4i16& b) {
  asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(a), "+v"(b) : "n"(N));
}
template <int N>
__device__ __forceinline__ void lgkm_wait2(u32x4& a, u32x4& b) {
  asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(a), "+v"(b) : "n"(N));
}
template <int N, class T>
__device__ __forceinline__ void lgkm_wait1(T& a) {
  asm volatile("s_waitcnt lgkmcnt(%1)" : "+v"(a) : "n"(N));
}

// S^T += K . Q^T for one k-step once the K rows' read (with at most N later LDS reads) is in;
// the first step of a chain (FIRST) starts from zero. The s_nop covers the wait states after a
// just-written operand that the compiler does not see through the assembly.
template <int N, bool FIRST>
__device__ __forceinline__ void mfma_qk(f32x16& acc, const u32x4& k, const bf16x8_t& q) {
  if constexpr (FIRST)
    asm volatile("s_waitcnt lgkmcnt(%3)\n\ts_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0"
                 : "=&v"(acc) : "v"(k), "v"(q), "n"(N));
  else
    asm volatile("s_waitcnt lgkmcnt(%3)\n\ts_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0"
                 : "+v"(acc) : "v"(k), "v"(q), "n"(N));
}

// Wait until at most N direct-to-LDS loads of this wave are outstanding and its LDS writes are
// done, then synchronise the workgroup. (A workgroup fence would also drain the younger
// prefetches, which is exactly what the pipeline must not do.)
template <int N>
__device__ inline void wait_loads_and_barrier() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Every LDS write of this wave (and any LDS read) done, then the workgroup synchronised; loads
// stay in flight.
__device__ inline void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// LDS tile of 32 rows (a chunk's tokens, or 32 query rows) of P 16-byte pieces, P a multiple of
// 8: blocks of 8 rows x 8 pieces (128 bytes of each row), 1 KB each, block (row group, segment)
// at (rg * NSEG + seg) * 1024. One 64-lane direct global->LDS load fills one block, 8 lanes per
// row: each group of 8 lanes reads one 128-byte run of its row, and a lane needs one global
// address per row group, the segment being an immediate offset (an earlier layout of padded rows
// spent 18 vector instructions per load on finding each lane's row, and its loads straddled
// rows: 64 units of 16 heads took 81 us that way, 39 this way). Inside a block, piece p
// of row r sits in 16-byte slot p ^ tile_swizzle(r): any 16 consecutive rows then place the same
// piece in 16 different slots of the 256 bytes that all 64 banks serve (row parity picks the
// half). A transpose read's 16-lane group has rows of one parity, 4 apart, in the 128 bytes of one
// half; the latent kernel's two groups of 32 lanes share it and take each read's banks twice.
// Counted (SQ_LDS_BANK_CONFLICT per wave and chunk): latent 128 of 555 LDS cycles, two for each
// transpose read (padded rows: none of 401); grouped-query 32 of 156 (padded rows: 64 of 151).
template <int P>
struct Tile {
  static_assert(P % 8 == 0, "whole 128-byte segments");
  static constexpr int NSEG = P / 8;
  static constexpr int BYTES = kChunk * P * 16;
  __device__ static int row(int r) { return (r >> 3) * (NSEG * 1024) + (r & 7) * 128; }
};
__device__ inline int tile_swizzle(int r) { return (r >> 1) & 7; }

// Direct global->LDS load of 4 bytes per lane, to `lds` + 4 times the lane.
__device__ __forceinline__ void load_lds4(const uint8_t* src, uint8_t* lds) {
  __builtin_amdgcn_global_load_lds(src, (lds_void*)lds, 4, 0, 0);
}

// Direct global->LDS load of one block, segment SEG of row group rg: `src` is this lane's row (row
// 8 rg + lane / 8) already advanced by the lane's 16-byte piece. The load's immediate offset
// moves both addresses.
template <int P, int SEG>
__device__ __forceinline__ void stage_block(uint8_t* tile, int rg, const uint8_t* src) {
  __builtin_amdgcn_global_load_lds(
      src, (lds_void*)(tile + (rg * Tile<P>::NSEG + SEG) * 1024 - SEG * 128), 16, SEG * 128, 0);
}
template <int P>
__device__ __forceinline__ void stage_rows(uint8_t* tile, int rg, const uint8_t* src) {
  static_for<Tile<P>::NSEG>([&](auto seg) { stage_block<P, seg>(tile, rg, src); });
}
// The 16-byte piece (times 16) that a lane fetches for its row of row group rg.
__device__ inline int stage_piece(int lane, int rg) {
  return ((lane & 7) ^ tile_swizzle(8 * rg + (lane >> 3))) << 4;
}

// Logical row r of a 32-token MFMA tile -> LDS tile row (token) for the latent-attention kernel.
// With r = 16a + 8b + 4h + s the row is 16a + 4s + 2b + h: the P operand of a lane (k-step a,
// half h) then comes straight from its S^T accumulator, and each group of 16 lanes of a V transpose
// read touches rows 4 apart, which the swizzle spreads over the slots of their half (see Tile); the
// 16 K rows that one operand load reads are a permutation of 16 consecutive rows.
__device__ inline int mla_row(int r) {
  return 16 * (r >> 4) + 4 * (r & 3) + 2 * ((r >> 3) & 1) + ((r >> 2) & 1);
}

}  // namespace
}  // namespace hisparse
