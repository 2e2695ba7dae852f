// What the tensor-core kernels over the 4-bit cache share: named barriers, tensor-memory accesses, codes to operands, places of rows,
// and scores to weights where a thread owns a position.
#pragma once

#include "kv_q4.h"
#include "tc_ptx.h"

namespace cast {

__device__ __forceinline__ void named_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ bool named_or(int id, int threads, bool pred) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %3, 0;\n\t"
      "bar.red.or.pred q, %1, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(id), "r"(threads), "r"((uint32_t)pred)
      : "memory");
  return r != 0;
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
// 16 lanes x 8 C columns: lane quad l / 4 of the warp holds columns 8 g + 2 (l % 4) and the next of row l / 4 in r[4 g], r[4 g + 1],
// of row l / 4 + 8 in r[4 g + 2], r[4 g + 3].
template <int C>
__device__ __forceinline__ void tmem_st_quads(uint32_t taddr, const uint32_t (&r)[4 * C]) {
  static_assert(C == 2, "16 columns");
  asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Codes i and i + 4 of a word (its nibbles) as a pair of bf16. 16 + c: the code in the upper mantissa bits of 16, whose step is 1 / 8
// there and 1 with the code three bits up. 128 + c: the code in the lowest bits.
template <int I>
__device__ __forceinline__ uint32_t pair_plus16(uint32_t w) {
  return and_or(I == 0 ? w << 3 : I == 1 ? w >> 1 : I == 2 ? w >> 5 : w >> 9, 0x00780078u, 0x41804180u);
}
template <int I>
__device__ __forceinline__ uint32_t pair_minus8(uint32_t w) {
  const uint32_t x = and_or(w >> (4 * I), 0x000f000fu, 0x43004300u);
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), __floats2bfloat162_rn(136.f, 136.f));  // exact
  return *reinterpret_cast<const uint32_t*>(&d);
}

// Loads that stay where they are written: left to itself the compiler moves a load down to its use, a tile later.
__device__ __forceinline__ int ld_here(const int32_t* p) {
  int r;
  asm volatile("ld.global.nc.b32 %0, [%1];" : "=r"(r) : "l"(p));
  return r;
}
__device__ __forceinline__ void ld_here(uint32_t (&r)[4], const unsigned char* p) {
  asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "l"(p));
}
__device__ __forceinline__ void ld_here(uint32_t (&r)[2], const unsigned char* p) {
  asm volatile("ld.global.nc.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "l"(p));
}

// Pages, rows and pairs are requested tiles ahead of their use: nothing between the request and the use may look at what has
// been requested, so places without a row request another's (position total - 1, page 0) and are told apart when they are used.
// (Branches around the loads made every one of them a wait: 7 us a tile instead of less than one.)
template <bool kPaged>
__device__ __forceinline__ int request_page(const FastPaging& g, int b, int pos, int total) {
  if (!kPaged) return b;
  const int at = min(pos, total - 1);
  return ld_here(g.table + (size_t)b * g.seq_capacity + (uint32_t)(((uint64_t)(uint32_t)at * g.mul) >> g.shift));
}
// Index of the 4-bit row of a position: below 2^32, as the host has checked.
template <bool kPaged>
__device__ __forceinline__ uint32_t row_of(const FastPaging& g, int page, int h, int pos, int total) {
  const uint32_t at = min(pos, total - 1);
  if (!kPaged) return (uint32_t)(page * g.Hkv + h) * (uint32_t)g.seq_capacity + at;
  const uint32_t ps = g.page_size, slot = at - (uint32_t)(((uint64_t)at * g.mul) >> g.shift) * ps;
  return ((uint32_t)((uint32_t)page < (uint32_t)g.num_pages ? page : 0) * (uint32_t)g.Hkv + (uint32_t)h) * ps + slot;
}
// The same for a 16-bit cache, [page][slot][kv-head].
template <bool kPaged>
__device__ __forceinline__ uint32_t dense_row_of(const FastPaging& g, int page, int h, int pos, int total) {
  const uint32_t at = min(pos, total - 1);
  if (!kPaged) return ((uint32_t)page * (uint32_t)g.seq_capacity + at) * (uint32_t)g.Hkv + (uint32_t)h;
  const uint32_t ps = g.page_size, slot = at - (uint32_t)(((uint64_t)at * g.mul) >> g.shift) * ps;
  return ((uint32_t)((uint32_t)page < (uint32_t)g.num_pages ? page : 0) * ps + slot) * (uint32_t)g.Hkv + (uint32_t)h;
}
template <bool kPaged>
__device__ __forceinline__ bool page_ok(const FastPaging& g, int page) {
  return !kPaged || (uint32_t)page < (uint32_t)g.num_pages;
}

// A value per column (32 of them, in every lane), added or maximised over the lanes: lane l returns column l's.
template <bool kMax>
__device__ __forceinline__ float reduce_columns(float (&v)[32]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const bool up = (lane & o) != 0;
      const float mine = up ? v[i + o] : v[i], other = __shfl_xor_sync(0xffffffffu, up ? v[i] : v[i + o], o);
      v[i] = kMax ? fmaxf(mine, other) : mine + other;
    }
  }
  return v[0];
}

// Scores of a position become weights, 2^(ks score + kl sum(q) - reference) per column.
template <int NH>
__device__ __forceinline__ void weights(float (&p)[NH], const float* sq, const float* nm, float ks, float kl) {
#pragma unroll
  for (int c = 0; c < NH; c += 4) {
    const float4 q4 = *reinterpret_cast<const float4*>(sq + c), m4 = *reinterpret_cast<const float4*>(nm + c);
    const float q[4] = {q4.x, q4.y, q4.z, q4.w}, m[4] = {m4.x, m4.y, m4.z, m4.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) p[c + e] = fast_exp2(fmaf(ks, p[c + e], fmaf(kl, q[e], m[e])));
  }
}
// Nothing from the columns that do not see the position.
template <int NH>
__device__ __forceinline__ void mask_weights(float (&p)[NH], uint32_t vm) {
#pragma unroll
  for (int c = 0; c < NH; ++c) p[c] = (vm >> c) & 1u ? p[c] : 0.f;
}
// This thread's NH scores. (The wait is tied to the registers, so that no use of them can be scheduled above it.)
template <int NH>
__device__ __forceinline__ void read_scores(uint32_t taddr, float (&p)[NH]) {
#pragma unroll
  for (int c = 0; c < NH; c += 8) tmem_ld8(taddr + c, reinterpret_cast<uint32_t*>(p) + c);
#define P8(i) "+f"(p[i]), "+f"(p[i + 1]), "+f"(p[i + 2]), "+f"(p[i + 3]), "+f"(p[i + 4]), "+f"(p[i + 5]), "+f"(p[i + 6]), "+f"(p[i + 7])
  static_assert(NH == 8 || NH == 16 || NH == 24 || NH == 32, "whole loads");
  if constexpr (NH == 8) asm volatile("tcgen05.wait::ld.sync.aligned;" : P8(0) : : "memory");
  else if constexpr (NH == 16) asm volatile("tcgen05.wait::ld.sync.aligned;" : P8(0), P8(8) : : "memory");
  else if constexpr (NH == 24) asm volatile("tcgen05.wait::ld.sync.aligned;" : P8(0), P8(8), P8(16) : : "memory");
  else asm volatile("tcgen05.wait::ld.sync.aligned;" : P8(0), P8(8), P8(16), P8(24) : : "memory");
#undef P8
}

}  // namespace cast
