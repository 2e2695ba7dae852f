// The cache in 4 bits: where a row lies and what its codes stand for. Shared by the kernels that read and write it.
#pragma once

#include "cast_internal.h"

namespace cast {

// Paging of a cache, for one call. page_size 0: one run of seq_capacity positions per sequence.
struct Paging {
  const int32_t* table;
  int page_size, seq_capacity, num_pages;
  __host__ __device__ long long max_pos() const {
    return page_size == 0 ? seq_capacity : (long long)seq_capacity * page_size;
  }
};

// Positions of a sequence at most: below 2^31 by more than a tile or a round of a kernel, whose last indices may lie past the end.
constexpr long long kMaxPositions = (1ll << 31) - (1ll << 16);

// Page and slot of position `pos` of sequence b (0 <= pos < max_pos); false for a page id out of range.
__device__ __forceinline__ bool find_place(const Paging& g, int b, int pos, int& page, int& slot) {
  if (g.page_size == 0) {
    page = b;
    slot = pos;
    return true;
  }
  const int e = pos / g.page_size;
  page = g.table[(size_t)b * g.seq_capacity + e];
  slot = pos - e * g.page_size;
  return page >= 0 && page < g.num_pages;
}

// Index of a 4-bit row among the rows of its layer: [page][kv-head][slot].
__device__ __forceinline__ long long q4_row(const Paging& g, int Hkv, int h, int page, int slot) {
  return ((long long)page * Hkv + h) * (g.page_size == 0 ? g.seq_capacity : g.page_size) + slot;
}

// (step, low) of a row: two bf16 in a word, widened by a shift.
__device__ __forceinline__ float q4_step(uint32_t range) { return __uint_as_float(range << 16); }
__device__ __forceinline__ float q4_low(uint32_t range) { return __uint_as_float(range & 0xffff0000u); }

// (x & mask) | base in one instruction: written with operators it became two.
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t base) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(x), "r"(mask), "r"(base));
  return r;
}

// Paging with the division by the page size as a product: position / page_size = position * mul >> shift, exact for positions
// below 2^31 (the multiplier is at most page_size - 1 too large in 2^shift, shift = 31 + log2 of the page size, rounded up).
struct FastPaging {
  const int32_t* table;
  int page_size, seq_capacity, num_pages, Hkv, shift;
  uint32_t mul;
};
// False where the rows are too many for 32-bit indices (more than a device's memory holds).
inline bool fast_paging(const Paging& g, int B, int Hkv, FastPaging* f) {
  int lg = 0;
  while (g.page_size > 0 && (1ll << lg) < g.page_size) ++lg;
  *f = {g.table, g.page_size, g.seq_capacity, g.num_pages, Hkv, 31 + lg,
        g.page_size > 0 ? (uint32_t)(((1ull << (31 + lg)) + g.page_size - 1) / g.page_size) : 0u};
  return (long long)(g.page_size > 0 ? g.num_pages : B) * Hkv * (g.page_size > 0 ? g.page_size : g.seq_capacity) <= 0xffffffffll;
}

// Arguments that every q4 call checks alike.
inline cast_status check_q4(const cast_ctx* c, int B, int Hkv, int D, const Paging& g, const void* kc, const void* kr,
                            const void* vc, const void* vr, size_t code_stride, size_t range_stride) {
  if (!c || !kc || !kr || !vc || !vr || B < 1 || Hkv < 1 || g.page_size < 0 || g.seq_capacity < 1 ||
      (g.page_size > 0 && (!g.table || g.num_pages < 1)) || !on_device(c))
    return CAST_ERR_INVALID_ARG;
  if (B > c->cfg.max_batch || g.max_pos() > kMaxPositions) return CAST_ERR_CAPACITY;
  if (D != 64 && D != 128) return CAST_ERR_SHAPE;
  if (((uintptr_t)kc | (uintptr_t)vc | code_stride) & 15 || ((uintptr_t)kr | (uintptr_t)vr | range_stride) & 3)
    return CAST_ERR_SHAPE;
  return CAST_OK;
}

}  // namespace cast
