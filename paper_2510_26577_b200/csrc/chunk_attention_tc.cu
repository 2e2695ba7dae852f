// Tensor-core path of cast_chunk_attention and cast_tree_attention_window: bf16, heads of 128 or 64 dims (sm_100a: tcgen05 + TMEM + TMA).
//
// One CTA per SM works its stretch of the line of tiles (chunk_attn.h). A tile is 128 positions, taken in two steps of 64; a block of 128 query rows against a step is two
// products: S = Q K^T (128 x 64 x HD) into tensor memory, then, with the weights P written over the scores as bf16 (64 dims: two terms), O += P V with P from tensor memory and V as
// it lies in the cache (MN-major). Tensor memory holds two lanes of that, each with two buffers of scores and an output, so that a lane's next scores are there
// when its softmax has done with a step. An item's rows decide how the two lanes share it:
//   more than one block of rows (prompts, wide trees): lane 0 and lane 1 take a block each, and the K and V tiles serve both;
//   one block (decoding, small trees): lane 0 takes the first half of every tile and lane 1 the second, each with its own running sums, and they join at the end.
// Twelve warps: four of softmax per lane (a thread a row), one that walks the line, hands the items out through a ring in shared memory and loads Q and K (TMA), one that
// loads V and cleans it, and per lane one that issues its products: a buffer's P V, then the next Q K^T into it, across the items' ends, so loads, products and softmax of the next item run under the output of the last.
// What the single warps do per tile is a chain of dependent instructions and as much a bound as bytes and products are: one issuer for both lanes, loads of 64
// positions, integer divisions by the page size, a load of the page table per tile were 1 us each or more. With every warp walking the line for itself the walk's
// state was spilled, and beside 227 KB of shared memory local memory does not stay in L1: few instructions between two steps took 600 cycles. (Two threads a row, half
// of a step's positions each or every other step, took the softmax no less time, and the issuers more.)
//
// Softmax in one pass: P = 2^(s * scale + r) with a reference r per row that starts at 0 and moves, by a whole power of two, only when a tile's row sum
// reaches 2^60 or all that a row has seen sums to less than 2^-60; the scores are still in tensor memory then, O is scaled there.
//
// What a row does not see must not reach it, and 0 times NaN is NaN: V's warp goes over the tiles that not every row of the item sees whole. It sets the
// V rows nobody sees to zero (they may never have been loaded), looks through those that some rows see, zeroes the ones that hold a NaN or an
// infinity and notes them; the softmax threads that do see such a row add its weighted values to O themselves, in fp32. Scores of hidden
// positions are masked by select.
//
// What it measures (bf16, heads of 128) and what bounds it:
//   two sequences of 32768 + 1000 new tokens, 28/4 heads: 0.95 ms, 1005 TFLOP/s, 62 % of a dense product's rate. A step of both lanes is worth 1020 cycles of softmax (exponentials,
//     masks, sums, rounding: 64 columns of 256 rows) behind a chain of 760 from scores to weights; softmax alone takes 0.75 ms, products and issuers alone 0.70. Issue slots 46 % busy, tensor pipe 44 %;
//   one prompt of 4096, 32/8 heads: 172 us, 800 TFLOP/s: the same, with half of the diagonal's tiles masked, and starts and ends;
//   64 sequences of 512-4096, one token each, 32/8 heads: 128 us, 4.7 TB/s, 72 % of a copy's rate, whatever the pages (16 scattered or in order, 128). Over uniform batches a call is 20 us of
//     start, 2 an item of an SM and 1.47 a tile of an SM, which is memory's rate; with 64 dims 19, 4 and 1.16, where memory would take 0.74;
//   one sequence of 8192, 60 tokens of a tree under a window of 1024: 25 us, a chain: launch and plan 3.8, first scores 2, two to four tiles of 1.1 to 1.5, output 2, the join of an
//     item's partials 6.
#include <math.h>

#include "chunk_attn.h"
#include "tc_ptx.h"

namespace cast {

namespace {

constexpr int kRows = 128;       // query rows of a lane (UMMA M)
constexpr int kTile = 128;       // positions per tile
constexpr int kStep = 64;        // positions per buffer of scores
constexpr int kThreadsC = 384;
constexpr int kItems = 4;          // items handed out ahead
constexpr int kItemReaders = 11;   // warps that read them
constexpr int kRegQ = kRows * 128;   // a 64-dim half of a row block, 128-byte rows
constexpr int kRegKV = kTile * 128;  // a 64-dim half of a tile
constexpr uint32_t kColS = 0, kColO = 256, kLaneCols = 128, kTmemColumns = 512;  // a lane: two buffers of 64 scores; its output

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

template <int HD>
struct Mem {
  static constexpr int kHalves = HD / 64;
  // The weights enter P V as bf16, of 64 dims as two bf16 terms, as in the tree attention without a window. (Two terms are a product and some instructions of the softmax
  // more. 64 dims: decoding of 64 sequences of 512-4096 111 -> 114 us per layer, trees of 6-12 tokens under a window of 2048 114 -> 129, two prompts of 4096, 16/16 heads, 164 -> 179. 128 dims, where they are one term: decoding 127 -> 136,
  // one prompt of 4096 172 -> 190, 2 x 32768 + 1000 948 -> 1097, one tree under a window 26 -> 31, for an error of 0.00166 instead of 0.00235 of an output
  // that is itself rounded to bf16.)
  static constexpr bool kSplitP = HD == 64;
  static constexpr int kStagesK = HD == 64 ? 4 : 2, kStagesV = HD == 64 ? 5 : 3;
  static constexpr int kQ = kHalves * kRegQ, kTileBytes = kHalves * kRegKV;
  static constexpr int kAtQ = 0;                                // two slots
  static constexpr int kAtK = 2 * kQ;
  static constexpr int kAtV = kAtK + kStagesK * kTileBytes;
  static constexpr int kAtMisc = kAtV + kStagesV * kTileBytes;
};

// An item, as it is handed out.
struct Item {
  int end, pair, whole;       // behind the last; two row blocks, one per lane, else the lanes take a half of every tile each; all of the item's tiles are here
  int b, h, T;                // sequence, kv-head, tiles here (0: its rows see nothing, zeros are written)
  int tile0, st, wt;          // index of the first of them; index i is tile i below st, else wt + i - st
  int lo, hi, s_end;          // positions that some row sees: [lo, hi) and [0, s_end)
  int tf, rows;               // first token, query rows
  int no0, no1a, no1b;        // pairs pass over the halves of tiles that no row sees: the first half of tile no0 here, the second of no1a and no1b (-1: of none)
  int hi_min, lo_max, sinks;  // every row sees up to hi_min, as far as the window allows, and from lo_max on or below `sinks`
  int L, n, off;              // of the sequence
  int c_lo, c_hi;             // CTAs that share the item
  __device__ __forceinline__ int pos(int i) const {  // of its tile i here
    const int t = tile0 + i;
    return (t < st ? t : wt + (t - st)) * 128;
  }
};

template <int HD>
struct Misc {
  using M = Mem<HD>;
  uint64_t item_full[kItems], item_free[kItems];
  uint64_t q_full[2], q_free[2];
  uint64_t k_full[M::kStagesK], k_free[M::kStagesK];
  uint64_t v_full[M::kStagesV], v_free[M::kStagesV];
  uint64_t v_raw[M::kStagesV];   // what v_full is to a tile that is cleaned first: V's warp waits for these, in turn, and completes v_full
  uint64_t s_full[2][2], p_full[2][2], pv_done[2][2];  // [lane][buffer]: scores there, weights there, their P V over
  uint32_t tmem;
  int last[3];  // this CTA joins the partials: of lane 0's block, lane 1's, of a single block
  uint32_t bad[M::kStagesV][kTile / 32];  // positions of the V tile that the softmax threads take over
  alignas(16) uint32_t anc[M::kSplitP ? 2 * kRows : 1][4];  // a tree row's mask, where two terms leave no registers for it (spilled, those trees took 139 us per layer)
  float2 row[kRows];                      // what the threads of a row tell one another at an item's end
  Item item[kItems];
};

struct TcArgs {
  int tokens;      // whole tokens of a row block
  int q_tokens;    // tokens of a copy of Q
  int box;         // positions of a copy of K or V (paged)
  int page_shift;  // position / page size = position * page_mul >> page_shift (an integer division is a chain of 130 cycles, and a loader has four a tile)
  uint32_t page_mul;
  float scale_log2;
};

// Whether n positions from pos0 on hold some that some rows of the item see and others do not.
__device__ __forceinline__ bool in_part(const Item& it, int pos0, int n) {
  return (it.hi_min < it.hi && pos0 + n > it.hi_min && pos0 < it.hi) || (pos0 < it.lo_max && pos0 + n > it.lo && pos0 + n > it.sinks);
}
// Whether V's tile has to be looked at: not every row sees all of it.
__device__ __forceinline__ bool to_be_cleaned(const Item& it, int pos0) {
  return pos0 + kTile > it.hi_min || (pos0 < max(it.lo_max, it.lo) && pos0 + kTile > it.s_end);
}

__device__ __forceinline__ uint32_t bits_below(int x) { return x <= 0 ? 0u : x >= 32 ? 0xffffffffu : (1u << x) - 1u; }

// 2^x of a pair without the special-function unit: x = n + f with n the nearest integer (Cody and Waite's reduction; adding 1.5 2^23 rounds and leaves n in the low bits), 2^f
// by a cubic (minimax on [-1/2, 1/2] by Remez's exchange, 7.5e-5 off at most: 2^-13.7, where P is rounded by up to 2^-8), n into the exponent. x below -126
// gives 2^-126. Nothing of it is right for x above 127, infinities or NaN: `check` gets x * 0, which makes the sum no number there, and the step is then done again.
__device__ __forceinline__ void exp2_pair(unsigned long long x, float& p0, float& p1, unsigned long long& check) {
  const unsigned long long magic = pack_f2(12582912.f, 12582912.f), one = pack_f2(1.f, 1.f), minus = pack_f2(-1.f, -1.f);
  check = fma_f2(x, pack_f2(0.f, 0.f), check);
  float x0, x1;
  unpack_f2(x, x0, x1);
  x = pack_f2(fminf(fmaxf(x0, -126.f), 127.f), fminf(fmaxf(x1, -126.f), 127.f));
  const unsigned long long t = add_f2(x, magic), f = fma_f2(fma_f2(t, one, pack_f2(-12582912.f, -12582912.f)), minus, x);
  unsigned long long q = fma_f2(f, pack_f2(0.0551716685f, 0.0551716685f), pack_f2(0.2426111251f, 0.2426111251f));
  q = fma_f2(f, q, pack_f2(0.6932609677f, 0.6932609677f));
  q = fma_f2(f, q, pack_f2(0.9999280572f, 0.9999280572f));
  float t0, t1, q0, q1;
  unpack_f2(t, t0, t1);
  unpack_f2(q, q0, q1);
  p0 = __uint_as_float(__float_as_uint(q0) + (__float_as_uint(t0) << 23));
  p1 = __uint_as_float(__float_as_uint(q1) + (__float_as_uint(t1) << 23));
}

// 32 scores of this thread's row: P = 2^(s * scale + r) as bf16 pairs, the sum of the unrounded weights as a packed pair. Unmasked, kShare of 16 pairs go past the
// special-function unit, which bounds the rest (16 exponentials a cycle and SM where the products of a step take 4 cycles for as many; two layers of a prompt of 4096 353 -> 344 us, calls bound by memory
// or their start the same). kSplit: `lk` receives what the
// rounding of P left over, as bf16 pairs again, and every exponential is the unit's: a weight in the product is right to 2^-17. Where `mine` is false, pk and lk keep what they have.
template <bool kMasked, bool kSplit>
__device__ __forceinline__ void weigh(const uint32_t* s, unsigned long long sc2, unsigned long long ref2, uint32_t seen,
                                      unsigned long long& sum, unsigned long long& check, uint32_t* pk, uint32_t* lk, bool mine = true) {
  constexpr int kShare = kSplit ? 0 : 4;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const unsigned long long x = fma_f2(pack_f2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), sc2, ref2);
    float p0, p1;
    if (!kMasked && e * kShare / 16 != (e + 1) * kShare / 16) {
      exp2_pair(x, p0, p1, check);
    } else {
      unpack_f2(x, p0, p1);
      p0 = fast_exp2(p0);
      p1 = fast_exp2(p1);
    }
    if (kMasked) {
      p0 = ((seen >> (2 * e)) & 1u) ? p0 : 0.f;
      p1 = ((seen >> (2 * e + 1)) & 1u) ? p1 : 0.f;
    }
    sum = add_f2(sum, pack_f2(p0, p1));
    const __nv_bfloat162 h = __floats2bfloat162_rn(p0, p1);
    const uint32_t w = *reinterpret_cast<const uint32_t*>(&h);
    if (kSplit) {
      float r0, r1;
      unpack_f2(add_f2(pack_f2(p0, p1), pack_f2(-__uint_as_float(w << 16), -__uint_as_float(w & 0xffff0000u))), r0, r1);
      const __nv_bfloat162 l = __floats2bfloat162_rn(r0, r1);
      lk[e] = mine ? *reinterpret_cast<const uint32_t*>(&l) : lk[e];
    }
    pk[e] = mine ? w : pk[e];
  }
}

// Whether a phase is over, without waiting (mbar_test may suspend the warp for a while): for warps that have something else to look at.
__device__ __forceinline__ bool mbar_poll(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return __all_sync(0xffffffffu, ok != 0);
}

// Loads from tensor memory with their wait: between the two the registers hold nothing yet, and in a kernel under register pressure the compiler, which does not
// know that, may move or spill them there.
__device__ __forceinline__ void tmem_get1(uint32_t taddr, uint32_t& r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r)
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_get32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_get64(uint32_t taddr, uint32_t (&r)[64]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
      "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
      "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
        "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
        "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
        "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
        "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
      : "r"(taddr)
      : "memory");
}

// Partials: [CTA][2][lane][HD / 4][128 rows] of four columns, so that a warp, a row per thread, writes and reads 512 bytes at a time (row after row, its stores
// went to 32 sectors each and 128 rows took 3.3 us); references and sums [CTA][2][lane][128 rows].
__device__ __forceinline__ size_t part_block(int c, bool first, int lane_of) { return ((size_t)c * 2 + (first ? 1 : 0)) * 2 + lane_of; }

__device__ __forceinline__ void store_row4(__nv_bfloat16* dst, float a, float b, float c, float d) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(a, b), hi = __floats2bfloat162_rn(c, d);
  *reinterpret_cast<uint2*>(dst) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}

// Rows on their way out, in Q's place: 16 bytes of row r, swizzled, so that the threads of a row and then rows in one piece pass without conflicts.
template <int HD>
__device__ __forceinline__ uint4* staged(unsigned char* stage, int r, int chunk) {
  return reinterpret_cast<uint4*>(stage + r * (HD * 2) + ((chunk ^ (r & (HD / 8 - 1))) << 4));
}
template <int HD>
__device__ __forceinline__ void stage_row8(unsigned char* stage, int r, int chunk, float4 a, float4 b) {
  uint2 u[2];
  store_row4(reinterpret_cast<__nv_bfloat16*>(&u[0]), a.x, a.y, a.z, a.w);
  store_row4(reinterpret_cast<__nv_bfloat16*>(&u[1]), b.x, b.y, b.z, b.w);
  *staged<HD>(stage, r, chunk) = make_uint4(u[0].x, u[0].y, u[1].x, u[1].y);
}

// An item's partials of one lane, joined in CTA order (contributors c_lo..c_hi; place 1 of the first, 0 of the others) by `threads` threads: many rows 128 threads to a
// part of the columns, two contributors of eight times four columns in flight, into `stage` (the layout in which rows leave the CTA: straight to their places, eight bytes of
// 32 rows at a time, cost 4 us); few rows four columns a thread, with eight contributors in flight, straight to their places.
constexpr int kFewRows = 16;
template <int HD>
__device__ __noinline__ void merge_rows(const ChunkParams& p, unsigned char* stage, __nv_bfloat16* out0, int t, int threads, int rows, int c_lo, int c_hi, int lane_of) {
  constexpr int C4 = HD / 4;
  const float4* part = reinterpret_cast<const float4*>(p.part_o);
  auto block = [&](int c) { return part_block(c, c == c_lo, lane_of); };
  auto pair_of = [&](int c, int row) { return __ldcg(p.part_ml + block(c) * kRows + row); };
  auto out_of = [&](int row) { return out0 + ((size_t)(row / p.G) * p.Hq + row % p.G) * HD; };
  if (rows > kFewRows) {
    const int r = t & (kRows - 1), cols = C4 * kRows / threads, col0 = t / kRows * cols;
    if (r >= rows) return;
    float top = -INFINITY, l = 0.f;
    for (int c0 = c_lo; c0 <= c_hi; c0 += 8) {
      float2 ml[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) ml[k] = c0 + k <= c_hi ? pair_of(c0 + k, r) : make_float2(-INFINITY, 0.f);
      const float before = top;
#pragma unroll
      for (int k = 0; k < 8; ++k) top = fmaxf(top, ml[k].x);
      if (l != 0.f) l *= exp2f(before - top);
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (ml[k].x > -INFINITY) l = fmaf(exp2f(ml[k].x - top), ml[k].y, l);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
    for (int k = col0; k < col0 + cols; k += 8) {
      float4 acc[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
      for (int c0 = c_lo; c0 <= c_hi; c0 += 2) {
        float4 x[2][8];
        float f[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int c = min(c0 + u, c_hi);
          f[u] = c0 + u <= c_hi ? pair_of(c, r).x : -INFINITY;
#pragma unroll
          for (int e = 0; e < 8; ++e) x[u][e] = __ldcg(part + (block(c) * C4 + k + e) * kRows + r);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (f[u] == -INFINITY) continue;
          const float w = exp2f(f[u] - top);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            acc[e].x = fmaf(w, x[u][e].x, acc[e].x);
            acc[e].y = fmaf(w, x[u][e].y, acc[e].y);
            acc[e].z = fmaf(w, x[u][e].z, acc[e].z);
            acc[e].w = fmaf(w, x[u][e].w, acc[e].w);
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 8; e += 2)
        stage_row8<HD>(stage, r, (k + e) / 2, make_float4(acc[e].x * inv, acc[e].y * inv, acc[e].z * inv, acc[e].w * inv),
                       make_float4(acc[e + 1].x * inv, acc[e + 1].y * inv, acc[e + 1].z * inv, acc[e + 1].w * inv));
    }
    return;
  }
  for (int e = t; e < rows * C4; e += threads) {
    const int row = e / C4, k = e % C4;
    float top = -INFINITY;
#pragma unroll 8
    for (int c = c_lo; c <= c_hi; ++c) top = fmaxf(top, pair_of(c, row).x);
    float l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int c = c_lo; c <= c_hi; ++c) {
      const float2 ml = pair_of(c, row);
      const float4 x = __ldcg(part + (block(c) * C4 + k) * kRows + row);
      const float f = ml.x > -INFINITY ? exp2f(ml.x - top) : 0.f;
      if (f != 0.f) {
        l = fmaf(f, ml.y, l);
        acc.x = fmaf(f, x.x, acc.x);
        acc.y = fmaf(f, x.y, acc.y);
        acc.z = fmaf(f, x.z, acc.z);
        acc.w = fmaf(f, x.w, acc.w);
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    store_row4(out_of(row) + k * 4, acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
  }
}

template <int HD, bool kTree>
__global__ void __launch_bounds__(kThreadsC, 1)
chunk_attn_tc_kernel(const __grid_constant__ ChunkParams p, const __grid_constant__ TcArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v) {
  using M = Mem<HD>;
  extern __shared__ __align__(1024) unsigned char smem[];
  Misc<HD>& ms = *reinterpret_cast<Misc<HD>*>(smem + M::kAtMisc);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_q)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_k)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_v)) : "memory");
    for (int i = 0; i < kItems; ++i) {
      mbar_init(&ms.item_full[i], 1);
      mbar_init(&ms.item_free[i], kItemReaders);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ms.q_full[i], 1);
      mbar_init(&ms.q_free[i], 4);  // (by both lanes' products and softmax)
      for (int j = 0; j < 2; ++j) {
        mbar_init(&ms.s_full[i][j], 1);
        mbar_init(&ms.p_full[i][j], kRows / 32);
        mbar_init(&ms.pv_done[i][j], 1);
      }
    }
    for (int i = 0; i < M::kStagesK; ++i) {
      mbar_init(&ms.k_full[i], 1);
      mbar_init(&ms.k_free[i], 2);  // (by both lanes)
    }
    for (int i = 0; i < M::kStagesV; ++i) {
      mbar_init(&ms.v_full[i], 1);
      mbar_init(&ms.v_free[i], 2);
      mbar_init(&ms.v_raw[i], 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  }
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const bool aligned = (smem_u32(smem) & 1023u) == 0u;  // the swizzled regions need it
  if (!aligned && tid == 0) report(p.st, CAST_ERR_CUDA, 1024);
  if (warp == 10) {
    // Tensor memory is taken behind the wait (a predecessor may hold some until it ends), and the dependents are released behind that.
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ms.tmem)), "n"(kTmemColumns));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }
  if (warp < 8 || warp >= 10) {  // who needs its address
    tc_fence_before();
    asm volatile("bar.sync 12, 320;" ::: "memory");
    tc_fence_after();
  }
  const uint32_t tmem = ms.tmem;
  // The next item of the ring, `taken` of them before; null behind the last, or where a wait has run out. All lanes of a warp call; a warp gives an item back when it
  // has read it for the last time.
  int taken = 0;
  auto take = [&]() -> const Item* {
    if (!mbar_wait(&ms.item_full[taken % kItems], (taken / kItems) & 1)) {
      if (lane == 0) report(p.st, CAST_ERR_TIMEOUT, blockIdx.x);
      return nullptr;
    }
    const Item* it = &ms.item[taken % kItems];
    return it->end ? nullptr : it;
  };
  auto give_back = [&] {
    __syncwarp();
    if (lane == 0) mbar_arrive(&ms.item_free[taken % kItems]);
    ++taken;
  };
  if (warp == 8 || warp == 9) {
    // =========================== loads: Q and K, or V ===========================
    const bool is_v = warp == 9;
    const int stages = is_v ? M::kStagesV : M::kStagesK;
    int stage = 0, round = 0;  // of the next tile
    auto page_at = [&](int pos) { return (int)(((unsigned long long)(uint32_t)pos * a.page_mul) >> a.page_shift); };
    uint64_t* full = is_v ? ms.v_full : ms.k_full;
    uint64_t* free = is_v ? ms.v_free : ms.k_free;
    unsigned char* ring = smem + (is_v ? M::kAtV : M::kAtK);
    const CUtensorMap* map = is_v ? &map_v : &map_k;
    int tile = 0, qc = 0;  // tiles and Q slots so far
    bool ok = true;
    const int per_tile = p.g.page_size == 0 ? 1 : kTile / a.box;  // copies per half
    const int copy = lane / M::kHalves, half = lane % M::kHalves;
    // ---- the line (the warp of K alone)
    ChunkSeq seq[kPerLane] = {}, cur = {};
    long long upto[kPerLane] = {}, units = 0, line_at = 0, line_end = 0, item0 = 0;  // (item0: the item's first unit)
    int line_b = 0, rb = 0, blocks = 0, line_h = 0, made = 0;
    Span sp = {};
    int workers = 0;
    auto seq_of = [&](int b) {
      ChunkSeq s;
      const bool up = b >= 32;
      s.L = __shfl_sync(0xffffffffu, up ? seq[kPerLane - 1].L : seq[0].L, b & 31);
      s.n = __shfl_sync(0xffffffffu, up ? seq[kPerLane - 1].n : seq[0].n, b & 31);
      s.off = __shfl_sync(0xffffffffu, up ? seq[kPerLane - 1].off : seq[0].off, b & 31);
      s.F = (unsigned short)__shfl_sync(0xffffffffu, (int)(up ? seq[kPerLane - 1].F : seq[0].F), b & 31);
      s.d0 = (unsigned short)__shfl_sync(0xffffffffu, (int)(up ? seq[kPerLane - 1].d0 : seq[0].d0), b & 31);
      return s;
    };
    auto upto_of = [&](int b) { return __shfl_sync(0xffffffffu, b >= 32 ? upto[kPerLane - 1] : upto[0], b & 31); };
    auto seq_at = [&](long long u) {  // the sequence that unit u is in
      int b = 0;
#pragma unroll
      for (int j = 0; j < kPerLane; ++j) b += __popc(__ballot_sync(0xffffffffu, upto[j] <= u));
      return b;
    };
    static_assert(kPerLane == 2, "a lane holds two sequences");
    if (!is_v) {
      long long items;
      plan_warp<kTile, kTree>(p, seq, upto, units, items);
      workers = workers_of(p, units, items);
      if (aligned && units > 0 && (int)blockIdx.x < workers) {
        line_at = bound_of(units, workers, blockIdx.x);
        line_end = bound_of(units, workers, blockIdx.x + 1);
        line_b = seq_at(line_at);
        cur = seq_of(line_b);
        blocks = blocks_of(p, cur);
        item0 = line_b > 0 ? upto_of(line_b - 1) : 0;
        for (int rb0 = 0; blocks > 1; rb0 += 32) {  // the row block that the stretch begins in
          const long long own = rb0 + lane < blocks ? (long long)(block_span<kTile, kTree>(p, cur, rb0 + lane).n + kItemCost) * p.Hkv : 0;
          long long sum = own;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += y;
          }
          const int hit = __popc(__ballot_sync(0xffffffffu, sum <= line_at - item0));
          if (hit < 32) {
            rb = rb0 + hit;
            item0 += __shfl_sync(0xffffffffu, sum - own, hit);
            break;
          }
          item0 += __shfl_sync(0xffffffffu, sum, 31);
        }
        sp = block_span<kTile, kTree>(p, cur, rb);
        line_h = (int)mul_div(line_at - item0, 1, sp.n + kItemCost);
        item0 += (long long)line_h * (sp.n + kItemCost);
      }
    }
    // Hands out the next item that has tiles in this stretch (or the end); null where it is the end, or a wait has run out.
    auto make = [&]() -> const Item* {
      if (made >= kItems && !mbar_wait(&ms.item_free[made % kItems], ((made / kItems) - 1) & 1)) {
        ok = false;
        return nullptr;
      }
      Item& x = ms.item[made % kItems];
      bool found = false;
      while (line_at < line_end && !found) {
        const long long t0 = line_at - item0 - kItemCost, t1 = line_end - item0 - kItemCost;
        const int tile0 = t0 < 0 ? 0 : (int)t0, stop = t1 < 0 ? 0 : t1 < sp.n ? (int)t1 : sp.n;
        found = stop > tile0 || (sp.n == 0 && line_at == item0);
        if (found) {
          const bool whole = tile0 == 0 && stop == sp.n;
          const int c_lo = whole ? 0 : owner_of(units, workers, item0 + kItemCost), c_hi = whole ? 0 : owner_of(units, workers, item0 + kItemCost + sp.n - 1);
          if (lane == 0) {
            x.end = 0;
            x.whole = whole;
            x.b = line_b;
            x.h = line_h;
            x.T = stop - tile0;
            x.tile0 = tile0; x.st = sp.st; x.wt = sp.wt; x.lo = sp.lo; x.hi = sp.hi; x.s_end = sp.s_end;
            x.tf = first_token(p, cur, rb);
            const int tl = last_token(p, cur, rb);
            x.rows = (tl + 1 - x.tf) * p.G;
            sp.unseen_halves<kTile>(tile0, stop, x.no0, x.no1a, x.no1b);
            x.pair = x.rows > a.tokens * p.G;
            const long long hm = (long long)cur.L + (kTree ? 0 : x.tf + 1);
            x.hi_min = (int)(hm < sp.hi ? hm : sp.hi);
            const long long lm = p.window > 0 ? (long long)cur.L + (kTree ? CAST_MAX_TREE : tl) - p.window + 1 : 0;
            x.lo_max = (int)(lm < 0 ? 0 : lm < sp.hi ? lm : sp.hi);
            x.sinks = p.window > 0 ? p.sinks : 0;
            x.L = cur.L; x.n = cur.n; x.off = cur.off;
            x.c_lo = c_lo; x.c_hi = c_hi;
          }
        }
        item0 += sp.n + kItemCost;
        line_at = item0;
        if (line_at < line_end && ++line_h == p.Hkv) {
          line_h = 0;
          if (++rb == blocks) {
            rb = 0;
            line_b = seq_at(item0);
            cur = seq_of(line_b);
            blocks = blocks_of(p, cur);
          }
          sp = block_span<kTile, kTree>(p, cur, rb);
        }
      }
      if (lane == 0) {
        if (!found) x.end = 1;
        mbar_arrive(&ms.item_full[made % kItems]);
      }
      __syncwarp();
      ++made;
      return found ? &x : nullptr;
    };
    // V tiles to be cleaned, in turn: how many have been requested and how many are done; lane (number % stages) holds what there is to know about one.
    int to_clean = 0, cleaned = 0;
    int c_pos = 0, c_lo = 0, c_hi = 0, c_end = 0, c_part0 = 0, c_part1 = 0, c_part2 = 0, c_stage = 0;
    auto clean = [&] {
      const int src = cleaned % M::kStagesV;
      const int pos0 = __shfl_sync(0xffffffffu, c_pos, src), lo = __shfl_sync(0xffffffffu, c_lo, src), hi = __shfl_sync(0xffffffffu, c_hi, src);
      const int s_end = __shfl_sync(0xffffffffu, c_end, src), part0 = __shfl_sync(0xffffffffu, c_part0, src), part1 = __shfl_sync(0xffffffffu, c_part1, src);
      const int part2 = __shfl_sync(0xffffffffu, c_part2, src), stage = __shfl_sync(0xffffffffu, c_stage, src);
      unsigned char* v = smem + M::kAtV + stage * M::kTileBytes;
#pragma unroll 1
      for (int j = 0; j < kTile / 32; ++j) {
        const int r = j * 32 + lane, pos = pos0 + r;
        const bool seen = pos < hi && (pos >= lo || pos < s_end);
        bool bad = false;
        if (seen && (pos >= part0 || (pos >= part1 && pos < part2))) {
          uint32_t acc = 0;  // an exponent of all ones carries into the bit above it
#pragma unroll
          for (int c = 0; c < M::kHalves * 8; ++c) {
            const uint4 x = *reinterpret_cast<const uint4*>(v + (c >> 3) * kRegKV + r * 128 + (((c + lane) & 7) << 4));
            acc |= ((x.x & 0x7f807f80u) + 0x00800080u) | ((x.y & 0x7f807f80u) + 0x00800080u) | ((x.z & 0x7f807f80u) + 0x00800080u) |
                   ((x.w & 0x7f807f80u) + 0x00800080u);
          }
          bad = (acc & 0x80008000u) != 0;
        }
        if (!seen || bad) {
#pragma unroll
          for (int c = 0; c < M::kHalves * 8; ++c)
            *reinterpret_cast<uint4*>(v + (c >> 3) * kRegKV + r * 128 + (((c + lane) & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
        }
        const uint32_t word = __ballot_sync(0xffffffffu, bad);
        if (lane == 0) ms.bad[stage][j] = word;
      }
      fence_proxy_async();  // the product reads these rows through the async proxy
      __syncwarp();
      if (lane == 0) mbar_arrive(&ms.v_full[stage]);
      ++cleaned;
    };
    // Waits for a stage (bar null: for nothing), and meanwhile, or until all is done, cleans what has landed.
    auto wait_and_clean = [&](uint64_t* bar, uint32_t parity) {
      const long long start = clock64();
      for (;;) {
        if (cleaned == to_clean) return bar == nullptr || mbar_wait(bar, parity);
        if (bar != nullptr && mbar_poll(bar, parity)) return true;
        if (mbar_poll(&ms.v_raw[cleaned % M::kStagesV], (cleaned / M::kStagesV) & 1)) clean();
        if (__any_sync(0xffffffffu, clock64() - start > kWaitCycles)) return false;
      }
    };
    for (const Item* ip;;) {
      // (V's warp cleans while it waits for an item, too: what hands the next one out may be waiting for that)
      if (is_v) ok = wait_and_clean(&ms.item_full[taken % kItems], (taken / kItems) & 1);
      if (!ok) break;
      ip = is_v ? take() : make();
      if (ip == nullptr) break;
      const Item& it = *ip;
      const int T = it.T, kvh = it.h, seq_b = it.b;
      // Entries of the page table, 32 at a time (lane l holds entry first + l) and the next 32 on their way, so that no tile waits for its own (a load per tile was 0.6 us
      // of a loader's chain). They are judged when they are used: those of unseen positions may hold anything.
      const int32_t* table = p.g.table + (size_t)seq_b * p.g.seq_capacity;
      int first = -0x40000000, now32 = 0, next32 = 0;
      auto entries = [&](int e) { return e + lane < p.g.seq_capacity ? __ldg(table + e + lane) : -1; };
      // the page of this lane's copy of a tile; -1: nothing of it is seen (all lanes call)
      auto page_of = [&](int pos0) {
        const int pos = pos0 + copy * a.box, e0 = page_at(pos0), e = copy < per_tile ? page_at(pos) : e0;
        if (e0 < first || e0 >= first + 64) {
          first = e0;
          now32 = entries(first);
          next32 = entries(first + 32);
        } else if (e0 >= first + 32) {
          first += 32;
          now32 = next32;
          next32 = entries(first + 32);
        }
        const int lo32 = __shfl_sync(0xffffffffu, now32, (e - first) & 31), hi32 = __shfl_sync(0xffffffffu, next32, (e - first) & 31);
        if (copy >= per_tile || pos >= it.hi || (pos + a.box <= it.lo && pos >= it.s_end)) return -1;
        int page = e - first < 32 ? lo32 : hi32;
        if (page < 0 || page >= p.g.num_pages) {
          report(p.st, CAST_ERR_BAD_PAGE, seq_b);
          page = 0;
        }
        return page;
      };
      int page = p.g.page_size && T > 0 ? page_of(it.pos(0)) : 0;
      if (!is_v && T > 0) {
        for (int h = 0; h < (it.pair ? 2 : 1) && ok; ++h, ++qc) {
          const int slot = qc & 1;
          if (qc >= 2) ok = mbar_wait(&ms.q_free[slot], ((qc >> 1) - 1) & 1);
          if (!ok) break;
          if (lane == 0) mbar_expect_tx(&ms.q_full[slot], (uint32_t)(M::kHalves * a.q_tokens * p.G * 128));
          __syncwarp();
          if (lane < M::kHalves)
            tma_load_3d(&map_q, smem + M::kAtQ + slot * M::kQ + lane * kRegQ, &ms.q_full[slot], lane * 64, kvh * p.G, it.off + it.tf + h * a.tokens);
        }
      }
      for (int i = 0; i < T && ok; ++i, ++tile) {
        const int pos0 = it.pos(i);
        const int now = page;
        if (p.g.page_size && i + 1 < T) page = page_of(it.pos(i + 1));
        if (round > 0) {
          const uint32_t parity = (round - 1) & 1;
          ok = is_v ? wait_and_clean(&free[stage], parity) : mbar_wait(&free[stage], parity);
        }
        if (!ok) break;
        unsigned char* dst = ring + stage * M::kTileBytes + half * kRegKV;
        uint64_t* bar = &full[stage];
        if (is_v && to_be_cleaned(it, pos0)) {
          const int at = to_clean++ % M::kStagesV;
          bar = &ms.v_raw[at];
          if (lane == at) {
            c_pos = pos0; c_lo = it.lo; c_hi = it.hi; c_end = it.s_end; c_stage = stage;
            // what some rows see and others do not: from part0 on, and [part1, part2)
            c_part0 = it.hi_min;
            c_part1 = max(it.lo, it.sinks);
            c_part2 = it.lo_max;
          }
        }
        if (p.g.page_size == 0) {
          if (lane == 0) mbar_expect_tx(bar, M::kTileBytes);
          __syncwarp();
          if (lane < M::kHalves) tma_load_3d(map, dst, bar, half * 64, kvh, seq_b * p.g.seq_capacity + pos0);
        } else {
          const int copies = __popc(__ballot_sync(0xffffffffu, now >= 0));
          if (lane == 0) mbar_expect_tx(bar, (uint32_t)(copies * a.box * 128));
          __syncwarp();
          if (now >= 0) {
            const int pos = pos0 + copy * a.box;
            tma_load_4d(map, dst + copy * a.box * 128, bar, half * 64, kvh, pos - page_at(pos) * p.g.page_size, now);
          }
        }
        __syncwarp();
        if (++stage == stages) {
          stage = 0;
          ++round;
        }
      }
      if (is_v) give_back();
      if (!ok) break;
    }
    if (ok && is_v) ok = wait_and_clean(nullptr, 0);
    if (!ok) {  // a wait ran out: the copies in flight land before this CTA's shared memory is given up
      if (lane == 0) report(p.st, CAST_ERR_TIMEOUT, blockIdx.x);
      for (int j = max(0, tile - stages); j < tile; ++j) mbar_wait(&full[j % stages], (j / stages) & 1);
      for (int j = cleaned; j < to_clean; ++j) mbar_wait(&ms.v_raw[j % M::kStagesV], (j / M::kStagesV) & 1);
      for (int j = max(0, qc - 2); j < qc; ++j) mbar_wait(&ms.q_full[j & 1], (j >> 1) & 1);
    }
  } else if (warp >= 10) {
    // =========================== a lane's products ===========================
    const uint32_t idesc_qk = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kStep >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
    const uint32_t idesc_pv = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(HD >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
    // Counts and conditions pass through warp reductions and votes of equal values: the compiler then knows this control flow to be uniform and keeps what the
    // products' operands are made from in uniform registers, where the instructions take them (moved there one by one they are 100 cycles a product).
    const int h = __reduce_max_sync(0xffffffffu, warp - 10);
    const uint32_t tm = __reduce_or_sync(0xffffffffu, tmem) + h * kLaneCols;
    const uint64_t dq = umma_desc(smem_u32(smem + M::kAtQ), 16, 1024);
    const uint64_t dk = umma_desc(smem_u32(smem + M::kAtK), 16, 1024);
    const uint64_t dv = umma_desc(smem_u32(smem + M::kAtV), kRegKV, 1024);
    // Every tile and every slot of Q is waited for and released by both lanes, in order: no phase of a barrier is passed over, and none is mistaken for another.
    int kst = 0, kph = 0, vst = 0, vph = 0, qc = 0, steps = 0;
    int queued = 0, e0 = 0, e1 = 0;  // steps whose P V is to come, the older first: 0 buffer, 1 phase of p_full, 2 V's phase, 3 it releases V, 4 half of the tile, then V's stage
    bool ok = true;
    auto pop = [&] {
      const int buf = e0 & 1, stage = e0 >> 5;
      ok = mbar_wait(&ms.p_full[h][buf], (e0 >> 1) & 1) && mbar_wait(&ms.v_full[stage], (e0 >> 2) & 1);
      if (!ok) return;
      tc_fence_after();
      const uint64_t d = dv + (uint64_t)(stage * (M::kTileBytes >> 4) + ((e0 >> 4) & 1) * (kStep * 128 >> 4));
#pragma unroll
      for (int ks = 0; ks < kStep / 16 * (M::kSplitP ? 2 : 1); ++ks)  // (split: the same values again, under what was left over)
        umma_bf16_ts(tm + kColO, tm + kColS + buf * kStep + ks * 8, d + (uint64_t)(ks % (kStep / 16) * (2048 >> 4)), idesc_pv, 1u);
      umma_commit(&ms.pv_done[h][buf]);
      if (e0 & 8) umma_commit(&ms.v_free[stage]);
      e0 = e1;
      --queued;
    };
    // Waits for a load, and meanwhile works off what is ready.
    auto wait_load = [&](uint64_t* bar, uint32_t parity) {
      const long long start = clock64();
      while (ok) {
        if (queued == 0) {
          ok = mbar_wait(bar, parity);
          return;
        }
        if (mbar_poll(bar, parity)) return;
        if (mbar_poll(&ms.p_full[h][e0 & 1], (e0 >> 1) & 1)) pop();
        else if (__any_sync(0xffffffffu, clock64() - start > kWaitCycles)) ok = false;
      }
    };
    for (const Item* ip; ok;) {
      // (an item that is late does not hold up what is ready)
      wait_load(&ms.item_full[taken % kItems], (taken / kItems) & 1);
      if (!ok || !__any_sync(0xffffffffu, (ip = take()) != nullptr)) break;
      const int T = __reduce_max_sync(0xffffffffu, ip->T), pair = __reduce_max_sync(0xffffffffu, ip->pair);
      const int no0 = __reduce_max_sync(0xffffffffu, ip->no0), no1a = __reduce_max_sync(0xffffffffu, ip->no1a), no1b = __reduce_max_sync(0xffffffffu, ip->no1b);
      give_back();
      if (T == 0) continue;
      for (int j = 0; j <= pair && ok; ++j) wait_load(&ms.q_full[(qc + j) & 1], ((qc + j) >> 1) & 1);
      const uint64_t q = dq + (uint64_t)(((pair ? qc + h : qc) & 1) * (M::kQ >> 4));
      for (int i = 0; i < T && ok; ++i) {
        const int f0 = pair ? i == no0 : h, f1 = pair ? i != no1a && i != no1b : h;
        for (int f = f0; f <= f1 && ok; ++f, ++steps) {
          const int buf = steps & 1;
          if (queued == 2) pop();
          if (ok && f == f0) wait_load(&ms.k_full[kst], kph);
          if (!ok) break;
          tc_fence_after();
          const uint64_t k = dk + (uint64_t)(kst * (M::kTileBytes >> 4) + f * (kStep * 128 >> 4));
#pragma unroll
          for (int ks = 0; ks < HD / 16; ++ks)
            umma_bf16(tm + kColS + buf * kStep, q + (uint64_t)((ks >> 2) * (kRegQ >> 4) + (ks & 3) * 2),
                      k + (uint64_t)((ks >> 2) * (kRegKV >> 4) + (ks & 3) * 2), idesc_qk, ks > 0);
          umma_commit(&ms.s_full[h][buf]);
          const int last = f == f1 ? 1 : 0;
          if (last) umma_commit(&ms.k_free[kst]);
          const int e = buf | (((steps >> 1) & 1) << 1) | (vph << 2) | (last << 3) | (f << 4) | (vst << 5);
          if (queued == 0) e0 = e;
          else e1 = e;
          ++queued;
        }
        if (++kst == M::kStagesK) {
          kst = 0;
          kph ^= 1;
        }
        if (++vst == M::kStagesV) {
          vst = 0;
          vph ^= 1;
        }
      }
      for (int j = 0; j <= pair && ok; ++j) umma_commit(&ms.q_free[(qc + j) & 1]);
      qc += pair + 1;
    }
    while (ok && queued > 0) pop();
    if (!ok && lane == 0) report(p.st, CAST_ERR_TIMEOUT, blockIdx.x);
  } else {
    // =========================== softmax and output ===========================
    // (a warp reaches the 32 tensor-memory lanes of its number modulo four)
    const int h = warp >> 2, quad = warp & 3, r = quad * 32 + lane;
    const uint32_t rowsel = (uint32_t)(quad * 32) << 16;
    const uint32_t t_s0 = tmem + kColS + h * kLaneCols + rowsel, t_o = tmem + kColO + rowsel;  // (t_o: lane 0's output, lane 1's behind it)
    const int lane_id = 1 + h;
    auto sync_lane = [&] { asm volatile("bar.sync %0, 128;" ::"r"(lane_id) : "memory"); };
    auto sync_both = [&] { asm volatile("bar.sync 3, 256;" ::: "memory"); };
    const float sc = a.scale_log2;
    const unsigned long long sc2 = pack_f2(sc, sc);
    const int r_tok = r / p.G, r_head = r - r_tok * p.G;
    int vtile = 0, steps = 0, qc = 0;  // tiles so far, this lane's steps, Q slots
    bool ok = true;
    for (const Item* ip; (ip = take()) != nullptr; give_back()) {
      const Item& it = *ip;
      const int T = it.T;
      const bool pair = it.pair != 0;
      const ChunkSeq s = {it.L, it.n, it.off, 0, 0};
      // the row
      const int tok0 = it.tf + (pair ? h * a.tokens : 0), lane_rows = min(pair ? it.rows - h * a.tokens * p.G : it.rows, a.tokens * p.G);
      const bool row_ok = r < lane_rows, warp_live = quad * 32 < lane_rows;
      const int tok = tok0 + (row_ok ? r_tok : 0);
      if (T == 0) {
        if (row_ok && (pair || h == 0)) {
          __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.out) + (((size_t)it.off + tok) * p.Hq + it.h * p.G + r_head) * HD;
          for (int c = 0; c < HD / 8; ++c) *reinterpret_cast<uint4*>(out + c * 8) = make_uint4(0u, 0u, 0u, 0u);
        }
        continue;
      }
      const int depth = kTree && row_ok ? depth_of(p, s, tok) : 0;
      const RowSight rs = sight_of<kTree>(p, s, tok, depth);
      uint32_t aw[4] = {0u, 0u, 0u, 0u};
      if (kTree && row_ok) {
#pragma unroll
        for (int j = 0; j < 4; ++j) aw[j] = tree_word(p, s, tok, depth, j);
      }
      if (kTree && M::kSplitP) *reinterpret_cast<uint4*>(ms.anc[tid]) = make_uint4(aw[0], aw[1], aw[2], aw[3]);  // (this thread's alone)
      const int hi_all = __reduce_min_sync(0xffffffffu, row_ok ? rs.hi : 0x7fffffff), lo_all = __reduce_max_sync(0xffffffffu, row_ok ? rs.lo : 0);
      float ref = row_ok ? 0.f : -INFINITY, l_run = 0.f;  // a row that is none: its P is 0 for every finite score
      if (warp_live && ok) {
        uint32_t z[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) z[c] = 0u;
#pragma unroll
        for (int c = 0; c < HD; c += 32) tmem_st32(t_o + h * kLaneCols + c, z);
        tmem_wait_st();
      }
      const int no0 = pair ? it.no0 : -1, no1a = pair ? it.no1a : -1, no1b = pair ? it.no1b : -1;
      const int count = pair ? 2 * T - (no0 >= 0) - (no1a >= 0) - (no1b >= 0) : T, hi_plain = hi_all - kStep;
      int ti = 0, step_half = pair ? no0 == 0 : h, pos0 = it.pos(0) + step_half * kStep;
#pragma unroll 1
      for (int i = 0; i < count; ++i, ++steps) {
        const int buf = steps & 1;
        if (ok && !mbar_poll(&ms.s_full[h][buf], (steps >> 1) & 1)) ok = mbar_wait(&ms.s_full[h][buf], (steps >> 1) & 1);
        const int half = step_half, here = pos0, at = ti;
        if (pair && half == 0 && ti != no1a && ti != no1b) {  // the next step's place
          step_half = 1;
          pos0 += kStep;
        } else {
          ++ti;
          if (pair) step_half = ti == no0;
          pos0 = it.pos(ti) + step_half * kStep;
        }
        if (!warp_live) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&ms.p_full[h][buf]);
          continue;
        }
        // The lane's output at rest, for the rare cases that touch it: P V of the step before is over. (That of the one before it is, as these scores are there: no
        // phase is mistaken for an older one.)
        auto settle = [&] {
          if (ok && steps > 0) ok = mbar_wait(&ms.pv_done[h][buf ^ 1], ((steps - 1) >> 1) & 1);
          tc_fence_after();
        };
        const uint32_t t_s = t_s0 + buf * kStep;
        tc_fence_after();
        const bool plain = here <= hi_plain && (here >= lo_all || here + kStep <= rs.sinks);
        auto seen_word = [&](int j) -> uint32_t {  // what the row sees of positions here + 32 j on
          if (plain) return row_ok ? 0xffffffffu : 0u;
          const int base = here + j * 32;
          uint32_t v = bits_below(rs.hi - base) & (~bits_below(rs.lo - base) | bits_below(rs.sinks - base));
          if (kTree) {
            const int st = base - it.L, wi = st >> 5, sh = st & 31;  // (arithmetic shift)
            auto word = [&](int x) -> uint32_t {
              if constexpr (M::kSplitP) return (unsigned)x < 4u ? ms.anc[tid][x] : 0u;
              return x == 0 ? aw[0] : x == 1 ? aw[1] : x == 2 ? aw[2] : x == 3 ? aw[3] : 0u;
            };
            v |= __funnelshift_r(word(wi), word(wi + 1), sh);
          }
          return row_ok ? v : 0u;
        };
        uint32_t pk[32], lk[32];  // (lk: split weights alone)
        float l0, l1;
        {
          unsigned long long sum_a = pack_f2(0.f, 0.f), sum_b = sum_a, check = sum_a;
          const unsigned long long ref2 = pack_f2(ref, ref);
          uint32_t x[64];
          tmem_get64(t_s, x);
          if (plain) {
            weigh<false, M::kSplitP>(x, sc2, ref2, 0u, sum_a, check, pk, lk);
            weigh<false, M::kSplitP>(x + 32, sc2, ref2, 0u, sum_b, check, pk + 16, lk + 16);
          } else {
            weigh<true, M::kSplitP>(x, sc2, ref2, seen_word(0), sum_a, check, pk, lk);
            weigh<true, M::kSplitP>(x + 32, sc2, ref2, seen_word(1), sum_b, check, pk + 16, lk + 16);
          }
          unpack_f2(add_f2(add_f2(sum_a, sum_b), check), l0, l1);
          l0 += l1;
        }
        // far: 2^60 or more (or no number); low: less than 2^-60 so far, and something seen
        const bool far = row_ok && !(l0 < 1.15e18f);
        bool low = row_ok && l_run + l0 < 8.6e-19f;
        if (!plain) low = low && (seen_word(0) | seen_word(1)) != 0u;
        if (__any_sync(0xffffffffu, far || low)) {
          float top = -INFINITY;
#pragma unroll 1
          for (int j = 0; j < 2; ++j) {
            uint32_t x[32];
            tmem_get32(t_s + j * 32, x);
            const uint32_t v = seen_word(j);
#pragma unroll
            for (int c = 0; c < 32; ++c) top = fmaxf(top, ((v >> c) & 1u) ? __uint_as_float(x[c]) : -INFINITY);
          }
          float kf = 0.f;
          if (far || low) {
            const float e = fmaxf(top > -INFINITY ? fmaf(top, sc, ref) : -INFINITY, l_run > 0.f ? log2f(l_run) : -INFINITY);
            if (e > -INFINITY && e < INFINITY) kf = fminf(fmaxf(ceilf(e), -1.0e9f), 1.0e9f);
          }
          const float alpha = l_run > 0.f ? ldexpf(1.f, -(int)kf) : 1.f;
          if (__any_sync(0xffffffffu, alpha != 1.f)) {
            settle();
#pragma unroll 1
            for (int c = 0; c < HD; c += 32) {
              uint32_t x[32];
              tmem_get32(t_o + h * kLaneCols + c, x);
#pragma unroll
              for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * alpha);
              tmem_st32(t_o + h * kLaneCols + c, x);
            }
            tmem_wait_st();
          }
          l_run *= alpha;
          ref -= kf;
          // the step again, for the rows that it is about (the others keep what they have: a row's bits are not its neighbours' business)
          const bool mine = far || kf != 0.f;
          float again = 0.f;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t x[32];
            unsigned long long sum = pack_f2(0.f, 0.f), check = sum;
            tmem_get32(t_s + j * 32, x);
            weigh<true, M::kSplitP>(x, sc2, pack_f2(ref, ref), seen_word(j), sum, check, pk + 16 * j, lk + 16 * j, mine);
            float s0, s1;
            unpack_f2(sum, s0, s1);
            again += s0 + s1;
          }
          l0 = mine ? again : l0;
        }
        if (in_part(it, here, kStep)) {  // (also where this warp's rows see it whole)
          const int stage = (vtile + at) % M::kStagesV;
          if (ok) ok = mbar_wait(&ms.v_full[stage], ((vtile + at) / M::kStagesV) & 1);
          if (ms.bad[stage][half * 2] | ms.bad[stage][half * 2 + 1]) {
            // V rows that hold a NaN or an infinity, found when the tile was cleaned: their weighted values go to the output from here
            settle();
#pragma unroll 1
            for (int j = 0; j < 2; ++j) {
              const uint32_t seen = seen_word(j);
              for (uint32_t left = ms.bad[stage][half * 2 + j]; left; left &= left - 1) {
                const int bit = __ffs(left) - 1;
                if (!__any_sync(0xffffffffu, (seen >> bit) & 1u)) continue;
                uint32_t x, sa[32];
                tmem_get1(t_s + j * 32 + bit, x);
                const float wt = ((seen >> bit) & 1u) ? fast_exp2(fmaf(__uint_as_float(x), sc, ref)) : 0.f;
                int page = 0, slot = 0;
                if (!find_place(p.g, it.b, here + j * 32 + bit, page, slot)) page = 0;
                const size_t place = (((size_t)page * (p.g.page_size == 0 ? p.g.seq_capacity : p.g.page_size) + slot) * p.Hkv + it.h) * HD;
                const __nv_bfloat16* row = reinterpret_cast<const __nv_bfloat16*>(p.v) + place;
#pragma unroll 1
                for (int c = 0; c < HD; c += 32) {
                  tmem_get32(t_o + h * kLaneCols + c, sa);
#pragma unroll
                  for (int e = 0; e < 32; ++e) {
                    const float f = __bfloat162float(row[c + e]);
                    if ((seen >> bit) & 1u) sa[e] = __float_as_uint(fmaf(wt, f, __uint_as_float(sa[e])));
                  }
                  tmem_st32(t_o + h * kLaneCols + c, sa);
                }
                tmem_wait_st();
              }
            }
          }
        }
        tmem_st32(t_s, pk);
        if (M::kSplitP) tmem_st32(t_s + kStep / 2, lk);
        l_run += l0;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&ms.p_full[h][buf]);
      }
      vtile += T;
      // ---- the output, or this CTA's partial
      if (ok) ok = mbar_wait(&ms.pv_done[h][(steps - 1) & 1], ((steps - 1) >> 1) & 1);  // (and with it of all before)
      tc_fence_after();
      if (!ok) l_run = 0.f;  // a wait ran out: nothing of this counts
      const bool whole = it.whole != 0;
      // The row's sum, and what its outputs are multiplied by: the threads of a row tell one another.
      float m = l_run == 0.f ? -INFINITY : -ref, l = l_run, f0 = 1.f, f1 = 0.f;
      if (pair) {
        if (whole) f0 = l == 0.f ? 0.f : 1.f / l;
      } else {  // the lanes join: lane 0 puts the two together, each writes half of the columns
        if (h == 1) ms.row[r] = make_float2(m, l);
        tc_fence_before();
        sync_both();
        tc_fence_after();
        if (h == 0) {
          const float2 o = ms.row[r];
          const float top = fmaxf(m, o.x);
          f0 = m > -INFINITY ? exp2f(m - top) : 0.f;
          f1 = o.x > -INFINITY ? exp2f(o.x - top) : 0.f;
          l = (f0 != 0.f ? f0 * l : 0.f) + (f1 != 0.f ? f1 * o.y : 0.f);
          m = top;
          if (whole) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            f0 *= inv;
            f1 *= inv;
          }
          ms.row[r] = make_float2(f0, f1);
        }
        sync_both();
        const float2 f = ms.row[r];
        f0 = f.x;
        f1 = f.y;
      }
      __nv_bfloat16* const out0 = reinterpret_cast<__nv_bfloat16*>(p.out) + (((size_t)it.off + tok0) * p.Hq + it.h * p.G) * HD;  // the lane's first row
      const int c_lo = it.c_lo, c_hi = it.c_hi;
      const int lane_of = pair ? h : 0;
      const size_t mine_at = part_block(blockIdx.x, (int)blockIdx.x == c_lo, lane_of);
      float4* const part = reinterpret_cast<float4*>(p.part_o) + mine_at * (HD / 4) * kRows + r;
      // Q is done with: its place takes the rows on their way out
      const int slot = (pair ? qc + h : qc) & 1;
      unsigned char* const stage_rows = smem + M::kAtQ + slot * M::kQ;
      constexpr int CH = HD / 8;
      const int cols = pair ? HD : HD / 2, col0 = pair ? 0 : h * (HD / 2);  // this thread's columns
      if (warp_live) {
#pragma unroll 1
        for (int c = col0; c < col0 + cols; c += 32) {
          uint32_t o[32];
          float x[32];
          tmem_get32(t_o + (pair ? h : 0) * kLaneCols + c, o);
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = f0 != 0.f ? __uint_as_float(o[e]) * f0 : 0.f;
          if (!pair) {
            tmem_get32(t_o + kLaneCols + c, o);
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = f1 != 0.f ? fmaf(__uint_as_float(o[e]), f1, x[e]) : x[e];
          }
          if (whole) {
#pragma unroll
            for (int e = 0; e < 32; e += 8)
              stage_row8<HD>(stage_rows, r, (c + e) / 8, make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]), make_float4(x[e + 4], x[e + 5], x[e + 6], x[e + 7]));
          } else if (row_ok) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) __stcg(part + (size_t)((c + e) / 4) * kRows, make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]));
          }
        }
      }
      tc_fence_before();
      if (!whole && row_ok && (pair || h == 0)) __stcg(p.part_ml + mine_at * kRows + r, make_float2(m, l));
      if (pair) sync_lane();
      else sync_both();
      tc_fence_after();
      auto sync_rows = [&] {
        if (pair) sync_lane();
        else sync_both();
      };
      bool staged_all = whole;
      if (!whole) {
        if ((pair || h == 0) && r == 0) {
          // releases this CTA's partial (the barrier made it this thread's to release), acquires those that came earlier
          int32_t* ticket = p.ticket + 2 * c_lo + lane_of;
          int t;
          asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(t) : "l"(ticket) : "memory");
          ms.last[pair ? h : 2] = t == c_hi - c_lo;
          if (t == c_hi - c_lo) *ticket = 0;  // ready for the next launch
        }
        sync_rows();
        if (ms.last[pair ? h : 2]) {  // (both lanes join the partials of a single block)
          merge_rows<HD>(p, stage_rows, out0, pair ? r : tid, pair ? kRows : 2 * kRows, lane_rows, c_lo, c_hi, lane_of);
          staged_all = lane_rows > kFewRows;
          if (staged_all) sync_rows();
        }
      }
      if (staged_all) {
        const int at = pair ? r : tid, by = pair ? kRows : 2 * kRows;
        for (int e = at; e < lane_rows * CH; e += by) {
          const int rr = e / CH, c = e % CH, tk = rr / p.G;
          *reinterpret_cast<uint4*>(out0 + ((size_t)tk * p.Hq + rr - tk * p.G) * HD + c * 8) = *staged<HD>(stage_rows, rr, c);
        }
        fence_proxy_async();  // (the next copy of Q into this place goes by the async proxy)
        sync_lane();
      }
      if (r == 0) {
        mbar_arrive(&ms.q_free[qc & 1]);
        if (pair) mbar_arrive(&ms.q_free[(qc + 1) & 1]);
      }
      qc += pair ? 2 : 1;
    }
    if (!ok && r == 0) report(p.st, CAST_ERR_TIMEOUT, blockIdx.x);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 10) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemColumns));
  }
}

EncodeTiledFn encode_fn() {
  static const EncodeTiledFn fn = [] {
    void* sym = nullptr;
    cudaDriverEntryPointQueryResult res;
    const bool got = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &res) == cudaSuccess && res == cudaDriverEntryPointSuccess;
    return got ? reinterpret_cast<EncodeTiledFn>(sym) : nullptr;
  }();
  return fn;
}

bool make_map(CUtensorMap* map, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
  const EncodeTiledFn enc = encode_fn();
  const cuuint32_t one[4] = {1, 1, 1, 1};
  return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// K or V: {64 dims, one head, the copy's positions, one page}; without pages {64 dims, one head, a tile's positions}.
bool make_cache_map(CUtensorMap* map, const void* base, const ChunkParams& p, int D, int box) {
  const cuuint64_t row = (cuuint64_t)p.Hkv * D * 2;
  if (p.g.page_size == 0) {
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)p.Hkv, (cuuint64_t)p.B * p.g.seq_capacity}, strides[2] = {(cuuint64_t)D * 2, row};
    const cuuint32_t b[3] = {64, 1, kTile};
    return make_map(map, 3, base, dims, strides, b);
  }
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)p.Hkv, (cuuint64_t)p.g.page_size, (cuuint64_t)p.g.num_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)D * 2, row, row * p.g.page_size};
  const cuuint32_t b[4] = {64, 1, (cuuint32_t)box, 1};
  return make_map(map, 4, base, dims, strides, b);
}

template <int HD, bool kTree>
cast_status launch(const ChunkParams& p, const TcArgs& a, int grid, const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t s) {
  constexpr int bytes = Mem<HD>::kAtMisc + (int)sizeof(Misc<HD>);
  static_assert(bytes <= 227 * 1024, "shared memory of a CTA");
  auto kern = chunk_attn_tc_kernel<HD, kTree>;
  CAST_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid, 1, 1);
  cfg.blockDim = dim3(kThreadsC, 1, 1);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // launched while its predecessor drains; waits for it
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kern, p, a, mq, mk, mv) != cudaSuccess) {
    cudaGetLastError();
    return CAST_ERR_CUDA;
  }
  return launch_status();
}

}  // namespace

// Bytes behind the tickets: two partials of two row blocks per CTA.
size_t chunk_attention_tc_workspace(const cast_ctx* c, int D) {
  const size_t grid = c->num_sms < kChunkGrid ? c->num_sms : kChunkGrid;
  return grid * 2 * (2 * kRows) * (D + 2) * sizeof(float);
}

// False where the shape is not this path's: a page that is no multiple of 8 positions (a copy is 8 at least), a group of more heads than a
// row block has rows, scales that turn scores around, more positions than the copies' coordinates count.
bool chunk_attention_tc_launch(cast_ctx* c, ChunkParams& p, int D, void* workspace, cudaStream_t s, cast_status* status) {
  if (p.g.page_size % 8 != 0 || p.G > kRows || !(p.scale > 0.f)) return false;
  if (p.g.page_size == 0 && (long long)p.B * p.g.seq_capacity > kMaxPositions) return false;
  TcArgs a;
  a.tokens = kRows / p.G;
  const int most = p.anc ? p.Nmax : p.rows;
  a.q_tokens = a.tokens < most ? a.tokens : most;
  a.box = kTile;
  while (p.g.page_size % a.box != 0) a.box /= 2;
  FastPaging fast;
  fast_paging(p.g, p.B, p.Hkv, &fast);  // (what it says of 32-bit rows does not matter here: the copies count pages and slots)
  a.page_shift = fast.shift;
  a.page_mul = fast.mul;
  a.scale_log2 = p.scale * 1.4426950408889634f;
  // Pairs of row blocks share their tiles' loads. Where there are fewer of them than SMs, blocks by themselves spread over twice as many, and their lanes take half of the
  // positions each (one sequence of 8192, 60 tokens, 32/8 heads under a window of 1024: 36 -> 26 us).
  const long long pairs = p.Hkv * (p.row_start ? p.rows / (2 * a.tokens) + (long long)p.B : (long long)p.B * ((most + 2 * a.tokens - 1) / (2 * a.tokens)));
  p.block_tokens = pairs < c->num_sms ? a.tokens : 2 * a.tokens;
  p.block_rows = p.block_tokens * p.G;
  p.min_units = kItemCost + 2;
  // No more parts of an item than its join pays for (131 072 positions, one kv-head: 32 tokens 175 -> 95 us, one token 122 -> 73; 8192 positions, 12 tokens, 5
  // kv-heads 38 -> 35, 8 40 -> 36). With so many items that each has few parts anyway the rule changes nothing and costs nothing that shows.
  p.join = 2.f;
  const long long rows = p.row_start ? p.rows : (long long)p.B * p.rows;
  CUtensorMap mq, mk, mv;
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)p.Hq, (cuuint64_t)rows}, strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)p.Hq * D * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)p.G, (cuuint32_t)a.q_tokens};
  if (!make_map(&mq, 3, p.q, dims, strides, box) || !make_cache_map(&mk, p.k, p, D, a.box) || !make_cache_map(&mv, p.v, p, D, a.box)) return false;
  const int grid = c->num_sms < kChunkGrid ? c->num_sms : kChunkGrid;
  p.part_o = reinterpret_cast<float*>(workspace);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + (size_t)grid * 2 * (2 * kRows) * D);
  if (p.anc) *status = D == 64 ? launch<64, true>(p, a, grid, mq, mk, mv, s) : launch<128, true>(p, a, grid, mq, mk, mv, s);
  else *status = D == 64 ? launch<64, false>(p, a, grid, mq, mk, mv, s) : launch<128, false>(p, a, grid, mq, mk, mv, s);
  return true;
}

}  // namespace cast
