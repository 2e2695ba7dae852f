// Tensor-core path of cast_chunk_attention and cast_tree_attention_window: bf16, heads of 128 or 64 dims (sm_100a: tcgen05 + TMEM + TMA).
//
// One CTA per SM works its stretch of the line of tiles (chunk_attn.h). A tile is 128 positions; a block of 128 query rows against it is
// two products of 128 x 128 x HD: S = Q K^T into tensor memory, then, with the weights P written over the scores as bf16, O += P V with P
// from tensor memory and V as it lies in the cache (MN-major). Tensor memory holds two lanes of that, scores 128 columns and output HD each. An
// item's rows decide how the two lanes share it:
//   more than one block of rows (prompts, wide trees): lane 0 and lane 1 take a block each, and the K and V tiles serve both;
//   one block (decoding, small trees): the lanes take every other tile of the same rows, each with its own running sums, and join
//   them at the end - the tensor pipe works for one lane while the other one's exponentials run, where one lane alone would alternate.
// Twelve warps: four of softmax per lane (a thread a row), one that loads Q and K (TMA), one that loads V, one that issues the products, one
// that cleans V tiles. The issuer goes tile by tile: P V of a lane's tile before, then its next Q K^T, across the items' ends, so loads, products and
// softmax of the next item run under the output of the last.
//
// Softmax in one pass: P = 2^(s * scale + r) with a reference r per row that starts at 0 and moves, by a whole power of two, only when a tile's row sum
// reaches 2^60 or all that a row has seen sums to less than 2^-60; the scores are still in tensor memory then, O is scaled there.
//
// What a row does not see must not reach it, and 0 times NaN is NaN: the cleaner goes over the tiles that not every row of the item sees whole. It sets the
// V rows nobody sees to zero (they may never have been loaded), looks through those that some rows see, zeroes the ones that hold a NaN or an
// infinity and notes them; the softmax threads that do see such a row add its weighted values to O themselves, in fp32. Scores of hidden
// positions are masked by select.
#include <math.h>

#include "chunk_attn.h"
#include "tc_ptx.h"

namespace cast {

namespace {

constexpr int kRows = 128;       // query rows of a lane (UMMA M)
constexpr int kTile = 128;       // positions per tile
constexpr int kThreadsC = 384;
constexpr int kRegQ = kRows * 128;   // a 64-dim half of a row block, 128-byte rows
constexpr int kRegKV = kTile * 128;  // a 64-dim half of a tile
constexpr uint32_t kColS = 0, kColO = 256, kLaneCols = 128, kTmemColumns = 512;

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

template <int HD>
struct Mem {
  static constexpr int kHalves = HD / 64;
  static constexpr int kStagesK = HD == 64 ? 5 : 3, kStagesV = HD == 64 ? 4 : 2;
  static constexpr int kQ = kHalves * kRegQ, kTileBytes = kHalves * kRegKV;
  static constexpr int kAtQ = 0;                                // two slots
  static constexpr int kAtK = 2 * kQ;
  static constexpr int kAtV = kAtK + kStagesK * kTileBytes;
  static constexpr int kAtMisc = kAtV + kStagesV * kTileBytes;
};

template <int HD>
struct Misc {
  using M = Mem<HD>;
  uint64_t q_full[2], q_free[2];
  uint64_t k_full[M::kStagesK], k_free[M::kStagesK];
  uint64_t v_full[M::kStagesV], v_free[M::kStagesV];
  uint64_t v_raw[M::kStagesV];   // what v_full is to a tile that is cleaned first: the cleaner waits for these, in turn, and completes v_full
  uint64_t s_full[2], p_full[2], o_full[2];
  uint32_t tmem;
  int last[2];
  uint32_t bad[M::kStagesV][4];  // positions of the V tile that the softmax threads take over
  float2 ml[kRows];              // lane 1's references and sums, where lane 0 joins both
  ChunkPlan plan;
};

struct TcArgs {
  int tokens;      // whole tokens of a row block
  int q_tokens;    // tokens of a copy of Q
  int box;         // positions of a copy of K or V (paged)
  float scale_log2;
};

// The item in work, as every warp sees it.
struct Item {
  bool pair;        // two row blocks, one per lane; else the lanes take every other tile
  int rows;         // query rows of the item
  int tf;           // its first token
  int hi_min;       // every row sees up to here (that is not hidden by the window)
  long long lo_max; // the window of every row has begun here
};
template <bool kTree>
__device__ __forceinline__ Item item_of(const ChunkParams& p, const ChunkSeq& s, const ChunkWalk& w) {
  const int r0 = w.rb * p.block_rows, total = (s.n - s.F) * p.G;
  Item x;
  x.rows = min(p.block_rows, total - r0);
  x.pair = x.rows * 2 > p.block_rows;
  x.tf = s.F + r0 / p.G;
  const int tl = s.F + (r0 + x.rows - 1) / p.G;
  const long long hm = (long long)s.L + (kTree ? 0 : x.tf + 1);
  x.hi_min = (int)(hm < w.span.hi ? hm : w.span.hi);
  x.lo_max = p.window > 0 ? (long long)s.L + (kTree ? CAST_MAX_TREE : tl) - p.window + 1 : 0;
  return x;
}
// Positions that some rows of the item see and others do not.
__device__ __forceinline__ bool seen_in_part(const ChunkParams& p, const Span& sp, const Item& it, int pos) {
  return (pos >= it.hi_min && pos < sp.hi) || (pos >= sp.lo && pos >= p.sinks && pos < it.lo_max && pos < sp.hi);
}
__device__ __forceinline__ bool tile_in_part(const ChunkParams& p, const Span& sp, const Item& it, int pos0) {
  const bool end = it.hi_min < sp.hi && pos0 + kTile > it.hi_min && pos0 < sp.hi;
  return end || (pos0 < it.lo_max && pos0 + kTile > sp.lo && pos0 + kTile > p.sinks);
}
// Whether the cleaner has to look at the tile.
__device__ __forceinline__ bool tile_to_clean(const ChunkParams& p, const Span& sp, const Item& it, int pos0) {
  return pos0 + kTile > sp.hi || (pos0 < sp.lo && pos0 + kTile > sp.s_end) || tile_in_part(p, sp, it, pos0);
}

// Bits [a, b) of a word.
__device__ __forceinline__ uint32_t bits_below(int x) { return x <= 0 ? 0u : x >= 32 ? 0xffffffffu : (1u << x) - 1u; }

// 32 scores of this thread's row: P = 2^(s * scale + r) as bf16 pairs, the sum of the unrounded weights as a packed pair.
template <bool kMasked>
__device__ __forceinline__ void weigh(const uint32_t* s, unsigned long long sc2, unsigned long long ref2, uint32_t seen,
                                      unsigned long long& sum, uint32_t* pk) {
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    float x0, x1;
    unpack_f2(fma_f2(pack_f2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), sc2, ref2), x0, x1);
    float p0 = fast_exp2(x0), p1 = fast_exp2(x1);
    if (kMasked) {
      p0 = ((seen >> (2 * e)) & 1u) ? p0 : 0.f;
      p1 = ((seen >> (2 * e + 1)) & 1u) ? p1 : 0.f;
    }
    sum = add_f2(sum, pack_f2(p0, p1));
    const __nv_bfloat162 h = __floats2bfloat162_rn(p0, p1);
    pk[e] = *reinterpret_cast<const uint32_t*>(&h);
  }
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

// An item's partials, joined by the four warps of a lane in CTA order (contributors c_lo..c_hi; place 1 of the first, 0 of the others). A warp takes U
// rows side by side, HD / 32 columns a lane: the weights of 32 / U contributors of U rows come with one load, and the rows' loads of several contributors
// are in flight together (one element at a time, a round trip to L2 each, joined 128 rows in 27 us).
template <int HD, int U>
__device__ __noinline__ void merge_rows(const ChunkParams& p, const ChunkSeq& s, int kvh, int tok0, int rows, int c_lo, int c_hi, size_t lane0) {
  constexpr int NC = HD / 32, CP = 32 / U, KU = U == 1 ? 8 : 2;  // columns per lane, contributors per pass, contributors in flight
  const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) & 3;
  auto place = [&](int c) { return ((size_t)c * 2 + (c == c_lo ? 1 : 0)) * (2 * kRows) + lane0; };
  const int u_mine = lane / CP, c_mine = lane % CP;
  for (int r0 = warp * U; r0 < rows; r0 += 4 * U) {
    auto pair_of = [&](int c) { return c <= c_hi && r0 + u_mine < rows ? __ldcg(p.part_ml + place(c) + r0 + u_mine) : make_float2(-INFINITY, 0.f); };
    float2 ml = pair_of(c_lo + c_mine);
    float top = ml.x;
    for (int cb = c_lo + CP; cb <= c_hi; cb += CP) top = fmaxf(top, pair_of(cb + c_mine).x);
#pragma unroll
    for (int o = CP / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float acc[U][NC] = {}, l = 0.f;
    for (int cb = c_lo; cb <= c_hi; cb += CP) {
      if (cb > c_lo) ml = pair_of(cb + c_mine);
      const float wt = ml.x > -INFINITY ? exp2f(ml.x - top) : 0.f;
      l += ml.x > -INFINITY ? wt * ml.y : 0.f;
#pragma unroll 1
      for (int k0 = 0; k0 < CP && cb + k0 <= c_hi; k0 += KU) {
        float x[KU][U][NC];
#pragma unroll
        for (int k = 0; k < KU; ++k)
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const float* src = p.part_o + (place(min(cb + k0 + k, c_hi)) + min(r0 + u, rows - 1)) * HD + lane * NC;
            if constexpr (NC == 4) {
              const float4 v = __ldcg(reinterpret_cast<const float4*>(src));
              x[k][u][0] = v.x; x[k][u][1] = v.y; x[k][u][2] = v.z; x[k][u][3] = v.w;
            } else {
              const float2 v = __ldcg(reinterpret_cast<const float2*>(src));
              x[k][u][0] = v.x; x[k][u][1] = v.y;
            }
          }
#pragma unroll
        for (int k = 0; k < KU; ++k)
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const float f = __shfl_sync(0xffffffffu, wt, u * CP + min(k0 + k, CP - 1));
            if (k0 + k < CP && cb + k0 + k <= c_hi && f != 0.f) {
#pragma unroll
              for (int e = 0; e < NC; ++e) acc[u][e] = fmaf(f, x[k][u][e], acc[u][e]);
            }
          }
      }
    }
#pragma unroll
    for (int o = CP / 2; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float lt = __shfl_sync(0xffffffffu, l, u * CP), inv = lt == 0.f ? 0.f : 1.f / lt;
      const int rr = r0 + u;
      if (rr < rows) {
        uint32_t o[NC / 2];
#pragma unroll
        for (int e = 0; e < NC; e += 2) {
          const __nv_bfloat162 b2 = __floats2bfloat162_rn(acc[u][e] * inv, acc[u][e + 1] * inv);
          o[e / 2] = *reinterpret_cast<const uint32_t*>(&b2);
        }
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.out) + (((size_t)s.off + tok0 + rr / p.G) * p.Hq + kvh * p.G + rr % p.G) * HD + lane * NC;
        if constexpr (NC == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(o[0], o[1]);
        else *reinterpret_cast<uint32_t*>(dst) = o[0];
      }
    }
  }
}

template <int HD, bool kTree>
__global__ void __launch_bounds__(kThreadsC, 1)
chunk_attn_tc_kernel(const ChunkParams p, const TcArgs a, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v) {
  using M = Mem<HD>;
  extern __shared__ __align__(1024) unsigned char smem[];
  Misc<HD>& ms = *reinterpret_cast<Misc<HD>*>(smem + M::kAtMisc);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_q)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_k)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map_v)) : "memory");
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ms.q_full[i], 1);
      mbar_init(&ms.q_free[i], 1);
      mbar_init(&ms.s_full[i], 1);
      mbar_init(&ms.p_full[i], kRows);
      mbar_init(&ms.o_full[i], 1);
    }
    for (int i = 0; i < M::kStagesK; ++i) {
      mbar_init(&ms.k_full[i], 1);
      mbar_init(&ms.k_free[i], 1);
    }
    for (int i = 0; i < M::kStagesV; ++i) {
      mbar_init(&ms.v_full[i], 1);
      mbar_init(&ms.v_free[i], 1);
      mbar_init(&ms.v_raw[i], 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_proxy_async();
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // behind the wait (a predecessor may hold tensor memory until it ends), and the dependents are released behind the allocation
  if (warp == 10) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ms.tmem)), "n"(kTmemColumns));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  }
  const bool aligned = (smem_u32(smem) & 1023u) == 0u;  // the swizzled regions need it
  if (!aligned && tid == 0) report(p.st, CAST_ERR_CUDA, 1024);
  tc_fence_before();
  make_plan<kTile, kTree>(p, ms.plan);  // (ends with a barrier)
  tc_fence_after();
  const uint32_t tmem = ms.tmem;
  const ChunkPlan& plan = ms.plan;
  ChunkWalk w;
  bool more = aligned && walk_begin<kTile, kTree>(p, plan, w, blockIdx.x);
  auto next = [&] { more = walk_next<kTile, kTree>(p, plan, w); };

  // Registers: 384 x 168 at launch; the softmax threads take 208 (a tile's weights and half its scores are 128), the others give theirs: 256 x 208 + 128 x 80 = 63488 of 64512.
  auto give = [] { asm volatile("setmaxnreg.dec.sync.aligned.u32 80;"); };
  if (warp == 8 || warp == 9) {
    give();
    // =========================== loads: Q and K, or V ===========================
    const bool is_v = warp == 9;
    const int stages = is_v ? M::kStagesV : M::kStagesK;
    uint64_t* full = is_v ? ms.v_full : ms.k_full;
    uint64_t* free = is_v ? ms.v_free : ms.k_free;
    unsigned char* ring = smem + (is_v ? M::kAtV : M::kAtK);
    const CUtensorMap* map = is_v ? &map_v : &map_k;
    int tile = 0, qc = 0, cleaned = 0;  // tiles, Q slots and tiles for the cleaner so far
    bool ok = true;
    const int per_tile = p.g.page_size == 0 ? 1 : kTile / a.box;  // copies per half
    const int copy = lane / M::kHalves, half = lane % M::kHalves;
    for (; more && ok; next()) {
      const int T = w.t1 - w.t0;
      if (T <= 0) continue;
      const ChunkSeq s = plan.seq[w.b];
      const Item it = item_of<kTree>(p, s, w);
      if (!is_v) {
        for (int h = 0; h < (it.pair ? 2 : 1) && ok; ++h, ++qc) {
          const int slot = qc & 1;
          if (qc >= 2) ok = mbar_wait(&ms.q_free[slot], ((qc >> 1) - 1) & 1);
          if (!ok) break;
          if (lane == 0) mbar_expect_tx(&ms.q_full[slot], (uint32_t)(M::kHalves * a.q_tokens * p.G * 128));
          __syncwarp();
          if (lane < M::kHalves)
            tma_load_3d(&map_q, smem + M::kAtQ + slot * M::kQ + lane * kRegQ, &ms.q_full[slot], lane * 64, w.h * p.G, s.off + it.tf + h * a.tokens);
        }
      }
      // the page of this lane's copy of a tile, read one tile ahead; -1: nothing of it is seen
      auto page_of = [&](int i) {
        const int pos = w.span.tile(i) * kTile + copy * a.box;
        int page = -1;
        if (i < w.t1 && copy < per_tile && pos < w.span.hi && (pos + a.box > w.span.lo || pos < w.span.s_end))
          page = p.g.table[(size_t)w.b * p.g.seq_capacity + pos / p.g.page_size];
        else
          return -1;
        if (page < 0 || page >= p.g.num_pages) {
          report(p.st, CAST_ERR_BAD_PAGE, w.b);
          page = 0;
        }
        return page;
      };
      int page = p.g.page_size ? page_of(w.t0) : 0;
      for (int i = w.t0; i < w.t1 && ok; ++i, ++tile) {
        const int stage = tile % stages, pos0 = w.span.tile(i) * kTile;
        const int now = page;
        if (p.g.page_size) page = page_of(i + 1);
        if (tile >= stages) ok = mbar_wait(&free[stage], ((tile / stages) - 1) & 1);
        if (!ok) break;
        unsigned char* dst = ring + stage * M::kTileBytes + half * kRegKV;
        uint64_t* bar = &full[stage];
        if (is_v && tile_to_clean(p, w.span, it, pos0)) bar = &ms.v_raw[cleaned++ % M::kStagesV];
        if (p.g.page_size == 0) {
          if (lane == 0) mbar_expect_tx(bar, M::kTileBytes);
          __syncwarp();
          if (lane < M::kHalves) tma_load_3d(map, dst, bar, half * 64, w.h, w.b * p.g.seq_capacity + pos0);
        } else {
          const int copies = __popc(__ballot_sync(0xffffffffu, now >= 0));
          if (lane == 0) mbar_expect_tx(bar, (uint32_t)(copies * a.box * 128));
          __syncwarp();
          if (now >= 0) {
            const int pos = pos0 + copy * a.box;
            tma_load_4d(map, dst + copy * a.box * 128, bar, half * 64, w.h, pos % p.g.page_size, now);
          }
        }
        __syncwarp();
      }
    }
    if (!ok) {  // a wait ran out: the copies in flight land before this CTA's shared memory is given up
      if (lane == 0) report(p.st, CAST_ERR_TIMEOUT, blockIdx.x);
      for (int j = max(0, tile - stages); j < tile; ++j) mbar_wait(&full[j % stages], (j / stages) & 1);
      if (!is_v)
        for (int j = max(0, qc - 2); j < qc; ++j) mbar_wait(&ms.q_full[j & 1], (j >> 1) & 1);
    }
  } else if (warp == 10) {
    give();
    // =========================== products ===========================
    const uint32_t idesc_qk = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kTile >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
    const uint32_t idesc_pv = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(HD >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
    const uint32_t tm = __reduce_or_sync(0xffffffffu, tmem);  // (the same in all lanes: uniform registers, which the products' operands come from)
    const uint64_t dq = umma_desc(smem_u32(smem + M::kAtQ), 16, 1024);
    const uint64_t dk = umma_desc(smem_u32(smem + M::kAtK), 16, 1024);
    const uint64_t dv = umma_desc(smem_u32(smem + M::kAtV), kRegKV, 1024);
    int kst = 0, kph = 0, vst = 0, vph = 0, qc = 0, turn = 0, newest = 1;
    uint32_t pph = 0;                 // phase of p_full, a bit per lane
    // a lane's P V that waits: bit 0 there is one, 1 V's phase, 2 it releases V, 3 it is the item's last, then V's stage
    int pend0 = 0, pend1 = 0;
    bool ok = true;
    auto flush = [&](int h) {         // the lane's P V
      const int f = h ? pend1 : pend0;
      if (!ok || !(f & 1)) return;
      const int stage = f >> 4;
      ok = mbar_wait(&ms.p_full[h], (pph >> h) & 1) && mbar_wait(&ms.v_full[stage], (f >> 1) & 1);
      if (!ok) return;
      pph ^= 1u << h;
      tc_fence_after();
      const uint64_t d = dv + (uint64_t)(stage * (M::kTileBytes >> 4));
#pragma unroll
      for (int ks = 0; ks < kTile / 16; ++ks)
        umma_bf16_ts(tm + kColO + h * kLaneCols, tm + kColS + h * kLaneCols + ks * 8, d + (uint64_t)(ks * (2048 >> 4)), idesc_pv, 1u);
      if (f & 4) umma_commit(&ms.v_free[stage]);
      if (f & 8) umma_commit(&ms.o_full[h]);
      if (h) pend1 = 0;
      else pend0 = 0;
    };
    for (; more && ok; next()) {
      const int T = __reduce_max_sync(0xffffffffu, w.t1 - w.t0);
      if (T <= 0) continue;
      const ChunkSeq s = plan.seq[w.b];
      const Item it = item_of<kTree>(p, s, w);
      const int lanes = __reduce_max_sync(0xffffffffu, it.pair ? 2 : 1);
      // The older tile's P V goes first, always: a lane's softmax comes to an item only behind the join of the one before, which waits for
      // the other lane's P V there. (While the lanes take turns the order is right by itself.)
      if (lanes == 2 && newest == 0) flush(1);
      for (int i = 0; i < T && ok; ++i) {
        for (int j = 0; j < lanes && ok; ++j) {
          const int h = lanes == 2 ? j : (turn + i) & 1;
          flush(h);
          if (!ok) break;
          const int c = qc + j, slot = c & 1;
          if (i == 0) ok = mbar_wait(&ms.q_full[slot], (c >> 1) & 1);
          if (ok && j == 0) ok = mbar_wait(&ms.k_full[kst], kph);
          if (!ok) break;
          tc_fence_after();
          const uint64_t q = dq + (uint64_t)(slot * (M::kQ >> 4)), k = dk + (uint64_t)(kst * (M::kTileBytes >> 4));
#pragma unroll
          for (int ks = 0; ks < HD / 16; ++ks)
            umma_bf16(tm + kColS + h * kLaneCols, q + (uint64_t)((ks >> 2) * (kRegQ >> 4) + (ks & 3) * 2),
                      k + (uint64_t)((ks >> 2) * (kRegKV >> 4) + (ks & 3) * 2), idesc_qk, ks > 0);
          umma_commit(&ms.s_full[h]);
          if (j == lanes - 1) umma_commit(&ms.k_free[kst]);
          if (i == T - 1) umma_commit(&ms.q_free[slot]);
          const int f = 1 | (vph << 1) | (j == lanes - 1 ? 4 : 0) | (i + (lanes == 2 ? 1 : 2) >= T ? 8 : 0) | (vst << 4);
          if (h) pend1 = f;
          else pend0 = f;
          newest = h;
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
      qc += lanes;
      if (lanes == 1) turn = (turn + T) & 1;
    }
    flush(newest ^ 1);
    if (ok) flush(newest);
    if (!ok && lane == 0) report(p.st, CAST_ERR_TIMEOUT, blockIdx.x);
  } else if (warp == 11) {
    give();
    // =========================== V tiles that not every row sees whole ===========================
    int tile = 0, cleaned = 0;
    bool ok = true;
    for (; more && ok; next()) {
      const ChunkSeq s = plan.seq[w.b];
      const Item it = w.t1 > w.t0 ? item_of<kTree>(p, s, w) : Item();
      for (int i = w.t0; i < w.t1; ++i, ++tile) {
        const int stage = tile % M::kStagesV, pos0 = w.span.tile(i) * kTile;
        if (!tile_to_clean(p, w.span, it, pos0)) continue;
        ok = mbar_wait(&ms.v_raw[cleaned % M::kStagesV], (cleaned / M::kStagesV) & 1);
        if (!ok) break;
        {
          unsigned char* v = smem + M::kAtV + stage * M::kTileBytes;
          const bool part = tile_in_part(p, w.span, it, pos0);
#pragma unroll 1
          for (int j = 0; j < 4; ++j) {
            const int r = j * 32 + lane, pos = pos0 + r;
            const bool seen = pos < w.span.hi && (pos >= w.span.lo || pos < w.span.s_end);
            bool bad = false;
            if (part && seen && seen_in_part(p, w.span, it, pos)) {
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
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&ms.v_full[stage]);
        ++cleaned;
      }
    }
    if (!ok && lane == 0) report(p.st, CAST_ERR_TIMEOUT, blockIdx.x);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // =========================== softmax and output ===========================
    const int h = warp >> 2, r = tid & (kRows - 1), bar_id = 1 + h;
    const uint32_t rowsel = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + kColS + h * kLaneCols + rowsel, t_o = tmem + kColO + h * kLaneCols + rowsel;
    const float sc = a.scale_log2;
    const unsigned long long sc2 = pack_f2(sc, sc);
    int vtile = 0, steps = 0, items = 0, turn = 0;  // V tiles so far, this lane's tiles, this lane's items
    bool ok = true;
    for (; more; next()) {
      const int T = w.t1 - w.t0;
      const bool nothing = w.span.n == 0 && w.at == w.item0;
      if (T <= 0 && !nothing) continue;
      const ChunkSeq s = plan.seq[w.b];
      const Item it = item_of<kTree>(p, s, w);
      const int t_first = it.pair ? 0 : (h - turn) & 1;  // this lane's first tile: it takes all, or every other one
      const bool both = !it.pair && T > 1, mine = it.pair || t_first < T;
      if (!it.pair) turn = (turn + T) & 1;
      const int vt0 = vtile;
      vtile += T;
      if (!mine && !nothing) continue;  // (one tile, the other lane's)
      // the row
      const int lane_rows = it.pair ? min(max(it.rows - h * a.tokens * p.G, 0), a.tokens * p.G) : it.rows;
      const bool row_ok = r < lane_rows, warp_live = (warp & 3) * 32 < lane_rows;
      const int tok = it.tf + (it.pair ? h * a.tokens : 0) + (row_ok ? r / p.G : 0), head = w.h * p.G + (row_ok ? r % p.G : 0);
      __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(p.out) + (((size_t)s.off + tok) * p.Hq + head) * HD;
      if (nothing) {
        if (row_ok && (it.pair || h == 0))
          for (int c = 0; c < HD / 8; ++c) *reinterpret_cast<uint4*>(out + c * 8) = make_uint4(0u, 0u, 0u, 0u);
        continue;
      }
      const int depth = kTree && row_ok ? depth_of(p, s, tok) : 0;
      const RowSight rs = sight_of<kTree>(p, s, tok, depth);
      uint32_t aw[4] = {0u, 0u, 0u, 0u};
      if (kTree && row_ok) {
#pragma unroll
        for (int j = 0; j < 4; ++j) aw[j] = tree_word(p, s, tok, depth, j);
      }
      const int hi_all = __reduce_min_sync(0xffffffffu, row_ok ? rs.hi : 0x7fffffff), lo_all = __reduce_max_sync(0xffffffffu, row_ok ? rs.lo : 0);
      float ref = row_ok ? 0.f : -INFINITY, l_run = 0.f;  // a row that is none: its P is 0 for every finite score
      if (warp_live && ok) {
        uint32_t z[32];
#pragma unroll
        for (int c = 0; c < 32; ++c) z[c] = 0u;
#pragma unroll
        for (int c = 0; c < HD; c += 32) tmem_st32(t_o + c, z);
        tmem_wait_st();
      }
      for (int i = t_first; i < T; i += it.pair ? 1 : 2, ++steps) {
        if (ok) ok = mbar_wait(&ms.s_full[h], steps & 1);
        if (!ok) {
          tc_fence_before();
          mbar_arrive(&ms.p_full[h]);
          continue;
        }
        if (!warp_live) {
          tc_fence_before();
          mbar_arrive(&ms.p_full[h]);
          continue;
        }
        tc_fence_after();
        const int pos0 = w.span.tile(w.t0 + i) * kTile;
        const bool plain = pos0 + kTile <= hi_all && (pos0 >= lo_all || pos0 + kTile <= rs.sinks);
        auto seen_word = [&](int j) -> uint32_t {  // what the row sees of positions pos0 + 32 j on
          const int base = pos0 + j * 32;
          uint32_t v = bits_below(rs.hi - base) & (~bits_below(rs.lo - base) | bits_below(rs.sinks - base));
          if (kTree) {
            const int st = base - s.L, wi = st >> 5, sh = st & 31;  // (arithmetic shift)
            auto word = [&](int x) { return x == 0 ? aw[0] : x == 1 ? aw[1] : x == 2 ? aw[2] : x == 3 ? aw[3] : 0u; };
            v |= __funnelshift_r(word(wi), word(wi + 1), sh);
          }
          return row_ok ? v : 0u;
        };
        uint32_t pk[64];
        unsigned long long sum2 = pack_f2(0.f, 0.f);
        {
          const unsigned long long ref2 = pack_f2(ref, ref);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t x[64];
            tmem_get64(t_s + j * 64, x);
            if (plain) {
              weigh<false>(x, sc2, ref2, 0u, sum2, pk + 32 * j);
              weigh<false>(x + 32, sc2, ref2, 0u, sum2, pk + 32 * j + 16);
            } else {
              weigh<true>(x, sc2, ref2, seen_word(2 * j), sum2, pk + 32 * j);
              weigh<true>(x + 32, sc2, ref2, seen_word(2 * j + 1), sum2, pk + 32 * j + 16);
            }
          }
        }
        float l0, l1;
        unpack_f2(sum2, l0, l1);
        l0 += l1;
        const bool far = row_ok && !(l0 < 1.15e18f);  // 2^60
        const bool low = row_ok && l_run + l0 < 8.6e-19f && (plain || (seen_word(0) | seen_word(1) | seen_word(2) | seen_word(3)) != 0u);  // 2^-60, something seen
        if (__any_sync(0xffffffffu, far || low)) {
          uint32_t sa[32];
          // (P V of this lane's tile before is over: the product that made these scores was issued behind it)
          float top = -INFINITY;
#pragma unroll 1
          for (int j = 0; j < 4; ++j) {
            tmem_get32(t_s + j * 32, sa);
            const uint32_t v = plain ? 0xffffffffu : seen_word(j);
#pragma unroll
            for (int c = 0; c < 32; ++c) top = fmaxf(top, ((v >> c) & 1u) ? __uint_as_float(sa[c]) : -INFINITY);
          }
          float kf = 0.f;
          if (far || low) {
            const float e_tile = top > -INFINITY ? fmaf(top, sc, ref) : -INFINITY;
            const float e_acc = l_run > 0.f ? log2f(l_run) : -INFINITY;
            const float e = fmaxf(e_tile, e_acc);
            if (e > -INFINITY && e < INFINITY) kf = fminf(fmaxf(ceilf(e), -1.0e9f), 1.0e9f);
          }
          const float alpha = l_run > 0.f ? ldexpf(1.f, -(int)kf) : 1.f;
          if (__any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll 1
            for (int c = 0; c < HD; c += 32) {
              tmem_get32(t_o + c, sa);
#pragma unroll
              for (int e = 0; e < 32; ++e) sa[e] = __float_as_uint(__uint_as_float(sa[e]) * alpha);
              tmem_st32(t_o + c, sa);
            }
            tmem_wait_st();
          }
          l_run *= alpha;
          ref -= kf;
          sum2 = pack_f2(0.f, 0.f);
          const unsigned long long ref2 = pack_f2(ref, ref);
#pragma unroll
          for (int j = 0; j < 4; ++j) {  // the tile again (rows that did not move get the same values)
            tmem_get32(t_s + j * 32, sa);
            weigh<true>(sa, sc2, ref2, plain ? (row_ok ? 0xffffffffu : 0u) : seen_word(j), sum2, pk + 16 * j);
          }
          unpack_f2(sum2, l0, l1);
          l0 += l1;
        }
        if (tile_in_part(p, w.span, it, pos0)) {
          const int vt = vt0 + i, stage = vt % M::kStagesV;
          ok = mbar_wait(&ms.v_full[stage], (vt / M::kStagesV) & 1);
          if (ok) {
#pragma unroll 1
            for (int j = 0; j < 4; ++j) {
              const uint32_t v = seen_word(j);
              for (uint32_t left = ms.bad[stage][j]; left; left &= left - 1) {  // V rows that hold a NaN or an infinity, as the cleaner found them
                const int bit = __ffs(left) - 1, pos = pos0 + j * 32 + bit;
                if (!__any_sync(0xffffffffu, (v >> bit) & 1u)) continue;
                uint32_t x, sa[32];
                tmem_get1(t_s + j * 32 + bit, x);
                const float wt = ((v >> bit) & 1u) ? fast_exp2(fmaf(__uint_as_float(x), sc, ref)) : 0.f;
                int page = 0, slot = 0;
                if (!find_place(p.g, w.b, pos, page, slot)) page = 0;
                const size_t at = (((size_t)page * (p.g.page_size == 0 ? p.g.seq_capacity : p.g.page_size) + slot) * p.Hkv + w.h) * HD;
                const __nv_bfloat16* row = reinterpret_cast<const __nv_bfloat16*>(p.v) + at;
#pragma unroll 1
                for (int c = 0; c < HD; c += 32) {
                  tmem_get32(t_o + c, sa);
#pragma unroll
                  for (int e = 0; e < 32; ++e) {
                    const float f = __bfloat162float(row[c + e]);
                    if ((v >> bit) & 1u) sa[e] = __float_as_uint(fmaf(wt, f, __uint_as_float(sa[e])));
                  }
                  tmem_st32(t_o + c, sa);
                }
                tmem_wait_st();
              }
            }
          }
        }
        tmem_st32(t_s, pk);
        tmem_st32(t_s + 32, pk + 32);
        l_run += l0;
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&ms.p_full[h]);
      }
      // ---- the output, or this CTA's partial
      if (ok) ok = mbar_wait(&ms.o_full[h], items & 1);
      ++items;
      tc_fence_after();
      float m = l_run == 0.f || !ok ? -INFINITY : -ref, l = ok ? l_run : 0.f, f0 = 1.f, f1 = 0.f;
      if (both) {  // lane 0 joins both: each row's outputs lie at the same tensor-memory lane
        if (h == 1) ms.ml[r] = make_float2(m, l);
        tc_fence_before();
        asm volatile("bar.sync 3, 256;" ::: "memory");
        tc_fence_after();
        if (h == 0) {
          const float2 o = ms.ml[r];
          const float top = fmaxf(m, o.x);
          f0 = m > -INFINITY ? exp2f(m - top) : 0.f;
          f1 = o.x > -INFINITY ? exp2f(o.x - top) : 0.f;
          l = f0 * l + f1 * o.y;
          m = top;
        } else {
          asm volatile("bar.sync 4, 256;" ::: "memory");
          continue;
        }
      }
      const bool whole = w.t0 == 0 && w.t1 == w.span.n;
      const int c_lo = whole ? 0 : owner_of(plan, w.item0 + kItemCost), c_hi = whole ? 0 : owner_of(plan, w.item0 + kItemCost + w.span.n - 1);
      auto place = [&](int c) { return ((size_t)c * 2 + (c == c_lo ? 1 : 0)) * (2 * kRows) + (it.pair ? h * kRows : 0); };
      const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
      float* part = p.part_o + (place(blockIdx.x) + r) * HD;
      if (warp_live) {
#pragma unroll 1
        for (int c = 0; c < HD; c += 32) {
          uint32_t o[32];
          if (ok) {
            tmem_get32(t_o + c, o);
          }
          float x[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = ok && f0 != 0.f ? __uint_as_float(o[e]) * f0 : 0.f;
          if (both && ok) {
            tmem_get32(t_o + kLaneCols + c, o);
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = f1 != 0.f ? fmaf(__uint_as_float(o[e]), f1, x[e]) : x[e];
          }
          if (row_ok) {
            if (whole) {
#pragma unroll
              for (int e = 0; e < 32; e += 8) {
                uint32_t u[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const __nv_bfloat162 b2 = __floats2bfloat162_rn(x[e + 2 * k] * inv, x[e + 2 * k + 1] * inv);
                  u[k] = *reinterpret_cast<const uint32_t*>(&b2);
                }
                *reinterpret_cast<uint4*>(out + c + e) = make_uint4(u[0], u[1], u[2], u[3]);
              }
            } else {
#pragma unroll
              for (int e = 0; e < 32; e += 4) __stcg(reinterpret_cast<float4*>(part + c + e), make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]));
            }
          }
        }
      }
      if (both) {
        tc_fence_before();
        asm volatile("bar.sync 4, 256;" ::: "memory");
      }
      if (whole) continue;
      if (row_ok) __stcg(p.part_ml + place(blockIdx.x) + r, make_float2(m, l));
      asm volatile("bar.sync %0, 128;" ::"r"(bar_id) : "memory");
      if (r == 0) {
        // releases this CTA's partial (the barrier made it this thread's to release), acquires those that came earlier
        int32_t* ticket = p.ticket + 2 * c_lo + (it.pair ? h : 0);
        int t;
        asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(t) : "l"(ticket) : "memory");
        ms.last[h] = t == c_hi - c_lo;
        if (t == c_hi - c_lo) *ticket = 0;  // ready for the next launch
      }
      asm volatile("bar.sync %0, 128;" ::"r"(bar_id) : "memory");
      if (!ms.last[h]) continue;
      const size_t lane0 = it.pair ? h * kRows : 0;
      const int tk0 = it.tf + (it.pair ? h * a.tokens : 0);
      if (lane_rows <= 4) merge_rows<HD, 1>(p, s, w.h, tk0, lane_rows, c_lo, c_hi, lane0);
      else merge_rows<HD, 8>(p, s, w.h, tk0, lane_rows, c_lo, c_hi, lane0);
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
  a.scale_log2 = p.scale * 1.4426950408889634f;
  p.block_rows = 2 * a.tokens * p.G;
  p.min_units = kItemCost + 2;
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
