// Tensor-core path of cast_tree_attention_q4: bf16 queries over the 4-bit cache (sm_100a: tcgen05 + TMEM).
//
// With step and low of a row taken out of the products, the codes themselves enter the matrix units, exactly, as small
// integers in bf16:
//   q . k_p = step_p (q . c_p) + low_p sum(q)        sum_p w_p v_p = sum_p (w_p step_p) (c_p - 8) + sum_p w_p (low_p + 8 step_p)
// so a score carries no rounding but the accumulation's, and a weight (times its row's step) one to bf16; the last sum stays in fp32.
//
// Positions are the rows of both products, queries the columns: S^T = C_k Q^T (128 positions x N queries) and
// O^T = C_v^T P^T (dims x N). A query column is a (tree token, head of the GQA group) pair, up to 48 per work item; N is 16 for items of
// up to 16 of them and 48 otherwise: a small tree costs that, not a block of 128 rows, and its exponentials spread over all lanes. A thread of the softmax
// owns one position: step and low are scalars of its own, masks are one word per position, and sums run in registers over
// all its tiles, reduced across lanes once per item. What is paid for that: the maximum of a column lies across lanes, so the
// running reference of a column is not its maximum but the first visible tile's, moved when a weight reaches 2^60 (bf16 and fp32 have
// the range), which one vote per tile finds.
//
// Eight warps, two CTAs per SM, every warp with the same work: in a tile, its 16 rows of V codes to shared memory (c - 8, 128-byte
// swizzled: the MN-major A operand as they lie), the softmax of 32 positions x half of the columns, its 16 rows of the next
// tile's K codes to tensor memory (16 + c, the A operand; the dims in the order the quad of lanes holds them, and Q in the same order);
// then the CTA meets, a warp issues S^T of the next tile and O^T of this one, and the products run under the next tile's V codes
// and under the other CTA. Codes and pairs are requested a tile ahead, into registers. (Warps of their own for K, V, pairs, the MMAs and
// the softmax, 18 in one CTA per SM, took six times as long: five streams of unrolled code on one SM's instruction cache, every
// instruction about ten cycles apart.)
// Work is one line of tiles, item after item (sequence, kv-head, block of 48 rows), cut into pieces, one per CTA: item by item while
// there are few items, else evenly, so that ragged batches load the machine evenly. An item that lies across CTAs leaves partials in the workspace; the last CTA to finish it
// (an atomic ticket, nothing spins) merges them in CTA order. All mbarrier waits are bounded: on expiry the CTA records
// CAST_ERR_TIMEOUT, stops touching the operands and runs out.
//
// Measured, heads of 128 dims, per layer: 64 sequences of 512 to 4096, 12 tokens, 32 / 8 heads 162 us (26 to read the cache); 4 of
// 32768, 96 tokens, 28 / 4 heads 672 us (109 for the products at the matrix units' measured rate); one of 2048, 60 tokens 31 us
// (25 with 12).
// Neither memory (12 %) nor the matrix units (8 %) bound it but the instructions that turn codes into operands and scores into
// weights, with their waits: issue slots are 44 % busy with 16 warps per SM, which is what the registers allow. A single short
// sequence is bound by the chain launch - queries - first scores - partials - merge. Tried and slower: warps of their own per task (above);
// four warps with 48 columns each; the sums l and z as a third product (its operand's memory leaves one CTA per SM); K codes
// double-buffered; the first attempt's weights redone in place of the vote; the merge in loops over rows (tiles 8 % slower: it is the
// tiles' register allocation that changes).
#include <math.h>

#include "q4_tc.h"

namespace cast {

namespace {

constexpr int kTile = 128;       // positions per tile (UMMA M)
constexpr int kRows = 48;        // query columns per item at most (UMMA N): half of them, three times eight, are a thread's
constexpr int kHalf = kRows / 2;
constexpr int kThreadsQ4 = 256;
constexpr int kMaxGrid = 512;
constexpr int kMaxJoin = 32;     // CTAs that share an item, about
constexpr float kFar = 1.15292150460684698e18f;  // 2^60

struct Q4Params {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  const unsigned char *kc, *vc;
  const uint32_t *kr, *vr;
  int B, Ncap, Nmax, Hq, Hkv, G, words;
  FastPaging g;
  const int32_t* kv_len;
  const int32_t* n_tree;
  const int32_t* first_row;
  const uint32_t* anc;
  float scale_log2;
  float* part_o;    // [grid][2][kRows][HD], dims in the order of the tensor-memory lanes
  float2* part_ml;  // [grid][2][kRows] reference (log2 units), sum
  int32_t* ticket;  // [B][Hkv][row blocks]
  int nrb;          // row blocks that a sequence has at most
  DevState* st;
};

template <int HD>
struct Lay {
  static constexpr int kW = HD / 32;                 // words of codes per thread and row (four threads to a row)
  static constexpr int kSmemQ = 0;                   // HD / 64 regions [48 rows][64] bf16
  static constexpr int kRegionQ = kRows * 128;
  static constexpr int kSmemV = kSmemQ + HD / 64 * kRegionQ;
  static constexpr int kRegionV = kTile * 128;       // [128 positions][64] bf16
  static constexpr int kBufV = HD / 64 * kRegionV;
  static constexpr int kSmemP = kSmemV + 2 * kBufV;  // [128 positions][64] bf16, 48 of them used
  static constexpr int kBufP = kTile * 128;
  static constexpr int kSmemMisc = kSmemP + kBufP;
};

template <int N>
struct Count {
  static constexpr int value = N;
};

// A place on the line of tiles.
struct Walk {
  int b, h, rb, t;  // sequence, kv-head, row block, tile of the item
  int left;         // tiles from here to the end of the CTA's piece, this one included; behind the end the place stays the last
};
struct Misc {
  uint64_t bar_s, bar_o;
  uint32_t tmem;
  int last, workers;
  long long piece;                     // tiles of a CTA, rounded down; the first `rest` CTAs take one more
  int rest;
  int whole;                           // pieces end with their items: the line is cut item by item
  Walk seg;                            // the item in work, from its first tile here on
  Walk ahead;                          // the furthest tile in `step`
  alignas(16) int4 step[8];            // tile i of the CTA at i % 8: sequence, kv-head, first position, positions of the sequence
  long long pre[CAST_MAX_BATCH + 1];   // tiles of the sequences before
  long long bound[kMaxGrid + 1];       // first tile of every CTA
  int cta[CAST_MAX_BATCH], per[CAST_MAX_BATCH];  // cut item by item: CTAs of the sequences before, CTAs of an item
  int L[CAST_MAX_BATCH], N[CAST_MAX_BATCH], F[CAST_MAX_BATCH], tl[CAST_MAX_BATCH], nr[CAST_MAX_BATCH], total[CAST_MAX_BATCH];
  alignas(16) float sq[kRows];         // sums of the query rows
  alignas(16) float nm[kRows];         // references, log2 units, negated; inf: none yet
  alignas(16) float alpha[kRows];      // what a moved reference scales by
  alignas(16) uint32_t at[kRows];      // a query row's first element in q and out
  alignas(16) float tot_l[kRows];
  alignas(16) float tot_z[kRows];
  float red_l[4][kRows], red_z[4][kRows];
  float colmax[8][kHalf];
  uint32_t vis[2][CAST_MAX_TREE];      // columns (32 + 16) that see a tree token
};

constexpr int kTmemK = 0, kTmemS = 64, kTmemO = 128, kTmemCols = 256;  // K codes 64, scores 48, output 48

__device__ __forceinline__ void advance(Walk& w, const Misc& s, const Q4Params& p) {
  if (--w.left <= 0 || ++w.t < s.tl[w.b]) return;
  w.t = 0;
  if (++w.rb < s.nr[w.b]) return;
  w.rb = 0;
  if (++w.h < p.Hkv) return;
  w.h = 0;
  do ++w.b;
  while (s.tl[w.b] == 0);  // (tiles are left, so a sequence with tiles follows)
}

// Sums on, weights times step to the B operand. (One copy of it: with a masked one beside it every sum was moved between two
// registers every tile.)
template <int NH>
__device__ __forceinline__ void hand_over(const float (&p)[NH], float (&l)[NH], float (&z)[NH], unsigned char* row, int r7, int chunk0, float vs,
                                          float vl) {
#pragma unroll
  for (int c8 = 0; c8 < NH / 8; ++c8) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = c8 * 8 + 2 * e;
      l[c] += p[c];
      l[c + 1] += p[c + 1];
      z[c] = fmaf(p[c], vl, z[c]);
      z[c + 1] = fmaf(p[c + 1], vl, z[c + 1]);
      const __nv_bfloat162 h = __floats2bfloat162_rn(p[c] * vs, p[c + 1] * vs);
      w[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(row + (((chunk0 + c8) ^ r7) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// Merge of an item's partials by the CTA that finished it last: contributors in CTA order, a thread
// per 8 lanes of a row (which are 8 neighbouring dims). (Not inlined: its registers are not to press on the tiles'.)
template <int HD>
__device__ __noinline__ void merge_item(const Q4Params& p, const Misc& s, int rows, int c_lo, int c_hi, long long first) {
  constexpr int CPR = HD / 8, RPP = kThreadsQ4 / CPR;  // threads per row, rows at a time
  const int ch = threadIdx.x % CPR;
  constexpr int RP = (kRows + RPP - 1) / RPP;          // rows per thread: side by side, every round trip is paid once
  const int r0 = threadIdx.x / CPR;
  auto slot_of = [&](int c) { return ((uint32_t)c * 2 + (s.bound[c] > first ? 0 : 1)) * kRows; };
  auto pair_of = [&](int c, int r) {
    return c > c_hi || s.bound[c + 1] <= s.bound[c] || r >= rows ? make_float2(-INFINITY, 0.f) : __ldcg(p.part_ml + slot_of(c) + r);
  };
  float2 ml[RP];
  float M[RP], l[RP], acc[RP][8];
#pragma unroll
  for (int u = 0; u < RP; ++u) ml[u] = pair_of(c_lo + ch, r0 + u * RPP);  // a contributor per thread of the row
#pragma unroll
  for (int u = 0; u < RP; ++u) {
    M[u] = ml[u].x;
    for (int cb = c_lo + CPR; cb <= c_hi; cb += CPR) M[u] = fmaxf(M[u], pair_of(cb + ch, r0 + u * RPP).x);
#pragma unroll
    for (int o = CPR / 2; o > 0; o >>= 1) M[u] = fmaxf(M[u], __shfl_xor_sync(0xffffffffu, M[u], o));
    l[u] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[u][e] = 0.f;
  }
#pragma unroll 1
  for (int cb = c_lo; cb <= c_hi; cb += CPR) {
    float wm[RP], lm[RP];
#pragma unroll
    for (int u = 0; u < RP; ++u) {
      if (cb > c_lo) ml[u] = pair_of(cb + ch, r0 + u * RPP);
      wm[u] = ml[u].x == -INFINITY ? 0.f : exp2f(ml[u].x - M[u]);
      lm[u] = wm[u] * ml[u].y;
    }
    const uint32_t off = slot_of(min(cb + ch, c_hi)) * HD;
#pragma unroll 1
    for (int k0 = 0; k0 < CPR && cb + k0 <= c_hi; k0 += 4) {
      float4 x[RP][4], y[RP][4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float* at = p.part_o + __shfl_sync(0xffffffffu, off, k0 + k, CPR) + ch * 8;
#pragma unroll
        for (int u = 0; u < RP; ++u) {
          x[u][k] = __ldcg(reinterpret_cast<const float4*>(at + min(r0 + u * RPP, rows - 1) * HD));
          y[u][k] = __ldcg(reinterpret_cast<const float4*>(at + min(r0 + u * RPP, rows - 1) * HD + 4));
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int u = 0; u < RP; ++u) {
          const float wk = __shfl_sync(0xffffffffu, wm[u], k0 + k, CPR);
          l[u] += __shfl_sync(0xffffffffu, lm[u], k0 + k, CPR);
          if (wk != 0.f) {  // (a contributor that is none, or saw nothing: its place may hold anything)
            acc[u][0] += wk * x[u][k].x; acc[u][1] += wk * x[u][k].y; acc[u][2] += wk * x[u][k].z; acc[u][3] += wk * x[u][k].w;
            acc[u][4] += wk * y[u][k].x; acc[u][5] += wk * y[u][k].y; acc[u][6] += wk * y[u][k].z; acc[u][7] += wk * y[u][k].w;
          }
        }
    }
  }
  // lanes 8 ch + j: dims base + {0, 4, 1, 5, 2, 6, 3, 7}
  const int dim = HD == 128 ? 32 * ((ch & 7) >> 1) + 8 * (2 * (ch >> 3) + (ch & 1)) : 8 * ch;
#pragma unroll
  for (int u = 0; u < RP; ++u) {
    const int r = r0 + u * RPP;
    if (r >= rows) continue;
    const float inv = l[u] == 0.f ? 0.f : 1.f / l[u];
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int a = e < 2 ? 4 * e : 4 * e - 7;  // 0, 4, 1, 5
      const __nv_bfloat162 h = __floats2bfloat162_rn(acc[u][a] * inv, acc[u][a + 2] * inv);
      o[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p.out + s.at[r] + dim) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// New references for the columns of a group of four warps (all of them call), from the tile's largest scores (`p`: the scores, as
// they come); what the columns have gathered (first: nothing yet) follows. An item's first tile, and scores that climb by 2^60.
template <int NH>
__device__ __forceinline__ void move_references(Misc& s, const float (&p)[NH], int cg, int c0, int wg_bar, bool first, uint32_t t_o, float ks,
                                                float kl, uint32_t vm, float (&l)[NH], float (&z)[NH]) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, mine = (int)threadIdx.x & 127;
  {
    float v[32];
#pragma unroll
    for (int c = 0; c < 32; ++c) v[c] = c < NH && ((vm >> c) & 1u) ? fmaf(ks, p[c < NH ? c : 0], kl * s.sq[c0 + (c < NH ? c : 0)]) : -INFINITY;
    const float y = reduce_columns<true>(v);
    if (lane < NH) s.colmax[warp][lane] = y;
  }
  named_sync(wg_bar, 128);
  if (mine < NH) {
    const float nm_old = s.nm[c0 + mine];
    const float mx = fmaxf(fmaxf(s.colmax[cg * 4][mine], s.colmax[cg * 4 + 1][mine]), fmaxf(s.colmax[cg * 4 + 2][mine], s.colmax[cg * 4 + 3][mine]));
    const float nm_new = nm_old == INFINITY || mx + nm_old >= 59.f ? -mx : nm_old;
    s.alpha[c0 + mine] = nm_old == INFINITY || nm_new == nm_old ? 1.f : exp2f(nm_new - nm_old);
    s.nm[c0 + mine] = nm_new;
  }
  named_sync(wg_bar, 128);
  if (first) return;
#pragma unroll 1
  for (int c8 = 0; c8 < NH; c8 += 8) {
    uint32_t o[8];
    tmem_ld8(t_o + c8, o);
    tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * s.alpha[c0 + c8 + e]);
    tmem_st8(t_o + c8, o);
  }
  tmem_wait_st();
#pragma unroll
  for (int c = 0; c < NH; ++c) {
    l[c] *= s.alpha[c0 + c];
    z[c] *= s.alpha[c0 + c];
  }
}

template <int HD, bool kPaged>
__global__ void __launch_bounds__(kThreadsQ4, 2) tree_attn_q4_kernel(const __grid_constant__ Q4Params p) {
  extern __shared__ __align__(1024) unsigned char smem[];
  using LY = Lay<HD>;
  constexpr int W = LY::kW;
  Misc& s = *reinterpret_cast<Misc*>(smem + LY::kSmemMisc);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // Everything, tensor memory included, behind the wait; the warp that allocates releases the dependents after it has.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem)), "n"(kTmemCols));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (lane == 0) {
      mbar_init(&s.bar_s, 1);
      mbar_init(&s.bar_o, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      fence_proxy_async();
    }
    __syncwarp();
  } else if (warp == 0) {
    // the line of tiles
    constexpr int KB = CAST_MAX_BATCH / 32;
    const long long max_pos = p.g.page_size == 0 ? p.g.seq_capacity : (long long)p.g.seq_capacity * p.g.page_size;
    long long run = 0;
    int items = 0;
    int Nv[KB], Lv[KB], Fv[KB], hn[KB], tn[KB], longest = 0;
#pragma unroll
    for (int k = 0; k < KB; ++k) {  // all loads first: one memory round trip
      const int b = k * 32 + lane;
      Nv[k] = b < p.B ? p.n_tree[b] : 0;
      Lv[k] = b < p.B ? p.kv_len[b] : 0;
      Fv[k] = b < p.B && p.first_row != nullptr ? p.first_row[b] : 0;
    }
#pragma unroll
    for (int k = 0; k < KB; ++k) {
      const int b = k * 32 + lane;
      if (Nv[k] > p.Nmax && blockIdx.x == 0) report(p.st, CAST_ERR_BAD_TREE, b);
      const int N = clampi(Nv[k], 0, p.Nmax), F = clampi(Fv[k], 0, N), L = max(Lv[k], 0);
      const bool over = (long long)L + N > max_pos;
      if (over && N > F && blockIdx.x == 0) report(p.st, CAST_ERR_BAD_PAGE, b);
      const int total = (int)(over ? max_pos : (long long)L + N);
      const int nr = ((N - F) * p.G + kRows - 1) / kRows, tl = nr > 0 ? (total + kTile - 1) / kTile : 0;
      const long long mine = (long long)p.Hkv * nr * tl;
      long long upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
      }
      items += __reduce_add_sync(0xffffffffu, p.Hkv * nr);
      s.pre[b] = run + upto - mine;
      run += __shfl_sync(0xffffffffu, upto, 31);
      hn[k] = p.Hkv * nr;
      tn[k] = tl;
      longest = max(longest, __reduce_max_sync(0xffffffffu, tl));
      s.L[b] = L; s.N[b] = N; s.F[b] = F; s.tl[b] = tl; s.nr[b] = nr; s.total[b] = total;
    }
    // Cut item by item where that makes no piece more than three tiles longer than an even cut would: a CTA that works on two items
    // pays the queries, the first references and the handing over twice, as much as three tiles (one sequence of 2048 with 60
    // tokens, cut evenly, had its last partial at 31 us, at 21 cut like this). Pieces of three tiles at least (one, two, four for a
    // sequence of 2048 with 12 tokens: 30, 26, 27 us for 25), no item over more CTAs than a merge is worth.
    const long long even = (run + gridDim.x - 1) / gridDim.x;
    const int q0 = (int)max(max(3ll, even), (long long)((longest + kMaxJoin - 1) / kMaxJoin));
    int q = q0 + 3, ctas = 0;
    auto cut = [&] {
      int sum = 0;
#pragma unroll
      for (int k = 0; k < KB; ++k) sum += hn[k] * ((tn[k] + q - 1) / q);
      ctas = __reduce_add_sync(0xffffffffu, sum);
      return ctas <= (int)gridDim.x;
    };
    const bool fits = cut();
    if (fits) {
#pragma unroll 1
      for (q = q0; q < q0 + 3 && !cut(); ++q) {}
      if (q == q0 + 3) cut();
      int before = 0;
#pragma unroll
      for (int k = 0; k < KB; ++k) {
        const int per = (tn[k] + q - 1) / q, mine = hn[k] * per;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int x = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += x;
        }
        s.cta[k * 32 + lane] = before + upto - mine;
        s.per[k * 32 + lane] = per;
        before += __shfl_sync(0xffffffffu, upto, 31);
      }
    }
    if (lane == 0) {
      s.pre[CAST_MAX_BATCH] = run;
      s.whole = fits;
      // (else:) the same for an even cut, but no fewer pieces than items, which cost as much as three tiles whatever their length (64
      // sequences of 20 to 100, 12 tokens: 39 us per layer, 28)
      long long workers = max((run + 2) / 3, (long long)items);
      workers = workers < (long long)items * kMaxJoin ? workers : (long long)items * kMaxJoin;
      workers = workers < (long long)gridDim.x ? workers : (long long)gridDim.x;
      s.workers = fits ? ctas : (int)workers;
      s.piece = workers > 0 ? run / workers : 0;
      s.rest = workers > 0 ? (int)(run - s.piece * workers) : 0;
    }
  }
  __syncthreads();
  // where the pieces begin
  for (int c = tid; c <= (int)gridDim.x; c += kThreadsQ4) {
    const long long T = s.pre[CAST_MAX_BATCH];
    long long x = T;
    if (c < s.workers) {
      x = s.piece * c + min(c, s.rest);
      if (s.whole) {
        int b = 0;  // the last sequence that starts at or before c (one without tiles starts where the next does)
#pragma unroll
        for (int o = CAST_MAX_BATCH / 2; o > 0; o >>= 1) b += s.cta[b + o] <= c ? o : 0;
        const int in = c - s.cta[b], item = in / s.per[b], k = in - item * s.per[b];
        x = s.pre[b] + (long long)item * s.tl[b] + (int)((long long)k * s.tl[b] / s.per[b]);
      }
    }
    s.bound[c] = x;
    if (c == (int)blockIdx.x && x < T) {
      int b = 0;
      while (s.pre[b + 1] <= x) ++b;
      const long long in = x - s.pre[b];
      const int hr = in <= 0x7fffffffll ? (int)((uint32_t)in / (uint32_t)s.tl[b]) : (int)(in / s.tl[b]);
      s.seg.b = b;
      s.seg.h = hr / s.nr[b];
      s.seg.rb = hr - s.seg.h * s.nr[b];
      s.seg.t = (int)(in - (long long)hr * s.tl[b]);
    }
  }
  auto look_ahead = [&](int i) {  // (thread 0) tile i into `step`
    Walk w = s.ahead;
    s.step[i & 7] = make_int4(w.b, w.h, w.t * kTile, s.total[w.b]);
    advance(w, s, p);
    s.ahead = w;
  };
  const bool aligned = (smem_u32(smem) & 1023u) == 0u;  // the swizzled operand regions need a 1 KB aligned base
  __syncthreads();
  if (tid == 0) {
    if (!aligned) report(p.st, CAST_ERR_CUDA, 1024);
    s.seg.left = aligned ? (int)(s.bound[blockIdx.x + 1] - s.bound[blockIdx.x]) : 0;
    s.ahead = s.seg;
    if (s.seg.left > 0)
      for (int i = 0; i < 4; ++i) look_ahead(i);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __reduce_or_sync(0xffffffffu, s.tmem);

  const int part = warp & 3, cg = warp >> 2, wg_bar = 1 + cg;     // lanes of tensor memory, half of the columns
  const int posl = part * 32 + lane;                              // this thread's position in a tile
  const int r = lane >> 2, tq = lane & 3, row16 = part * 32 + cg * 16 + r;  // its quad's rows of the codes: row16 and row16 + 8
  const uint32_t t_part = (uint32_t)(part * 32) << 16;

  // ---- codes and pairs, a tile ahead. Every lane finds the place of its position's row; a quad of lanes loads a row of codes.
  uint32_t kc[2][W], vc[2][W], nkr = 0, nvr = 0;
  // Of the tile whose K codes are in kc, and of that in vc: this thread's position has a row. (The codes of one without may be
  // anything: they are finite, and weigh nothing.)
  bool live_k = false, live_v = false;
  int page = 0;
  uint32_t row = 0;                // of the tile in kc
  auto next_page = [&](int i) {
    const int4 e = s.step[i & 7];
    page = request_page<kPaged>(p.g, e.x, e.z + posl, e.w);
  };
  auto next_row = [&](int i) {
    const int4 e = s.step[i & 7];
    row = row_of<kPaged>(p.g, page, e.y, e.z + posl, e.w);
    const bool fine = page_ok<kPaged>(p.g, page);
    if (kPaged && !fine && e.z + posl < e.w) report(p.st, CAST_ERR_BAD_PAGE, e.x);
    live_k = fine && e.z + posl < e.w;
  };
  auto request = [&](const unsigned char* codes, uint32_t (&c)[2][W]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const unsigned char* at = codes + (size_t)__shfl_sync(0xffffffffu, row, cg * 16 + 8 * j + r) * (HD / 2) + tq * (4 * W);
      ld_here(c[j], at);
    }
  };
  // K codes (in kc) to tensor memory
  auto store_k = [&](bool ok) {
    if (ok) {
#pragma unroll
      for (int i = 0; i < W; ++i) {  // word i's pairs 0, 1 go to the group of 16 dims 2 i, pairs 2, 3 to 2 i + 1
        const uint32_t a = kc[0][i], c = kc[1][i];
        const uint32_t out[8] = {pair_plus16<0>(a), pair_plus16<1>(a), pair_plus16<0>(c), pair_plus16<1>(c),
                                 pair_plus16<2>(a), pair_plus16<3>(a), pair_plus16<2>(c), pair_plus16<3>(c)};
        tmem_st_quads<2>(tmem + kTmemK + 16 * i + ((uint32_t)(part * 32 + cg * 16) << 16), out);
      }
    }
    if (ok) tmem_wait_st();
  };
  unsigned char* const v_row = smem + LY::kSmemV + row16 * 128;
  const int chunk[2] = {((2 * tq) ^ r) << 4, ((2 * tq + 1) ^ r) << 4};
  // V codes of the tile in vc to shared memory; the tile behind it (whose row is `row`) requested
  auto store_v = [&](int buf, bool ok) {
    if (ok) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const uint32_t c = vc[j][i];
          *reinterpret_cast<uint4*>(v_row + buf * LY::kBufV + (W == 4 ? i >> 1 : 0) * LY::kRegionV + j * 1024 + chunk[i & 1]) =
              make_uint4(pair_minus8<0>(c), pair_minus8<1>(c), pair_minus8<2>(c), pair_minus8<3>(c));
        }
    }
    request(p.vc, vc);
  };
  auto request_pair = [&] {
    nkr = ld_here(reinterpret_cast<const int32_t*>(p.kr) + row);
    nvr = ld_here(reinterpret_cast<const int32_t*>(p.vr) + row);
  };
  if (s.seg.left > 0) {
    next_page(0);
    next_row(0);
    next_page(1);
    request(p.kc, kc);
    request(p.vc, vc);
    request_pair();
    live_v = live_k;
  }

  // ---- the products: one warp, converged
  auto issue_s = [&](uint32_t shape) {
    const uint64_t dq = umma_desc(smem_u32(smem + LY::kSmemQ), 16, 1024);
#pragma unroll
    for (int k = 0; k < HD / 16; ++k)
      umma_bf16_ts(tmem + kTmemS, tmem + kTmemK + k * 8, dq + (uint64_t)((k >> 2) * (LY::kRegionQ >> 4) + (k & 3) * 2), shape, k > 0);
    umma_commit(&s.bar_s);
  };
  auto issue_o = [&](uint32_t shape, int buf, bool first) {
    // both operands are MN-major; 64 dims: both halves of M alike
    const uint64_t dv = umma_desc(smem_u32(smem + LY::kSmemV + buf * LY::kBufV), HD == 128 ? LY::kRegionV : 0, 1024);
    const uint64_t dp = umma_desc(smem_u32(smem + LY::kSmemP), 0, 1024);
#pragma unroll
    for (int k = 0; k < kTile / 16; ++k)
      umma_bf16(tmem + kTmemO, dv + (uint64_t)(k * (2048 >> 4)), dp + (uint64_t)(k * (2048 >> 4)), shape | (1u << 15) | (1u << 16),
                !first || k > 0 ? 1u : 0u);
    umma_commit(&s.bar_o);
  };

  int it = 0;
  bool ok = true;
  // One item, or what this CTA has of it; NH columns to a thread.
  auto work = [&](auto nh_c) {
    constexpr int NH = decltype(nh_c)::value;
    const int t0 = s.seg.t, n = min(s.seg.left, s.tl[s.seg.b] - t0), L = s.L[s.seg.b];
    const int rows_all = (s.N[s.seg.b] - s.F[s.seg.b]) * p.G - s.seg.rb * kRows, c0 = cg * NH;
    constexpr uint32_t shape = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(NH >> 2) << 17) | ((uint32_t)(kTile >> 4) << 24);
    // ---- the query rows, their dims in the order of the codes in tensor memory; their sums
    if (tid < kRows) {
      const int b = s.seg.b, grow = s.F[b] * p.G + s.seg.rb * kRows + tid, tok = grow / p.G;
      s.at[tid] = (uint32_t)(((b * p.Ncap + tok) * p.Hq + s.seg.h * p.G + (grow - tok * p.G)) * HD);
      s.nm[tid] = tid < rows_all ? INFINITY : 0.f;
    }
    __syncthreads();
    {
      constexpr int VPR = HD / 8, STEPS = kRows * VPR / kThreadsQ4;
      static_assert(kRows * VPR % kThreadsQ4 == 0 || HD == 64, "whole steps");
      uint4 x[STEPS + (HD == 64 ? 1 : 0)];
#pragma unroll
      for (int k = 0; k * kThreadsQ4 < kRows * VPR; ++k) {
        const int i = tid + k * kThreadsQ4, qr = i / VPR, v = i % VPR;
        x[k] = qr < min(rows_all, kRows) ? __ldg(reinterpret_cast<const uint4*>(p.q + s.at[qr] + v * 8)) : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int k = 0; k * kThreadsQ4 < kRows * VPR; ++k) {
        const int i = tid + k * kThreadsQ4, qr = i / VPR, v = i % VPR, t = v / W, wd = v % W;
        if (qr >= kRows) break;  // (whole warps: half of the last step at 64 dims)
        float f[8], sum = 0.f;
        Vec<__nv_bfloat16>::unpack(x[k], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += f[e];
#pragma unroll
        for (int o = VPR / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (v == 0) s.sq[qr] = sum;
        // dims 0, 4, 1, 5 and 2, 6, 3, 7 of the eight
        const uint2 lo = make_uint2(__byte_perm(x[k].x, x[k].z, 0x5410), __byte_perm(x[k].x, x[k].z, 0x7632));
        const uint2 hi = make_uint2(__byte_perm(x[k].y, x[k].w, 0x5410), __byte_perm(x[k].y, x[k].w, 0x7632));
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int g = 2 * wd + half, ch = 2 * (g & 3) + (t >> 1);
          *reinterpret_cast<uint2*>(smem + LY::kSmemQ + (g >> 2) * LY::kRegionQ + swz(qr, ch) + 8 * (t & 1)) = half ? hi : lo;
        }
      }
    }
    const bool tail = (t0 + n) * kTile > L;
    if (tail) {  // which columns see which tree token: 32 x 32 bits a warp, turned by votes
      const int b = s.seg.b, N = s.N[b], grow0 = s.F[b] * p.G + s.seg.rb * kRows, rows = min(rows_all, kRows);
      const int ch = warp & 1, wd = warp >> 1, qr = ch * 32 + lane;
      uint32_t bits = 0u;
      if (qr < rows && wd < p.words) {
        bits = __ldg(p.anc + ((size_t)b * p.Ncap + (grow0 + qr) / p.G) * p.words + wd);
        const int last = N - wd * 32;
        bits = last >= 32 ? bits : last > 0 ? bits & ((1u << last) - 1u) : 0u;
      }
      uint32_t mine = 0u;
#pragma unroll 8
      for (int j = 0; j < 32; ++j) {
        const uint32_t v = __ballot_sync(0xffffffffu, (bits >> j) & 1u);
        if (lane == j) mine = v;
      }
      s.vis[ch][wd * 32 + lane] = mine;
    }
    store_k(ok);
    fence_proxy_async();
    tc_fence_before();
    __syncthreads();
    if (warp == 0 && ok) {
      tc_fence_after();
      issue_s(shape);
    }

    float l[NH], z[NH];
#pragma unroll
    for (int c = 0; c < NH; ++c) l[c] = z[c] = 0.f;
    constexpr uint32_t full = (1u << NH) - 1u;
#pragma unroll 1
    for (int i = 0; i < n; ++i, ++it) {
      const uint32_t phase = (uint32_t)it & 1u;
      // this tile's pair and rows without a place (those of `row` are the next tile's by now)
      const float st_k = q4_step(nkr), st_v = q4_step(nvr);
      const bool live = live_v;
      // (a V row without a finite value: the scores become NaN, for the columns that see them; 0 * NaN would reach the others)
      const float mid_v = fmaf(8.f, st_v, q4_low(nvr));
      const bool sound = fabsf(mid_v) < INFINITY;
      const float ks = live ? p.scale_log2 * (sound ? st_k : mid_v - mid_v) : 0.f;
      const float kl = live ? p.scale_log2 * fmaf(-16.f, st_k, q4_low(nkr)) : 0.f;
      const float vs = live && sound ? st_v : 0.f, vl = live && sound ? mid_v : 0.f;
      // ---- V codes (the buffer's last reader was O^T of tile it - 2, awaited with the tile before), and all requests for the tile
      // behind: the fence at this one's end waits for them, so they go out first thing (behind it, a K request cost a memory latency)
      next_row(it + 1);
      request(p.kc, kc);
      request_pair();
      store_v(it & 1, ok);
      next_page(it + 2);
      live_v = live_k;
      uint32_t vm = live ? full : 0u;
      if (tail) {
        const int j = (t0 + i) * kTile + posl - L;
        if (j >= 0 && live) vm = (uint32_t)(((unsigned long long)s.vis[0][j] | ((unsigned long long)s.vis[1][j] << 32)) >> c0) & full;
      }
      const bool plain = __all_sync(0xffffffffu, vm == full);
      // ---- the scores, and the place of the weights (O^T of the tile before has read its own)
      if (ok) {
        ok = mbar_wait(&s.bar_s, phase) && (it == 0 || mbar_wait(&s.bar_o, phase ^ 1u));
        if (!ok && lane == 0) report(p.st, CAST_ERR_TIMEOUT, s.seg.b);
      }
      float pr[NH];
      tc_fence_after();
      const uint32_t t_s = tmem + kTmemS + c0 + t_part;
      auto to_weights = [&] {
        weights<NH>(pr, s.sq + c0, s.nm + c0, ks, kl);
        if (!plain) mask_weights<NH>(pr, vm);
      };
      bool far = false;
      if (ok) {
        read_scores<NH>(t_s, pr);
        if (i > 0) {
          to_weights();
          float top = 0.f;
#pragma unroll
          for (int c = 0; c < NH; c += 2) top = max3(top, pr[c], pr[c + 1]);
          far = top >= kFar;
        }
      }
      // The first tile, a column without a reference yet, or a weight far above it: the tile's maxima decide, in all four warps
      // of the columns. (O^T is at rest.)
      if (i == 0 || named_or(wg_bar, 128, !ok || far)) {
        if (named_or(wg_bar, 128, !ok)) ok = false;
        if (ok) {
          if (i > 0) read_scores<NH>(t_s, pr);
          move_references<NH>(s, pr, cg, c0, wg_bar, i == 0, tmem + kTmemO + c0 + t_part, ks, kl, vm, l, z);
          to_weights();
        }
      }
      if (ok) {
        unsigned char* p_row = smem + LY::kSmemP + posl * 128;
        hand_over<NH>(pr, l, z, p_row, posl & 7, c0 >> 3, vs, vl);
      }
      if (i + 1 < n) store_k(ok);  // (S^T of this tile has read the codes before)
      if (tid == 0) look_ahead(it + 4);
      fence_proxy_async();
      tc_fence_before();
      if (__syncthreads_or(!ok)) ok = false;
      if (warp == __reduce_max_sync(0xffffffffu, it & 7) && ok) {  // in turn: sixteen instructions and their descriptors are a lot for one warp
        tc_fence_after();
        if (i + 1 < n) issue_s(shape);
        issue_o(shape, it & 1, i == 0);
      }
    }

    // ---- the item's end: sums over the lanes, then over the warps of a column
    {
      float v[32];
#pragma unroll
      for (int c = 0; c < 32; ++c) v[c] = c < NH ? l[c < NH ? c : 0] : 0.f;
      const float suml = reduce_columns<false>(v);
#pragma unroll
      for (int c = 0; c < 32; ++c) v[c] = c < NH ? z[c < NH ? c : 0] : 0.f;
      const float sumz = reduce_columns<false>(v);
      if (lane < NH) {
        s.red_l[part][c0 + lane] = suml;
        s.red_z[part][c0 + lane] = sumz;
      }
    }
    if (ok) {
      ok = mbar_wait(&s.bar_o, (uint32_t)(it - 1) & 1u);
      if (!ok && lane == 0) report(p.st, CAST_ERR_TIMEOUT, s.seg.b);
    }
    named_sync(wg_bar, 128);
    if ((tid & 127) < NH) {
      const int c = c0 + (tid & 127);
      const float lt = s.red_l[0][c] + s.red_l[1][c] + s.red_l[2][c] + s.red_l[3][c];
      s.tot_l[c] = n < s.tl[s.seg.b] ? lt : lt == 0.f ? 0.f : 1.f / lt;  // a whole item: its reciprocal
      s.tot_z[c] = s.red_z[0][c] + s.red_z[1][c] + s.red_z[2][c] + s.red_z[3][c];
    }
    named_sync(wg_bar, 128);
    const int b = s.seg.b, h = s.seg.h, rb = s.seg.rb, tl = s.tl[b], rows = min(rows_all, kRows);
    const bool whole = n == tl;
    const long long first = s.pre[b] + (long long)(h * s.nr[b] + rb) * tl;  // the item's first tile
    // lane m of O^T: dims in the order of merge_item
    const int ch = posl >> 3, j8 = posl & 7;
    const int dim = (HD == 128 ? 32 * ((ch & 7) >> 1) + 8 * (2 * (ch >> 3) + (ch & 1)) : 8 * ch) + ((j8 >> 1) | ((j8 & 1) << 2));
    const int slot = (int)blockIdx.x * 2 + (s.bound[blockIdx.x] > first ? 0 : 1);
    if (ok) {
      tc_fence_after();
      float o[NH];
      read_scores<NH>(tmem + kTmemO + c0 + t_part, o);
      if (HD == 128 || posl < 64) {
        float* const part_row = p.part_o + (size_t)slot * kRows * HD + posl;
#pragma unroll
        for (int c = 0; c < NH; ++c) {
          const float x = o[c] + s.tot_z[c0 + c];
          if (c0 + c < rows) {
            if (whole) p.out[s.at[c0 + c] + dim] = __float2bfloat16_rn(x * s.tot_l[c0 + c]);
            else __stcg(part_row + (c0 + c) * HD, x);
          }
        }
      }
    }
    tc_fence_before();
    if (!whole) {
      if ((tid & 127) < NH) {
        const int c = c0 + (tid & 127);
        const float lt = s.tot_l[c];  // (NaN: its own reference may be none, and must not let the merge pass it over)
        __stcg(p.part_ml + (size_t)slot * kRows + c, ok ? make_float2(lt == lt ? -s.nm[c] : INFINITY, lt) : make_float2(-INFINITY, 0.f));
      }
      // the CTAs that share the item
      const long long end = first + tl;
      int c_lo = blockIdx.x, c_hi = blockIdx.x;
      while (s.bound[c_lo] > first) --c_lo;
      while (s.bound[c_hi + 1] < end) ++c_hi;
      __syncthreads();
      if (tid == 0) {
        int parts = 0;
        for (int c = c_lo; c <= c_hi; ++c) parts += s.bound[c + 1] > s.bound[c];
        // releases this CTA's partial (the barrier made it this thread's to release), acquires those that came earlier
        int32_t* cnt = p.ticket + ((size_t)b * p.Hkv + h) * p.nrb + rb;
        int t;
        asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(t) : "l"(cnt) : "memory");
        s.last = t == parts - 1;
        if (t == parts - 1) *cnt = 0;  // ready for the next launch
      }
      __syncthreads();
      if (s.last) merge_item<HD>(p, s, rows, c_lo, c_hi, first);
    }
    __syncthreads();  // (all are done with the item's arrays)
    if (tid == 0) {
      Walk w = s.seg;
      w.t += n - 1;
      w.left -= n - 1;
      advance(w, s, p);
      s.seg = w;
    }
    __syncthreads();
  };
#pragma unroll 1
  while (s.seg.left > 0) {  // up to 16 query rows, or up to 48: with the count known the columns' arithmetic is one straight block
    if ((s.N[s.seg.b] - s.F[s.seg.b]) * p.G - s.seg.rb * kRows <= 16) work(Count<8>());
    else work(Count<kHalf>());
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemCols));
}

constexpr size_t kPartBytes = (size_t)2 * kRows * (128 * sizeof(float) + sizeof(float2));  // per CTA

int q4_grid(const cast_ctx* c) { return 2 * c->num_sms < kMaxGrid ? 2 * c->num_sms : kMaxGrid; }
int q4_row_blocks(const cast_ctx* c, int Hq, int Hkv) { return (c->cfg.total_token * (Hq / Hkv) + kRows - 1) / kRows; }

}  // namespace

// The partials (of a size that no shape changes) come first, the tickets behind them: those start at zero, and every merge leaves
// its own at zero again, whatever the shape of the call.
cast_status tree_attention_q4_reserve(cast_ctx* c, int B, int Hq, int Hkv) {
  const size_t need = q4_grid(c) * kPartBytes + (size_t)B * Hkv * q4_row_blocks(c, Hq, Hkv) * sizeof(int32_t);
  return grow_workspace(&c->q4_ws, &c->q4_ws_bytes, need, need);
}

cast_status tree_attention_q4_launch(cast_ctx* c, const void* q, const void* k_codes, const void* k_range, const void* v_codes,
                                     const void* v_range, int B, int Hq, int Hkv, int D, const Paging& g, const int32_t* kv_len,
                                     const uint32_t* anc, const int32_t* n_tree, const int32_t* first_row, float scale, void* out,
                                     cudaStream_t stream) {
  const int grid = q4_grid(c);
  // elements of q are counted in 31 bits, rows of the cache in 32: more would not fit the device's memory
  if ((long long)B * c->cfg.max_tree * Hq * D > 0x7fffffffll) return CAST_ERR_CAPACITY;
  Q4Params p;
  if (!fast_paging(g, B, Hkv, &p.g)) return CAST_ERR_CAPACITY;
  p.nrb = q4_row_blocks(c, Hq, Hkv);
  // compute calls never allocate: the workspace comes from cast_reserve_attention_q4
  if (grid * kPartBytes + (size_t)B * Hkv * p.nrb * sizeof(int32_t) > c->q4_ws_bytes) return CAST_ERR_CAPACITY;
  p.q = (const __nv_bfloat16*)q; p.out = (__nv_bfloat16*)out;
  p.kc = (const unsigned char*)k_codes; p.vc = (const unsigned char*)v_codes;
  p.kr = (const uint32_t*)k_range; p.vr = (const uint32_t*)v_range;
  p.B = B; p.Ncap = c->cfg.max_tree; p.Nmax = c->cfg.total_token; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv; p.words = c->words;
  p.kv_len = kv_len; p.n_tree = n_tree; p.first_row = first_row; p.anc = anc;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.part_o = (float*)c->q4_ws;
  p.part_ml = (float2*)(p.part_o + (size_t)grid * 2 * kRows * 128);
  p.ticket = (int32_t*)((char*)c->q4_ws + grid * kPartBytes);
  p.st = c->state;
  auto* const kern = D == 64 ? (g.page_size > 0 ? tree_attn_q4_kernel<64, true> : tree_attn_q4_kernel<64, false>)
                             : (g.page_size > 0 ? tree_attn_q4_kernel<128, true> : tree_attn_q4_kernel<128, false>);
  const int smem = (D == 64 ? Lay<64>::kSmemMisc : Lay<128>::kSmemMisc) + (int)sizeof(Misc);
  CAST_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  CAST_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, 100));  // two CTAs per SM
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(kThreadsQ4, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // launched while its predecessor drains; waits for it
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kern, p) != cudaSuccess) {
    cudaGetLastError();
    return CAST_ERR_CUDA;
  }
  return CAST_OK;
}

}  // namespace cast
