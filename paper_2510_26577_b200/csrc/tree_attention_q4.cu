// Tensor-core path of cast_tree_attention_q4: bf16 queries over the 4-bit cache (sm_100a: tcgen05 + TMEM).
//
// With step and low of a row taken out of the products, the codes themselves enter the matrix units, exactly, as small
// integers in bf16:
//   q . k_p = step_p (q . c_p) + low_p sum(q)        sum_p w_p v_p = sum_p (w_p step_p) (c_p - 8) + sum_p w_p (low_p + 8 step_p)
// so a score carries no rounding but the accumulation's, and a weight (times its row's step) one to bf16; the last sum stays in fp32.
//
// Positions are the rows of both products, queries the columns: S^T = C_k Q^T (128 positions x N queries) and
// O^T = C_v^T P^T (dims x N). A query column is a (tree token, head of the GQA group) pair, up to 64 per work item, N rounded up to
// 16: a small tree costs what it has, not a block of 128 rows, and its exponentials spread over all lanes. A thread of the softmax
// owns one position: step and low are scalars of its own, masks are one word per position, and sums run in registers over
// all its tiles, reduced across lanes once per item. What is paid for that: the maximum of a column lies across lanes, so the
// running reference of a column is not its maximum but the first visible tile's, moved when a weight reaches 2^60 (bf16 and fp32 have
// the range), which one vote per tile finds.
//
// Roles of a CTA's 17 warps (one CTA per SM):
//   K producers (4): codes from global memory to registers two tiles ahead, unpacked to 16 + c, written to tensor memory as the
//                    A operand (the dims in the order the quad of lanes holds them; Q is staged in the same order)
//   V producers (4): the same codes to c - 8, 128-byte-swizzled rows in shared memory, the MN-major A operand as they lie
//   MMA issuer (1) : S^T of tile i+1 before O^T of tile i
//   softmax (8)    : two groups of four warps, a half of the columns each
// Work is one line of tiles, item after item (sequence, kv-head, block of 64 rows), cut into equal pieces, one per CTA: ragged
// batches load the machine evenly. An item that lies across CTAs leaves partials in the workspace; the last CTA to finish it
// (an atomic ticket, nothing spins) merges them in CTA order. All mbarrier waits are bounded: on expiry the CTA records
// CAST_ERR_TIMEOUT, stops touching the operands and runs out.
#include <math.h>

#include "kv_q4.h"
#include "tc_ptx.h"

namespace cast {

namespace {

constexpr int kTile = 128;       // positions per tile (UMMA M)
constexpr int kRows = 64;        // query columns per item at most (UMMA N)
constexpr int kSoftThreads = 256;
constexpr int kWarpK = 8, kWarpV = 12, kWarpMma = 16;
constexpr int kThreadsQ4 = 640;  // (registers are allotted per four warps: the issuer's group has three idle ones)
// Registers per thread: 96 at launch (640 threads), then the groups of four warps take what they need of the 61440.
constexpr int kRegsSoft = 136, kRegsProduce = 88, kRegsIssue = 24;
static_assert(256 * kRegsSoft + 256 * kRegsProduce + 128 * kRegsIssue <= 640 * 96, "the shares add up to no more than the launch has");
constexpr int kAhead = 2;        // tiles of codes in registers ahead of the one in work
constexpr int kMaxGrid = 256;
constexpr int kMaxJoin = 32;     // CTAs that share an item, about
constexpr float kFar = 1.15292150460684698e18f;  // 2^60

struct Q4Params {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  const unsigned char *kc, *vc;
  const uint32_t *kr, *vr;
  int B, Ncap, Nmax, Hq, Hkv, G, words;
  Paging g;
  uint32_t page_mul;  // position / page_size = position * page_mul >> page_shift
  int page_shift;
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
  static constexpr int kSmemQ = 0;                   // HD / 64 regions [64 rows][64] bf16
  static constexpr int kRegionQ = kRows * 128;
  static constexpr int kSmemV = kSmemQ + HD / 64 * kRegionQ;
  static constexpr int kRegionV = kTile * 128;       // [128 positions][64] bf16
  static constexpr int kBufV = HD / 64 * kRegionV;
  static constexpr int kSmemP = kSmemV + 2 * kBufV;  // [128 positions][64 rows] bf16
  static constexpr int kBufP = kTile * 128;
  static constexpr int kSmemMisc = kSmemP + 2 * kBufP;
};

struct Misc {
  uint64_t bar_ka[2], bar_s[2], bar_v[2], bar_p[2], bar_o[2], bar_q;
  uint32_t tmem;
  int last;
  long long pre[CAST_MAX_BATCH + 1];   // tiles of the sequences before
  long long bound[kMaxGrid + 1];       // first tile of every CTA
  int L[CAST_MAX_BATCH], N[CAST_MAX_BATCH], F[CAST_MAX_BATCH], tl[CAST_MAX_BATCH], nr[CAST_MAX_BATCH], total[CAST_MAX_BATCH];
  int workers;
  int b0, hr0, t0;                     // where this CTA starts
  alignas(16) float sq[kRows];         // sums of the query rows
  alignas(16) float m[kRows];          // references, log2 units; -inf: none yet
  alignas(16) float tot_l[kRows];
  alignas(16) float tot_z[kRows];
  float red_l[4][kRows], red_z[4][kRows];
  float colmax[8][kRows / 2];
  uint32_t vis[2][CAST_MAX_TREE];      // columns (32 + 32) that see a tree token
};

constexpr int kTmemK = 0, kTmemS = 128, kTmemO = 256, kTmemCols = 512;  // K codes 2 x 64, scores 2 x 64, output 64 (of 512: one CTA per SM)

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
  if constexpr (C == 8)
    asm volatile(
        "tcgen05.st.sync.aligned.16x256b.x8.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
          "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
          "r"(r[30]), "r"(r[31])
        : "memory");
  else
    asm volatile(
        "tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ unsigned long long mul_f2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Codes i and i + 4 of a word (its nibbles) as a pair of bf16. 16 + c: the code in the upper mantissa bits of 16, whose step is 1 / 8
// there and 1 with the code three bits up. 128 + c: the code in the lowest bits.
template <int I>
__device__ __forceinline__ uint32_t pair_plus16(uint32_t w) {
  const uint32_t s = I == 0 ? w << 3 : I == 1 ? w >> 1 : I == 2 ? w >> 5 : w >> 9;
  return (s & 0x00780078u) | 0x41804180u;
}
template <int I>
__device__ __forceinline__ uint32_t pair_minus8(uint32_t w) {
  const uint32_t x = ((w >> (4 * I)) & 0x000f000fu) | 0x43004300u;
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), __floats2bfloat162_rn(136.f, 136.f));  // exact
  return *reinterpret_cast<const uint32_t*>(&d);
}

// A place on the line of tiles.
struct Walk {
  int b, hr, t;   // sequence, kv-head * row blocks + row block, tile of the item
  int left;       // tiles from here to the end of the CTA's piece, this one included
};
__device__ __forceinline__ void advance(Walk& w, const Misc& s, const Q4Params& p) {
  --w.left;
  if (++w.t < s.tl[w.b] || w.left <= 0) return;
  w.t = 0;
  if (++w.hr < p.Hkv * s.nr[w.b]) return;
  w.hr = 0;
  do ++w.b;
  while (s.tl[w.b] == 0);  // (tiles are left, so a sequence with tiles follows)
}

// Page of a position (-1: none, or an id out of range) and its row among the 4-bit rows.
__device__ __forceinline__ int page_of(const Q4Params& p, int b, int pos, int total) {
  if (pos >= total) return -1;
  if (p.g.page_size == 0) return b;
  const int id = p.g.table[(size_t)b * p.g.seq_capacity + (int)(((uint64_t)(uint32_t)pos * p.page_mul) >> p.page_shift)];
  return id < 0 || id >= p.g.num_pages ? -2 : id;
}
__device__ __forceinline__ long long row_of(const Q4Params& p, int page, int h, int pos) {
  const int ps = p.g.page_size;
  if (ps == 0) return ((long long)page * p.Hkv + h) * p.g.seq_capacity + pos;
  return ((long long)page * p.Hkv + h) * ps + (pos - (int)(((uint64_t)(uint32_t)pos * p.page_mul) >> p.page_shift) * ps);
}

// A column's two sums over the 32 lanes, for 32 columns: lane l returns column l's.
__device__ __forceinline__ float reduce_columns(float (&v)[32]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const bool up = (lane & o) != 0;
      const float mine = up ? v[i + o] : v[i], other = up ? v[i] : v[i + o];
      v[i] = mine + __shfl_xor_sync(0xffffffffu, other, o);
    }
  }
  return v[0];
}

// ---- producers: kV = false: K codes to tensor memory; true: V codes to shared memory
template <int HD, bool kV>
__device__ __forceinline__ void produce(const Q4Params& p, Misc& s, unsigned char* smem, Walk start, uint32_t tmem) {
  using LY = Lay<HD>;
  constexpr int W = LY::kW;
  const int lane = threadIdx.x & 31, pw = ((int)threadIdx.x >> 5) & 3, r = lane >> 2, tq = lane & 3;
  uint32_t code[kAhead][4][W];
  int page[kAhead][4];
  Walk wi = start, wc = start;
  auto load_pages = [&](int (&pg)[4]) {
    if (wi.left <= 0) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) pg[j] = page_of(p, wi.b, wi.t * kTile + pw * 32 + 8 * j + r, s.total[wi.b]);
    advance(wi, s, p);
  };
  auto load_codes = [&](uint32_t (&c)[4][W], const int (&pg)[4]) {
    if (wc.left <= 0) return;
    const int h = wc.hr / s.nr[wc.b];
    const unsigned char* base = (kV ? p.vc : p.kc) + tq * (4 * W);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
#pragma unroll
      for (int w = 0; w < W; ++w) c[j][w] = 0u;
      if (pg[j] >= 0) {
        const unsigned char* at = base + row_of(p, pg[j], h, wc.t * kTile + pw * 32 + 8 * j + r) * (HD / 2);
        if constexpr (W == 4) {
          const uint4 x = __ldg(reinterpret_cast<const uint4*>(at));
          c[j][0] = x.x; c[j][1] = x.y; c[j][2] = x.z; c[j][3] = x.w;
        } else {
          const uint2 x = __ldg(reinterpret_cast<const uint2*>(at));
          c[j][0] = x.x; c[j][1] = x.y;
        }
      } else if (!kV && pg[j] == -2 && tq == 0) {
        report(p.st, CAST_ERR_BAD_PAGE, wc.b);
      }
    }
    advance(wc, s, p);
  };
#pragma unroll
  for (int d = 0; d < kAhead; ++d) load_pages(page[d]);
#pragma unroll
  for (int d = 0; d < kAhead; ++d) load_codes(code[d], page[d]);
#pragma unroll
  for (int d = 0; d < kAhead; ++d) load_pages(page[d]);
  bool ok = true;
  for (int it0 = 0; it0 < start.left; it0 += kAhead) {
#pragma unroll
    for (int d = 0; d < kAhead; ++d) {
      const int it = it0 + d;
      if (it >= start.left) break;
      static_assert(kAhead == 2, "buffer d is tile it's");
      // the buffer's last reader: S^T (K) or O^T (V) of tile it - 2
      if (it >= 2 && ok) {
        ok = mbar_wait(kV ? &s.bar_o[d] : &s.bar_s[d], (uint32_t)(((it >> 1) - 1) & 1));
        if (!ok && lane == 0) report(p.st, CAST_ERR_TIMEOUT, start.b);
      }
      if (ok) {
        if constexpr (kV) {
          unsigned char* buf = smem + LY::kSmemV + d * LY::kBufV;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int row = pw * 32 + 8 * j + r;
#pragma unroll
            for (int w = 0; w < W; ++w) {
              const uint32_t c = code[d][j][w];
              const int region = W == 4 ? w >> 1 : 0, chunk = 2 * tq + (w & 1);
              *reinterpret_cast<uint4*>(buf + region * LY::kRegionV + swz(row, chunk)) =
                  make_uint4(pair_minus8<0>(c), pair_minus8<1>(c), pair_minus8<2>(c), pair_minus8<3>(c));
            }
          }
          fence_proxy_async();
        } else {
          tc_fence_after();
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            uint32_t out[8 * W];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int w = 0; w < W; ++w) {  // word w's pairs 0, 1 go to the group of 16 dims 2 w, pairs 2, 3 to 2 w + 1
                const uint32_t c = code[d][2 * hf + j][w];
                out[8 * w + 2 * j] = pair_plus16<0>(c);
                out[8 * w + 2 * j + 1] = pair_plus16<1>(c);
                out[8 * w + 4 + 2 * j] = pair_plus16<2>(c);
                out[8 * w + 4 + 2 * j + 1] = pair_plus16<3>(c);
              }
            tmem_st_quads<2 * W>(tmem + kTmemK + d * 64 + ((uint32_t)(pw * 32 + hf * 16) << 16), out);
          }
          tmem_wait_st();
          tc_fence_before();
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(kV ? &s.bar_v[d] : &s.bar_ka[d]);
      load_codes(code[d], page[d]);
      load_pages(page[d]);
    }
  }
}

// ---- the MMA issuer (the whole warp, converged)
template <int HD>
__device__ __forceinline__ void issue(const Q4Params& p, Misc& s, unsigned char* smem, Walk w, uint32_t tmem) {
  using LY = Lay<HD>;
  const uint32_t tm = __reduce_or_sync(0xffffffffu, tmem);
  const uint64_t dq = umma_desc(smem_u32(smem + LY::kSmemQ), 16, 1024);
  const uint64_t dv = umma_desc(smem_u32(smem + LY::kSmemV), HD == 128 ? LY::kRegionV : 0, 1024);  // 64 dims: both halves of M alike
  const uint64_t dp = umma_desc(smem_u32(smem + LY::kSmemP), 0, 1024);
  int it = 0;
  uint32_t q_phase = 0;
  bool ok = true;
  while (w.left > 0 && ok) {
    const int tl = s.tl[w.b], n = __reduce_max_sync(0xffffffffu, min(w.left, tl - w.t));
    const int rows = min((s.N[w.b] - s.F[w.b]) * p.G - w.hr % s.nr[w.b] * kRows, kRows), N = __reduce_max_sync(0xffffffffu, (rows + 15) & -16);
    const uint32_t shape = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
    const uint32_t idesc_s = shape, idesc_o = shape | (1u << 15) | (1u << 16);  // both operands of the second product are MN-major
    auto scores = [&](int i) -> bool {
      if (!mbar_wait(&s.bar_ka[i & 1], (uint32_t)(i >> 1) & 1u)) return false;
      tc_fence_after();
#pragma unroll
      for (int ks = 0; ks < HD / 16; ++ks)
        umma_bf16_ts(tm + kTmemS + (i & 1) * 64, tm + kTmemK + (i & 1) * 64 + ks * 8,
                     dq + (uint64_t)((ks >> 2) * (LY::kRegionQ >> 4) + (ks & 3) * 2), idesc_s, ks > 0);
      umma_commit(&s.bar_s[i & 1]);
      return true;
    };
    ok = mbar_wait(&s.bar_q, q_phase) && scores(it);
    q_phase ^= 1;
    for (int i = 0; ok && i < n; ++i, ++it) {
      if (i + 1 < n) ok = scores(it + 1);
      ok = ok && mbar_wait(&s.bar_p[it & 1], (uint32_t)(it >> 1) & 1u) && mbar_wait(&s.bar_v[it & 1], (uint32_t)(it >> 1) & 1u);
      if (!ok) break;
      tc_fence_after();
      const uint64_t a = dv + (uint64_t)((it & 1) * (LY::kBufV >> 4)), bb = dp + (uint64_t)((it & 1) * (LY::kBufP >> 4));
#pragma unroll
      for (int ks = 0; ks < kTile / 16; ++ks)
        umma_bf16(tm + kTmemO, a + (uint64_t)(ks * (2048 >> 4)), bb + (uint64_t)(ks * (2048 >> 4)), idesc_o, (i > 0 || ks > 0) ? 1u : 0u);
      umma_commit(&s.bar_o[it & 1]);
    }
    for (int i = 0; i < n; ++i) advance(w, s, p);
  }
  if (!ok && (threadIdx.x & 31) == 0) report(p.st, CAST_ERR_TIMEOUT, w.b);
}

// ---- softmax of half of the columns (kMasked: `vm` says which of them see the position)
template <bool kMasked>
__device__ __forceinline__ void weights(float (&p)[32], const Misc& s, int c0, int nh, float ks, float kl, uint32_t vm) {
  const unsigned long long ks2 = pack_f2(ks, ks), kl2 = pack_f2(kl, kl);
#pragma unroll
  for (int c8 = 0; c8 < 4; ++c8) {
    if (c8 * 8 >= nh) break;
#pragma unroll
    for (int c = c8 * 8; c < c8 * 8 + 8; c += 4) {
      const float4 sq = *reinterpret_cast<const float4*>(&s.sq[c0 + c]), m = *reinterpret_cast<const float4*>(&s.m[c0 + c]);
      float x[4];
      unpack_f2(fma_f2(ks2, pack_f2(p[c], p[c + 1]), fma_f2(kl2, pack_f2(sq.x, sq.y), pack_f2(-m.x, -m.y))), x[0], x[1]);
      unpack_f2(fma_f2(ks2, pack_f2(p[c + 2], p[c + 3]), fma_f2(kl2, pack_f2(sq.z, sq.w), pack_f2(-m.z, -m.w))), x[2], x[3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y = fast_exp2(x[e]);
        p[c + e] = kMasked && !((vm >> (c + e)) & 1u) ? 0.f : y;
      }
    }
  }
}
template <bool kMasked>
__device__ __forceinline__ void hand_over(const float (&p)[32], unsigned long long (&l)[16], unsigned long long (&z)[16], unsigned char* row,
                                          int r7, int chunk0, int nh, float vs, float vl, uint32_t vm) {
  const unsigned long long vs2 = pack_f2(vs, vs), vl2 = pack_f2(vl, vl);
#pragma unroll
  for (int c8 = 0; c8 < 4; ++c8) {
    if (c8 * 8 >= nh) break;
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = c8 * 8 + 2 * e;
      const unsigned long long p2 = pack_f2(p[c], p[c + 1]);
      l[c / 2] = add_f2(l[c / 2], p2);
      float w0, w1;
      unpack_f2(mul_f2(p2, vs2), w0, w1);
      if (kMasked) {  // (a masked row of V without a value: 0 * NaN)
        const bool v0 = (vm >> c) & 1u, v1 = (vm >> (c + 1)) & 1u;
        z[c / 2] = fma_f2(p2, pack_f2(v0 ? vl : 0.f, v1 ? vl : 0.f), z[c / 2]);
        w0 = v0 ? w0 : 0.f;
        w1 = v1 ? w1 : 0.f;
      } else {
        z[c / 2] = fma_f2(p2, vl2, z[c / 2]);
      }
      const __nv_bfloat162 h = __floats2bfloat162_rn(w0, w1);
      w[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(row + (((chunk0 + c8) ^ r7) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// Merge of an item's partials by the 256 softmax threads of the CTA that finished it last: contributors in CTA order, a thread
// per 8 lanes of a row (which are 8 neighbouring dims).
template <int HD>
__device__ __forceinline__ void merge_item(const Q4Params& p, const Misc& s, int b, int h, int grow0, int rows, int c_lo, int c_hi,
                                           long long first) {
  constexpr int CPR = HD / 8, RPP = kSoftThreads / CPR;
  const int ch = threadIdx.x % CPR;
  for (int r = threadIdx.x / CPR; r < rows; r += RPP) {
    float M = -INFINITY;
    for (int c = c_lo; c <= c_hi; ++c) {
      const int slot = s.bound[c] > first ? 0 : 1;
      if (s.bound[c + 1] > s.bound[c]) M = fmaxf(M, __ldcg(p.part_ml + ((size_t)c * 2 + slot) * kRows + r).x);
    }
    float acc[8] = {}, l = 0.f;
#pragma unroll 2
    for (int c = c_lo; c <= c_hi; ++c) {
      if (s.bound[c + 1] <= s.bound[c]) continue;
      const size_t at = ((size_t)c * 2 + (s.bound[c] > first ? 0 : 1)) * kRows + r;
      const float2 ml = __ldcg(p.part_ml + at);
      const float4 x = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * HD + ch * 8));
      const float4 y = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * HD + ch * 8 + 4));
      const float w = ml.x == -INFINITY ? 0.f : exp2f(ml.x - M);
      l += w * ml.y;
      acc[0] += w * x.x; acc[1] += w * x.y; acc[2] += w * x.z; acc[3] += w * x.w;
      acc[4] += w * y.x; acc[5] += w * y.y; acc[6] += w * y.z; acc[7] += w * y.w;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    // lanes 8 ch + j: dims base + {0, 4, 1, 5, 2, 6, 3, 7}
    const int base = HD == 128 ? 32 * ((ch & 7) >> 1) + 8 * (2 * (ch >> 3) + (ch & 1)) : 8 * ch;
    const __nv_bfloat162 o0 = __floats2bfloat162_rn(acc[0] * inv, acc[2] * inv), o1 = __floats2bfloat162_rn(acc[4] * inv, acc[6] * inv),
                         o2 = __floats2bfloat162_rn(acc[1] * inv, acc[3] * inv), o3 = __floats2bfloat162_rn(acc[5] * inv, acc[7] * inv);
    const int grow = grow0 + r, t = grow / p.G;
    *reinterpret_cast<uint4*>(p.out + (((size_t)b * p.Ncap + t) * p.Hq + h * p.G + (grow - t * p.G)) * HD + base) =
        make_uint4(*reinterpret_cast<const uint32_t*>(&o0), *reinterpret_cast<const uint32_t*>(&o1),
                   *reinterpret_cast<const uint32_t*>(&o2), *reinterpret_cast<const uint32_t*>(&o3));
  }
}

template <int HD>
__device__ __forceinline__ void softmax(const Q4Params& p, Misc& s, unsigned char* smem, Walk w, uint32_t tmem) {
  using LY = Lay<HD>;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cg = warp >> 2, wg_bar = 1 + cg;
  const int posl = (warp & 3) * 32 + lane;                    // this thread's position in a tile, and its tensor-memory lane
  const uint32_t tl_sel = (uint32_t)((warp & 3) * 32) << 16;
  const float sc = p.scale_log2;
  // pairs of the row, one tile ahead; its page, two
  Walk wi = w, wr = w;
  int page = -1;
  uint32_t nkr = 0, nvr = 0;
  bool nlive = false;
  auto load_page = [&] {
    if (wi.left <= 0) return;
    page = page_of(p, wi.b, wi.t * kTile + posl, s.total[wi.b]);
    advance(wi, s, p);
  };
  auto load_pair = [&] {
    if (wr.left <= 0) return;
    nlive = page >= 0;
    if (nlive) {
      const long long row = row_of(p, page, wr.hr / s.nr[wr.b], wr.t * kTile + posl);
      nkr = __ldg(p.kr + row);
      nvr = __ldg(p.vr + row);
    }
    advance(wr, s, p);
  };
  load_page();
  load_pair();
  load_page();

  int it = 0;
  bool ok = true;
  while (w.left > 0) {
    const int b = w.b, nr = s.nr[b], h = w.hr / nr, rb = w.hr - h * nr, t0 = w.t, tl = s.tl[b], n = min(w.left, tl - t0);
    const int L = s.L[b], N = s.N[b], F = s.F[b], total = s.total[b];
    const int rows = min((N - F) * p.G - rb * kRows, kRows), nh = ((rows + 15) & -16) / 2, c0 = cg * nh, grow0 = F * p.G + rb * kRows;
    named_sync(3, kSoftThreads);  // the item before is done with the arrays below
    // ---- the query rows, their dims in the order of the codes in tensor memory; their sums
    {
      constexpr int VPR = HD / 8, W = LY::kW;
#pragma unroll 1
      for (int i = tid; i < 2 * nh * VPR; i += kSoftThreads) {
        const int r = i / VPR, v = i % VPR, t = v / W, wd = v % W;
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows) {
          const int grow = grow0 + r, tok = grow / p.G;
          x = __ldg(reinterpret_cast<const uint4*>(p.q + (((size_t)b * p.Ncap + tok) * p.Hq + h * p.G + (grow - tok * p.G)) * HD + v * 8));
        }
        float f[8], sum = 0.f;
        Vec<__nv_bfloat16>::unpack(x, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += f[e];
#pragma unroll
        for (int o = VPR / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (v == 0) {
          s.sq[r] = sum;
          s.m[r] = r < rows ? -INFINITY : 0.f;
        }
        // dims 0, 4, 1, 5 and 2, 6, 3, 7 of the eight
        const uint2 a = make_uint2(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632));
        const uint2 c = make_uint2(__byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632));
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int g = 2 * wd + half, chunk = 2 * (g & 3) + (t >> 1);
          *reinterpret_cast<uint2*>(smem + LY::kSmemQ + (g >> 2) * LY::kRegionQ + swz(r, chunk) + 8 * (t & 1)) = half ? c : a;
        }
      }
    }
    const bool tail = (t0 + n) * kTile > L;
    if (tail) {  // which columns see which tree token: 32 x 32 bits a warp, turned by votes
      const int ch = warp & 1, wd = warp >> 1, r = ch * 32 + lane;
      uint32_t bits = 0u;
      if (r < rows && wd < p.words) {
        bits = __ldg(p.anc + ((size_t)b * p.Ncap + (grow0 + r) / p.G) * p.words + wd);
        const int last = N - wd * 32;
        bits = last >= 32 ? bits : last > 0 ? bits & ((1u << last) - 1u) : 0u;
      }
      uint32_t mine = 0u;
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        const uint32_t v = __ballot_sync(0xffffffffu, (bits >> j) & 1u);
        if (lane == j) mine = v;
      }
      s.vis[ch][wd * 32 + lane] = mine;
    }
    fence_proxy_async();
    named_sync(3, kSoftThreads);
    if (tid == 0) mbar_arrive(&s.bar_q);

    unsigned long long l[16], z[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) l[c] = z[c] = 0ull;
    const uint32_t full = nh == 32 ? 0xffffffffu : (1u << nh) - 1u;
#pragma unroll 1
    for (int i = 0; i < n; ++i, ++it) {
      // this tile's pairs; the next one's are on their way meanwhile
      const bool live = nlive;
      const float st_k = q4_step(nkr), lo_k = q4_low(nkr), st_v = q4_step(nvr), lo_v = q4_low(nvr);
      const float ks = live ? sc * st_k : 0.f, kl = live ? sc * fmaf(-16.f, st_k, lo_k) : 0.f;
      const float vs = live ? st_v : 0.f, vl = live ? fmaf(8.f, st_v, lo_v) : 0.f;
      load_pair();
      load_page();
      const int pos = (t0 + i) * kTile + posl;
      uint32_t vm = live ? full : 0u;
      if (tail && live && pos >= L) {
        const int j = pos - L;
        const unsigned long long v = (unsigned long long)s.vis[0][j] | ((unsigned long long)s.vis[1][j] << 32);
        vm = (uint32_t)(v >> c0) & full;
      }
      const bool plain = __all_sync(0xffffffffu, vm == full);
      if (ok) {
        ok = mbar_wait(&s.bar_s[it & 1], (uint32_t)(it >> 1) & 1u);
        if (!ok && lane == 0) report(p.st, CAST_ERR_TIMEOUT, b);
      }
      const uint32_t ts = tmem + kTmemS + (it & 1) * 64 + c0 + tl_sel;
      float pr[32];
      auto read_scores = [&] {
        tc_fence_after();
#pragma unroll
        for (int c8 = 0; c8 < 4; ++c8) {
          if (c8 * 8 >= nh) break;
          tmem_ld8(ts + c8 * 8, reinterpret_cast<uint32_t*>(pr) + c8 * 8);
        }
        tmem_wait_ld_regs(reinterpret_cast<uint32_t(&)[32]>(pr));
      };
#pragma unroll
      for (int c = 0; c < 32; ++c) pr[c] = 0.f;
      if (ok) {
        read_scores();
        if (plain) weights<false>(pr, s, c0, nh, ks, kl, vm);
        else weights<true>(pr, s, c0, nh, ks, kl, vm);
      }
      float top = pr[0];
#pragma unroll
      for (int c = 1; c < 31; c += 2) top = fmaxf(top, fmaxf(pr[c], pr[c + 1]));
      top = fmaxf(top, pr[31]);
      if (named_or(wg_bar, 128, ok && top >= kFar)) {
        // a column without a reference yet, or a weight far above it: the tile's maxima decide (all four warps of the columns)
        float alpha_m[1];
        (void)alpha_m;
        if (ok) read_scores();
#pragma unroll
        for (int c = 0; c < 32; ++c) {
          if (c < nh) {
            float x = ok && ((vm >> c) & 1u) ? fmaf(ks, pr[c], kl * s.sq[c0 + c]) : -INFINITY;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
            if (lane == 0) s.colmax[warp][c] = x;
          }
        }
        if (ok && i > 0) {  // O^T has to be at rest
          ok = mbar_wait(&s.bar_o[(it - 1) & 1], (uint32_t)((it - 1) >> 1) & 1u);
          if (!ok && lane == 0) report(p.st, CAST_ERR_TIMEOUT, b);
        }
        named_sync(wg_bar, 128);
        auto moved = [&](int c, float& m_new) {  // the factor for what column c has gathered
          const float m_old = s.m[c0 + c];
          const float mx = fmaxf(fmaxf(s.colmax[cg * 4][c], s.colmax[cg * 4 + 1][c]), fmaxf(s.colmax[cg * 4 + 2][c], s.colmax[cg * 4 + 3][c]));
          m_new = m_old == -INFINITY || mx >= m_old + 59.f ? mx : m_old;
          return m_old == -INFINITY || m_new == m_old ? 1.f : exp2f(m_old - m_new);
        };
        if (ok) tc_fence_after();
#pragma unroll
        for (int c8 = 0; c8 < 4; ++c8) {
          if (c8 * 8 >= nh) break;
          uint32_t o[8];
          const bool scale_o = ok && i > 0;
          if (scale_o) {
            tmem_ld8(tmem + kTmemO + c0 + c8 * 8 + tl_sel, o);
            tmem_wait_ld();
          }
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const int c = c8 * 8 + e;
            float m0, m1;
            const float a0 = moved(c, m0), a1 = moved(c + 1, m1);
            const unsigned long long a2 = pack_f2(a0, a1);
            l[c / 2] = mul_f2(l[c / 2], a2);
            z[c / 2] = mul_f2(z[c / 2], a2);
            if (scale_o) {
              o[e] = __float_as_uint(__uint_as_float(o[e]) * a0);
              o[e + 1] = __float_as_uint(__uint_as_float(o[e + 1]) * a1);
            }
          }
          if (scale_o) tmem_st8(tmem + kTmemO + c0 + c8 * 8 + tl_sel, o);
        }
        if (ok) tmem_wait_st();
        float m_mine = 0.f;
        const int c_mine = tid & 127;
        if (c_mine < nh) moved(c_mine, m_mine);
        named_sync(wg_bar, 128);
        if (c_mine < nh) s.m[c0 + c_mine] = m_mine;
        named_sync(wg_bar, 128);
        if (ok) {
          read_scores();
          weights<true>(pr, s, c0, nh, ks, kl, vm);
        }
      }
      if (ok && it >= 2) {  // the weights of tile it - 2 have been read
        ok = mbar_wait(&s.bar_o[it & 1], (uint32_t)((it >> 1) - 1) & 1u);
        if (!ok && lane == 0) report(p.st, CAST_ERR_TIMEOUT, b);
      }
      if (ok) {
        unsigned char* row = smem + LY::kSmemP + (it & 1) * LY::kBufP + posl * 128;
        if (plain) hand_over<false>(pr, l, z, row, posl & 7, c0 >> 3, nh, vs, vl, vm);
        else hand_over<true>(pr, l, z, row, posl & 7, c0 >> 3, nh, vs, vl, vm);
        fence_proxy_async();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.bar_p[it & 1]);
    }

    // ---- the item's end: sums over the lanes, then over the warps of a column
    if (ok) {
      ok = mbar_wait(&s.bar_o[(it - 1) & 1], (uint32_t)((it - 1) >> 1) & 1u);
      if (!ok && lane == 0) report(p.st, CAST_ERR_TIMEOUT, b);
    }
    {
      float v[32];
#pragma unroll
      for (int c = 0; c < 16; ++c) unpack_f2(l[c], v[2 * c], v[2 * c + 1]);
      const float suml = reduce_columns(v);
#pragma unroll
      for (int c = 0; c < 16; ++c) unpack_f2(z[c], v[2 * c], v[2 * c + 1]);
      const float sumz = reduce_columns(v);
      if (lane < nh) {
        s.red_l[warp & 3][c0 + lane] = suml;
        s.red_z[warp & 3][c0 + lane] = sumz;
      }
    }
    named_sync(wg_bar, 128);
    if ((tid & 127) < nh) {
      const int c = c0 + (tid & 127);
      s.tot_l[c] = s.red_l[0][c] + s.red_l[1][c] + s.red_l[2][c] + s.red_l[3][c];
      s.tot_z[c] = s.red_z[0][c] + s.red_z[1][c] + s.red_z[2][c] + s.red_z[3][c];
    }
    named_sync(wg_bar, 128);
    const bool whole = n == tl;
    // lane m of O^T: dims in the order of merge_item
    const int ch = posl >> 3, j8 = posl & 7;
    const int dim = (HD == 128 ? 32 * ((ch & 7) >> 1) + 8 * (2 * (ch >> 3) + (ch & 1)) : 8 * ch) + ((j8 >> 1) | ((j8 & 1) << 2));
    const int slot = (int)blockIdx.x * 2 + (s.bound[blockIdx.x] > s.pre[b] + (long long)w.hr * tl ? 0 : 1);
    if (ok) {
      tc_fence_after();
#pragma unroll 1
      for (int c8 = 0; c8 * 8 < nh; ++c8) {
        uint32_t o[8];
        tmem_ld8(tmem + kTmemO + c0 + c8 * 8 + tl_sel, o);
        tmem_wait_ld();
        if (HD == 64 && posl >= 64) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = c0 + c8 * 8 + e;
          const float x = __uint_as_float(o[e]) + s.tot_z[c];
          if (c >= rows) continue;
          if (whole) {
            const float lt = s.tot_l[c];
            const int grow = grow0 + c, t = grow / p.G;
            p.out[(((size_t)b * p.Ncap + t) * p.Hq + h * p.G + (grow - t * p.G)) * HD + dim] =
                __float2bfloat16_rn(x * (lt == 0.f ? 0.f : 1.f / lt));
          } else {
            __stcg(p.part_o + ((size_t)slot * kRows + c) * HD + posl, x);
          }
        }
      }
    }
    tc_fence_before();
    if (!whole) {
      if ((tid & 127) < nh) {
        const int c = c0 + (tid & 127);
        __stcg(p.part_ml + (size_t)slot * kRows + c, ok ? make_float2(s.m[c], s.tot_l[c]) : make_float2(-INFINITY, 0.f));
      }
      // the CTAs that share the item
      const long long first = s.pre[b] + (long long)w.hr * tl, end = first + tl;
      int c_lo = blockIdx.x, c_hi = blockIdx.x;
      while (s.bound[c_lo] > first) --c_lo;
      while (s.bound[c_hi + 1] < end) ++c_hi;
      named_sync(3, kSoftThreads);
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
      named_sync(3, kSoftThreads);
      if (s.last) merge_item<HD>(p, s, b, h, grow0, rows, c_lo, c_hi, first);
    }
    for (int i = 0; i < n; ++i) advance(w, s, p);
  }
}

template <int HD>
__global__ void __launch_bounds__(kThreadsQ4, 1) tree_attn_q4_kernel(const Q4Params p) {
  extern __shared__ __align__(1024) unsigned char smem[];
  using LY = Lay<HD>;
  Misc& s = *reinterpret_cast<Misc*>(smem + LY::kSmemMisc);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // Everything, tensor memory included, behind the wait; the warp that allocates releases the dependents after it has.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (warp == kWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem)), "n"(kTmemCols));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (lane == 0) {
      for (int i = 0; i < 2; ++i) {
        mbar_init(&s.bar_ka[i], 4);
        mbar_init(&s.bar_s[i], 1);
        mbar_init(&s.bar_v[i], 4);
        mbar_init(&s.bar_p[i], 8);
        mbar_init(&s.bar_o[i], 1);
      }
      mbar_init(&s.bar_q, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      fence_proxy_async();
    }
    __syncwarp();
  } else if (warp == 0) {
    // the line of tiles
    constexpr int KB = CAST_MAX_BATCH / 32;
    const long long max_pos = p.g.max_pos();
    long long run = 0;
    int items = 0;
    int Nv[KB], Lv[KB], Fv[KB];
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
      long long mine = (long long)p.Hkv * nr * tl, upto = mine;
      int cnt = p.Hkv * nr;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
      }
      items += __reduce_add_sync(0xffffffffu, cnt);
      s.pre[b] = run + upto - mine;
      run += __shfl_sync(0xffffffffu, upto, 31);
      s.L[b] = L; s.N[b] = N; s.F[b] = F; s.tl[b] = tl; s.nr[b] = nr; s.total[b] = total;
    }
    if (lane == 0) {
      s.pre[CAST_MAX_BATCH] = run;
      // pieces of two tiles at least, and no item over more CTAs than a merge is worth
      long long workers = (run + 1) / 2;
      workers = workers < (long long)items * kMaxJoin ? workers : (long long)items * kMaxJoin;
      s.workers = (int)(workers < (long long)gridDim.x ? workers : (long long)gridDim.x);
    }
  }
  __syncthreads();
  // where the pieces begin
  if (tid <= (int)gridDim.x) {
    const long long T = s.pre[CAST_MAX_BATCH];
    long long x = tid >= s.workers ? T : T * tid / s.workers;
    s.bound[tid] = x;
    if (tid == (int)blockIdx.x && x < T) {
      int b = 0;
      while (s.pre[b + 1] <= x) ++b;
      const long long in = x - s.pre[b];
      s.b0 = b;
      s.hr0 = (int)(in / s.tl[b]);
      s.t0 = (int)(in - (long long)s.hr0 * s.tl[b]);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s.tmem;
  Walk w;
  w.left = (int)(s.bound[blockIdx.x + 1] - s.bound[blockIdx.x]);
  w.b = s.b0; w.hr = s.hr0; w.t = s.t0;
  const bool aligned = (smem_u32(smem) & 1023u) == 0u;  // the swizzled operand regions need a 1 KB aligned base
  if (!aligned && tid == 0) report(p.st, CAST_ERR_CUDA, 1024);
  if (w.left > 0 && aligned) {
    if (warp < kWarpK) {
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoft));
      softmax<HD>(p, s, smem, w, tmem);
    } else if (warp < kWarpMma) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsProduce));
      if (warp < kWarpV) produce<HD, false>(p, s, smem, w, tmem);
      else produce<HD, true>(p, s, smem, w, tmem);
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
      if (warp == kWarpMma) issue<HD>(p, s, smem, w, tmem);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kWarpMma)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemCols));
}

constexpr size_t kPartBytes = (size_t)2 * kRows * (128 * sizeof(float) + sizeof(float2));  // per CTA

int q4_grid(const cast_ctx* c) { return c->num_sms < kMaxGrid ? c->num_sms : kMaxGrid; }
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
  Q4Params p;
  p.nrb = q4_row_blocks(c, Hq, Hkv);
  // compute calls never allocate: the workspace comes from cast_reserve_attention_q4
  if (grid * kPartBytes + (size_t)B * Hkv * p.nrb * sizeof(int32_t) > c->q4_ws_bytes) return CAST_ERR_CAPACITY;
  p.q = (const __nv_bfloat16*)q; p.out = (__nv_bfloat16*)out;
  p.kc = (const unsigned char*)k_codes; p.vc = (const unsigned char*)v_codes;
  p.kr = (const uint32_t*)k_range; p.vr = (const uint32_t*)v_range;
  p.B = B; p.Ncap = c->cfg.max_tree; p.Nmax = c->cfg.total_token; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv; p.words = c->words;
  p.g = g;
  // exact for positions below 2^31: the multiplier is at most page_size - 1 too large in 2^page_shift, page_shift = 31 + log2 (rounded up)
  int lg = 0;
  while (g.page_size > 0 && (1ll << lg) < g.page_size) ++lg;
  p.page_shift = 31 + lg;
  p.page_mul = g.page_size > 0 ? (uint32_t)(((1ull << p.page_shift) + g.page_size - 1) / g.page_size) : 0u;
  p.kv_len = kv_len; p.n_tree = n_tree; p.first_row = first_row; p.anc = anc;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.part_o = (float*)c->q4_ws;
  p.part_ml = (float2*)(p.part_o + (size_t)grid * 2 * kRows * 128);
  p.ticket = (int32_t*)((char*)c->q4_ws + grid * kPartBytes);
  p.st = c->state;
  auto* const kern = D == 64 ? tree_attn_q4_kernel<64> : tree_attn_q4_kernel<128>;
  const int smem = (D == 64 ? Lay<64>::kSmemMisc : Lay<128>::kSmemMisc) + (int)sizeof(Misc);
  CAST_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
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
