// cast_attention_mass, cast_attention_mass_q4: the attention weight that the accepted rows gave every cached position.
//
//   mass[p] += sum_r e^(s_r(p) - m_r) / l_r,   s_r(p) = scale q_r . k_p,   l_r = sum_p e^(s_r(p) - m_r)
//
// over the rows r = (accepted token, head of the group) of a kv-head. The weights need every row's sum first, so the keys are
// read twice: pass 1 forms each row's (reference, sum) over a piece of the sequence, pass 2 merges the pieces' pairs, forms the
// scores again and adds the weights of a position over the rows in their order. A position's sum belongs to one thread: no
// atomics, the same bits every time.
//
// bf16 queries: mass_tc_kernel. As in the attention over 4-bit caches positions are the rows of the product and queries its columns,
// S^T = K Q^T (128 positions x up to 32 queries): a thread owns a position, the sum over the rows is its own, and in pass 2 nothing
// crosses lanes. 4-bit keys go through registers to tensor memory as exact small integers (c - 8), 16-bit ones by asynchronous copies to
// shared memory. Four warps a CTA, three or four CTAs per SM to run under each other's waits. fp32 queries: mass_kernel on the CUDA cores.
//
// Measured: 8 layers of 8 sequences of 1024 to 4096, 28 rows of bf16 per kv-head at most, 32 / 8 heads of 128: 140 us (54 to read the
// keys once; the two passes read 350 MB each at 58 % of the memory's rate). 2 layers of 4 sequences of 32768 in 4 bits, 28 / 4 heads, up to 49
// rows: 107 to 155 us by the rows accepted (12 to read the keys once): bound by the instructions of the codes and the exponentials, issue slots half busy. Slower:
// three CTAs per SM for the 4-bit pass 1, which then spills nothing (151 us); the next product sent off ahead of this one's scores, with two
// tiles' scores in tensor memory (153, and 155 for 148 with bf16 keys: the other CTAs hide a product's time already); columns by 24 (159).
// fp32, 4 layers of 4 sequences of 1000 to 2111: 32 / 8 heads of 128 226 us, 4-bit keys 196 (a warp without rows leaves the products to the
// others: 291 and 253 before); 8 / 8 heads of 64, 300 to 2111: 81 and 72.
#include <math.h>

#include "q4_tc.h"

using namespace cast;

namespace {

constexpr int kRB = 32;   // query rows per block
constexpr int kPT = 64;   // positions per tile
constexpr int kThreads = 256;
constexpr int kMaxSplit = 64;

struct MassParams {
  const void* q;
  const unsigned char* k;    // bf16 or fp32 rows (as the queries are), or codes
  const uint32_t* range;     // 4-bit caches: the pairs
  size_t q_stride, k_stride, range_stride;  // bytes per layer
  int B, Ncap, Hq, Hkv, G, max_rows, nsplit, path_stride;
  Paging g;
  FastPaging fg;
  const int32_t* path;
  const int32_t* accept_len;
  const int32_t* kv_len;
  float scale, scale_log2;
  float* mass;
  float2* part;  // [n_layers][B][Hkv][max_rows * G][nsplit] (reference, sum)
  DevState* st;
};

// What a CTA finds about its sequence: n accepted rows, len positions; n = 0 where there is nothing to add.
struct Seq {
  int n, len;
};
__device__ __forceinline__ Seq find_seq(const MassParams& p, int b, bool say) {
  const int a = p.accept_len[b];
  if (a < 0) return {0, 0};
  const Seq s = {a + 1, p.kv_len[b]};
  int bad = a >= p.max_rows || s.len < s.n ? CAST_ERR_BAD_TREE : s.len > p.g.max_pos() ? CAST_ERR_BAD_PAGE : 0;
  if (!bad && p.path != nullptr)
    for (int i = 0; i < s.n; ++i) {
      const int t = p.path[(size_t)b * p.path_stride + i];
      if (t < 0 || t >= p.Ncap) bad = CAST_ERR_BAD_TREE;
    }
  if (bad) {
    if (say) report(p.st, bad, b);
    return {0, 0};
  }
  return s;
}

// Sixteen dims of a key row of a fp32 or 4-bit cache.
template <int D, bool kQ4>
__device__ __forceinline__ void load_key_piece(const MassParams& p, int layer, long long row, int ch, float (&f)[16]) {
  if constexpr (kQ4) {
    const uint32_t r = *(reinterpret_cast<const uint32_t*>(reinterpret_cast<const unsigned char*>(p.range) + p.range_stride * layer) + row);
    const uint2 w = *reinterpret_cast<const uint2*>(p.k + p.k_stride * layer + row * (D / 2) + ch * 8);
    const float step = q4_step(r), low = q4_low(r);
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] = fmaf(step, (float)(((e < 8 ? w.x : w.y) >> (4 * (e % 8))) & 15u), low);
  } else {
    const float4* src = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.k + p.k_stride * layer) + row * D + ch * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 x = src[i];
      f[4 * i] = x.x; f[4 * i + 1] = x.y; f[4 * i + 2] = x.z; f[4 * i + 3] = x.w;
    }
  }
}

template <int D, bool kQ4, int kPass>
__global__ void __launch_bounds__(kThreads) mass_kernel(const MassParams p) {
  constexpr int KS = D + 4, SS = kPT + 4;
  extern __shared__ __align__(16) float smem[];
  float* Qs = smem;            // [kRB][KS], scaled
  float* Ks = Qs + kRB * KS;   // [kPT][KS]
  float* Ss = Ks + kPT * KS;   // [kRB][SS]
  __shared__ float row_m[kRB], row_l[kRB];
  __shared__ long long slot_s[kPT];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int split = blockIdx.x % p.nsplit, kvh = blockIdx.x / p.nsplit, b = blockIdx.y, layer = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const Seq sq = find_seq(p, b, kPass == 1 && tid == 0 && blockIdx.x == 0 && layer == 0);
  if (sq.n == 0) return;
  const int rows = sq.n * p.G, ntiles = (sq.len + kPT - 1) / kPT;
  const int t0 = (int)((long long)split * ntiles / p.nsplit), t1 = (int)((long long)(split + 1) * ntiles / p.nsplit);
  const size_t seg = ((size_t)layer * p.B + b) * p.Hkv + kvh;
  float2* const part = p.part + seg * (size_t)(p.max_rows * p.G) * p.nsplit;
  const int ty = tid / 16, tx = tid % 16;
  for (int r0 = 0; r0 < rows; r0 += kRB) {
    __syncthreads();
    const float* q = reinterpret_cast<const float*>(reinterpret_cast<const unsigned char*>(p.q) + p.q_stride * layer);
    for (int i = tid; i < kRB * D; i += kThreads) {
      const int r = i / D, d = i % D, row = r0 + r;
      float x = 0.f;
      if (row < rows) {
        const int j = row / p.G, t = p.path ? p.path[(size_t)b * p.path_stride + j] : j;
        x = q[(((size_t)b * p.Ncap + t) * p.Hq + kvh * p.G + row % p.G) * D + d] * p.scale;
      }
      Qs[r * KS + d] = x;
    }
    if (tid < kRB) {
      float m = -INFINITY, l = 0.f;
      if (kPass == 2 && r0 + tid < rows) {
        for (int s = 0; s < p.nsplit; ++s) m = fmaxf(m, part[(size_t)(r0 + tid) * p.nsplit + s].x);
        for (int s = 0; s < p.nsplit; ++s) {
          const float2 x = part[(size_t)(r0 + tid) * p.nsplit + s];
          if (x.y != 0.f) l += x.y * expf(x.x - m);
        }
      }
      row_m[tid] = m;
      row_l[tid] = kPass == 2 ? (l != 0.f ? 1.f / l : 0.f) : l;
    }
    for (int tile = t0; tile < t1; ++tile) {
      __syncthreads();  // the tile before is consumed
      if (tid < kPT) {
        const int pos = tile * kPT + tid;
        long long slot = -1;
        int page, in_page;
        if (pos < sq.len) {
          if (!find_place(p.g, b, pos, page, in_page)) report(p.st, CAST_ERR_BAD_PAGE, b);
          else if (kQ4) slot = q4_row(p.g, p.Hkv, kvh, page, in_page);
          else slot = ((long long)page * (p.g.page_size == 0 ? p.g.seq_capacity : p.g.page_size) + in_page) * p.Hkv + kvh;
        }
        slot_s[tid] = slot;
      }
      __syncthreads();
      for (int i = tid; i < kPT * (D / 16); i += kThreads) {
        const int pl = i / (D / 16), ch = i % (D / 16);
        float f[16] = {};
        if (slot_s[pl] >= 0) load_key_piece<D, kQ4>(p, layer, slot_s[pl], ch, f);
#pragma unroll
        for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4*>(Ks + pl * KS + ch * 16 + e) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
      }
      __syncthreads();
      const bool any_row = r0 + 4 * warp < rows;  // a warp's four rows, here and below
      float acc[2][4] = {};
#pragma unroll 4
      for (int d = 0; d < D && any_row; d += 4) {  // (by 16 bytes: the rows lie 16 apart modulo 128, eight threads of them meet no bank twice)
        float4 a[2], k[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) a[i] = *reinterpret_cast<const float4*>(Qs + (2 * ty + i) * KS + d);
#pragma unroll
        for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const float4*>(Ks + (tx + 16 * j) * KS + d);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[i][j] = fmaf(a[i].w, k[j].w, fmaf(a[i].z, k[j].z, fmaf(a[i].y, k[j].y, fmaf(a[i].x, k[j].x, acc[i][j]))));
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = 2 * ty + i, row = r0 + r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int pl = tx + 16 * j, pos = tile * kPT + pl;
          const bool vis = row < rows && slot_s[pl] >= 0 && pos < sq.len - sq.n + row / p.G + 1;
          Ss[r * SS + pl] = vis ? acc[i][j] : -INFINITY;
        }
      }
      __syncthreads();
      if (kPass == 1) {
#pragma unroll
        for (int rr = 0; rr < 4 && any_row; ++rr) {
          const int r = 4 * warp + rr;
          const float s0 = Ss[r * SS + lane], s1 = Ss[r * SS + lane + 32];
          float mx = fmaxf(s0, s1);
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
          const float m_old = row_m[r], m_new = fmaxf(m_old, mx);
          // (a score that is NaN is no maximum, but its exponential reaches the sum)
          const float base = m_new > -INFINITY ? m_new : 0.f;
          float sum = expf(s0 - base) + expf(s1 - base);
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          __syncwarp();
          if (lane == 0) {
            row_l[r] = (m_old > -INFINITY ? row_l[r] * expf(m_old - base) : row_l[r]) + sum;
            row_m[r] = m_new;
          }
          __syncwarp();
        }
      } else if (tid < kPT) {
        const int pos = tile * kPT + tid;
        if (slot_s[tid] >= 0) {
          float sum = 0.f;
          for (int r = 0; r < kRB && r0 + r < rows; ++r) {
            const float s = Ss[r * SS + tid];
            if (s != -INFINITY) sum += expf(s - row_m[r]) * row_l[r];
          }
          p.mass[seg * (size_t)p.g.max_pos() + pos] += sum;
        }
      }
    }
    if (kPass == 1) {
      __syncthreads();
      if (tid < kRB && r0 + tid < rows) part[(size_t)(r0 + tid) * p.nsplit + split] = make_float2(row_m[tid], row_l[tid]);
    }
  }
}

// ------------------------------------------------------------------------------------------ bf16 queries: tensor cores
constexpr int kTile = 128;      // positions per tile (UMMA M)
constexpr int kCols = 32;       // query columns per block (UMMA N)
constexpr int kThreadsTc = 128;
constexpr int kMinTiles = 2;    // of a piece (one sequence of 8192, 2 layers: 34 us, pieces of one 44, of three 37)
constexpr float kFar = 1.15292150460684698e18f;  // 2^60

template <int N>
struct Cols {
  static constexpr int value = N;
};

template <int HD, bool kQ4>
struct MassLay {
  static constexpr int kRegionQ = kCols * 128;                  // [32 rows][64] bf16
  static constexpr int kSmemK = 8 * 1024;                       // 16-bit keys: two stages of HD / 64 regions [128 positions][64]
  static constexpr int kRegionK = kTile * 128;
  static constexpr int kStageK = HD / 64 * kRegionK;
  static constexpr int kSmemMisc = kSmemK + (kQ4 ? 0 : 2 * kStageK);
  static constexpr int kTmemS = kQ4 ? 64 : 0, kTmemCols = kQ4 ? 128 : 32;
};
struct MassMisc {
  uint64_t bar_s;
  uint32_t tmem;
  alignas(16) float sq[kCols];     // sums of the query rows (4-bit keys)
  alignas(16) float nm[kCols];     // references, log2 units, negated; inf: none yet. Pass 2: the rows' log-sums
  alignas(16) float alpha[kCols];
  float colmax[4][kCols];
};

template <int HD, bool kPaged, bool kQ4, int kPass>
__global__ void __launch_bounds__(kThreadsTc, kQ4 ? 4 : 3) mass_tc_kernel(const MassParams p) {
  extern __shared__ __align__(1024) unsigned char smem_tc[];
  using LY = MassLay<HD, kQ4>;
  constexpr int W = HD / 32, VPR = HD / 8;  // words of codes per thread and row; 16-byte pieces of a 16-bit row
  MassMisc& s = *reinterpret_cast<MassMisc*>(smem_tc + LY::kSmemMisc);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem)), "n"(LY::kTmemCols));
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (lane == 0) {
      mbar_init(&s.bar_s, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      fence_proxy_async();
    }
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __reduce_or_sync(0xffffffffu, s.tmem);
  const int split = blockIdx.x % p.nsplit, kvh = blockIdx.x / p.nsplit, b = blockIdx.y, layer = blockIdx.z;
  const Seq sq = find_seq(p, b, kPass == 1 && tid == 0 && blockIdx.x == 0 && layer == 0);
  // pieces of kMinTiles tiles at least, whatever the capacity that the launch was sized for
  const int ntiles = (sq.len + kTile - 1) / kTile, G = p.G, pieces = min(p.nsplit, (ntiles + kMinTiles - 1) / kMinTiles);
  const int rows_all = split < pieces ? sq.n * G : 0;
  const int t0 = (int)((long long)split * ntiles / max(pieces, 1)), n = (int)((long long)(split + 1) * ntiles / max(pieces, 1)) - t0;
  const size_t seg = ((size_t)layer * p.B + b) * p.Hkv + kvh;
  float2* const part = p.part + seg * (size_t)(p.max_rows * G) * p.nsplit;
  const bool aligned = (smem_u32(smem_tc) & 1023u) == 0u;  // the swizzled operand regions need a 1 KB aligned base
  if (!aligned && tid == 0) report(p.st, CAST_ERR_CUDA, 1024);
  const unsigned char* const keys = p.k + p.k_stride * layer;
  const int32_t* const range = reinterpret_cast<const int32_t*>(reinterpret_cast<const unsigned char*>(p.range) + p.range_stride * layer);
  const __nv_bfloat16* const q = reinterpret_cast<const __nv_bfloat16*>(reinterpret_cast<const unsigned char*>(p.q) + p.q_stride * layer);
  const int r = lane >> 2, tq = lane & 3;
  const uint32_t t_part = (uint32_t)(warp * 32) << 16;
  float* const mass = p.mass + seg * (size_t)p.g.max_pos();
  uint32_t it = 0;  // tiles so far: the barrier's phase
  bool ok = aligned;

  auto block = [&](auto nh_c, int r0) {
    constexpr int NH = decltype(nh_c)::value;
    constexpr uint32_t shape = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(NH >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
    const int rows = min(rows_all - r0, NH);
    const uint32_t full = rows >= 32 ? 0xffffffffu : (1u << rows) - 1u;
    // ---- the query rows; 4-bit keys: their dims in the order of the codes in tensor memory, and their sums
#pragma unroll 1
    for (int i = tid; i < NH * VPR; i += kThreadsTc) {
      const int qr = i / VPR, v = i % VPR;
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (qr < rows) {
        const int j = (r0 + qr) / G, t = p.path ? p.path[(size_t)b * p.path_stride + j] : j;
        x = *reinterpret_cast<const uint4*>(q + (((size_t)b * p.Ncap + t) * p.Hq + kvh * G + (r0 + qr - j * G)) * HD + v * 8);
      }
      if constexpr (kQ4) {
        float f[8], sum = 0.f;
        Vec<__nv_bfloat16>::unpack(x, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += f[e];
#pragma unroll
        for (int o = VPR / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (v == 0) s.sq[qr] = sum;
        // dims 0, 4, 1, 5 and 2, 6, 3, 7 of the eight
        const uint2 lo = make_uint2(__byte_perm(x.x, x.z, 0x5410), __byte_perm(x.x, x.z, 0x7632));
        const uint2 hi = make_uint2(__byte_perm(x.y, x.w, 0x5410), __byte_perm(x.y, x.w, 0x7632));
        const int t = v / W, wd = v % W;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const int g = 2 * wd + half, ch = 2 * (g & 3) + (t >> 1);
          *reinterpret_cast<uint2*>(smem_tc + (g >> 2) * LY::kRegionQ + swz(qr, ch) + 8 * (t & 1)) = half ? hi : lo;
        }
      } else {
        *reinterpret_cast<uint4*>(smem_tc + (v >> 3) * LY::kRegionQ + swz(qr, v & 7)) = x;
      }
    }
    if (!kQ4 && tid < NH) s.sq[tid] = 0.f;
    if (kPass == 1) {
      if (tid < NH) s.nm[tid] = tid < rows ? INFINITY : 0.f;
    } else if (tid < 4 * NH) {  // the row's sum from the pieces' pairs: four threads to a row
      const int row = tid >> 2, sub = tid & 3;
      const float2* pairs = part + (size_t)(r0 + min(row, rows - 1)) * p.nsplit;
      float m = -INFINITY, l = 0.f;
#pragma unroll 8
      for (int i = sub; i < pieces; i += 4) m = fmaxf(m, pairs[i].x);
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
      m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
#pragma unroll 4
      for (int i = sub; i < pieces; i += 4) {
        const float2 x = pairs[i];
        l += x.x == -INFINITY && x.y == 0.f ? 0.f : x.y * exp2f(x.x - m);
      }
      l += __shfl_xor_sync(0xffffffffu, l, 1);
      l += __shfl_xor_sync(0xffffffffu, l, 2);
      if (sub == 0) s.nm[row] = row < rows ? -(m + log2f(l)) : -INFINITY;  // (a column without a row weighs nothing)
    }
    // ---- keys, a tile ahead: every lane finds the place of its own position's row
    uint32_t kc[4][W], row = 0;
    int page = 0, nkr = 0;
    bool live_next = false;
    auto next_page = [&](int i) { page = request_page<kPaged>(p.fg, b, (t0 + min(i, n - 1)) * kTile + tid, sq.len); };
    auto next_row = [&](int i) {
      const int pos = (t0 + min(i, n - 1)) * kTile + tid;
      row = kQ4 ? row_of<kPaged>(p.fg, page, kvh, pos, sq.len) : dense_row_of<kPaged>(p.fg, page, kvh, pos, sq.len);
      live_next = page_ok<kPaged>(p.fg, page) && pos < sq.len;
      if (kPaged && kPass == 1 && !page_ok<kPaged>(p.fg, page) && pos < sq.len) report(p.st, CAST_ERR_BAD_PAGE, b);
    };
    auto request = [&](int i) {
      if constexpr (kQ4) {
        nkr = ld_here(range + row);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          ld_here(kc[j], keys + (size_t)__shfl_sync(0xffffffffu, row, 8 * j + r) * (HD / 2) + tq * (4 * W));
      } else {
        unsigned char* stage = smem_tc + LY::kSmemK + (i & 1) * LY::kStageK;
        constexpr int RPI = 32 / VPR;  // rows per instruction
#pragma unroll
        for (int j = 0; j < 32 / RPI; ++j) {
          const int rr = j * RPI + lane / VPR, v = lane % VPR;
          const unsigned char* src = keys + (size_t)__shfl_sync(0xffffffffu, row, rr) * (HD * 2) + v * 16;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(stage + (v >> 3) * LY::kRegionK + swz(warp * 32 + rr, v & 7))),
                       "l"(src)
                       : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
    };
    if (n > 0) {
      next_page(0);
      next_row(0);
      next_page(1);
      request(0);
    }
    float l[NH];
#pragma unroll
    for (int c = 0; c < NH; ++c) l[c] = 0.f;
#pragma unroll 1
    for (int i = 0; i < n; ++i, ++it) {
      const bool live = live_next;
      float ks = p.scale_log2, kl = 0.f;
      if constexpr (kQ4) {
        const float st = q4_step((uint32_t)nkr);
        ks = live ? p.scale_log2 * st : 0.f;
        kl = live ? p.scale_log2 * fmaf(8.f, st, q4_low((uint32_t)nkr)) : 0.f;
        if (ok) {
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
            for (int w = 0; w < W; ++w) {  // word w's pairs 0, 1 go to the group of 16 dims 2 w, pairs 2, 3 to 2 w + 1
              const uint32_t a = kc[2 * hf][w], c = kc[2 * hf + 1][w];
              const uint32_t out[8] = {pair_minus8<0>(a), pair_minus8<1>(a), pair_minus8<0>(c), pair_minus8<1>(c),
                                       pair_minus8<2>(a), pair_minus8<3>(a), pair_minus8<2>(c), pair_minus8<3>(c)};
              tmem_st_quads<2>(tmem + 16 * w + t_part + ((uint32_t)(hf * 16) << 16), out);
            }
          }
        }
      }
      if constexpr (kQ4) {
        if (ok) tmem_wait_st();
      } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      fence_proxy_async();
      tc_fence_before();
      __syncthreads();
      if (warp == __reduce_max_sync(0xffffffffu, (int)(it & 3u)) && ok) {
        tc_fence_after();
        const uint64_t dq = umma_desc(smem_u32(smem_tc), 16, 1024);
        const uint64_t dk = umma_desc(smem_u32(smem_tc + LY::kSmemK + (i & 1) * LY::kStageK), 16, 1024);
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          const uint64_t bq = dq + (uint64_t)((k >> 2) * (LY::kRegionQ >> 4) + (k & 3) * 2);
          if constexpr (kQ4) umma_bf16_ts(tmem + LY::kTmemS, tmem + k * 8, bq, shape, k > 0);
          else umma_bf16(tmem + LY::kTmemS, dk + (uint64_t)((k >> 2) * (LY::kRegionK >> 4) + (k & 3) * 2), bq, shape, k > 0);
        }
        umma_commit(&s.bar_s);
      }
      // The tile behind: requested here because the fence waits for whatever is out. (Its 16-bit stage was last read by the product of
      // tile i - 1, which is over.)
      next_row(i + 1);
      next_page(i + 2);
      request(i + 1);
      // row i of n sees the positions below len - n + i + 1
      const int pos = (t0 + i) * kTile + tid, j = pos - (sq.len - sq.n);
      uint32_t vm = live ? full : 0u;
      if (j > 0) {
        const int c = j * G - r0;
        vm = c >= 32 ? 0u : c > 0 ? vm & (0xffffffffu << c) : vm;
      }
      const bool plain = __all_sync(0xffffffffu, vm == full);
      if (ok) {
        ok = mbar_wait(&s.bar_s, it & 1u);
        if (!ok && lane == 0) report(p.st, CAST_ERR_TIMEOUT, b);
      }
      tc_fence_after();
      float pr[NH];
      auto to_weights = [&] {
        weights<NH>(pr, s.sq, s.nm, ks, kl);
        if (!plain) mask_weights<NH>(pr, vm);
      };
      if (ok) read_scores<NH>(tmem + LY::kTmemS + t_part, pr);
      else {
#pragma unroll
        for (int c = 0; c < NH; ++c) pr[c] = 0.f;
      }
      if (kPass == 1) {
        bool far = false;
        if (i > 0) {
          to_weights();
          float top = 0.f;
#pragma unroll
          for (int c = 0; c < NH; c += 2) top = max3(top, pr[c], pr[c + 1]);
          far = top >= kFar;
        }
        // The first tile, a column without a reference yet, or a weight far above it: the tile's maxima decide.
        if (i == 0 || __syncthreads_or(far)) {
          if (i > 0 && ok) read_scores<NH>(tmem + LY::kTmemS + t_part, pr);
          {
            float v[32];
#pragma unroll
            for (int c = 0; c < 32; ++c)
              v[c] = c < NH && ((vm >> c) & 1u) ? fmaf(ks, pr[c < NH ? c : 0], kl * s.sq[c < NH ? c : 0]) : -INFINITY;
            s.colmax[warp][lane] = reduce_columns<true>(v);
          }
          __syncthreads();
          if (tid < NH) {
            const float old = s.nm[tid], mx = fmaxf(fmaxf(s.colmax[0][tid], s.colmax[1][tid]), fmaxf(s.colmax[2][tid], s.colmax[3][tid]));
            const float now = old == INFINITY || mx + old >= 59.f ? -mx : old;
            s.alpha[tid] = old == INFINITY || now == old ? 1.f : exp2f(now - old);
            s.nm[tid] = now;
          }
          __syncthreads();
#pragma unroll
          for (int c = 0; c < NH; ++c) l[c] *= s.alpha[c];
          to_weights();
        }
#pragma unroll
        for (int c = 0; c < NH; ++c) l[c] += pr[c];
      } else {
        to_weights();
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < NH; ++c) sum += pr[c];
        if (vm != 0u && ok) mass[pos] += sum;
      }
    }
    if constexpr (!kQ4) asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (kPass == 1) {
      float v[32];
#pragma unroll
      for (int c = 0; c < 32; ++c) v[c] = c < NH ? l[c < NH ? c : 0] : 0.f;
      __syncthreads();
      s.colmax[warp][lane] = reduce_columns<false>(v);
      __syncthreads();
      if (tid < rows) {
        const float sum = s.colmax[0][tid] + s.colmax[1][tid] + s.colmax[2][tid] + s.colmax[3][tid];
        part[(size_t)(r0 + tid) * p.nsplit + split] = n > 0 ? make_float2(-s.nm[tid], sum) : make_float2(-INFINITY, 0.f);
      }
    }
    __syncthreads();  // the block is done with the arrays
  };
#pragma unroll 1
  for (int r0 = 0; r0 < rows_all; r0 += kCols) {
    if (rows_all - r0 <= 16) block(Cols<16>(), r0);
    else block(Cols<kCols>(), r0);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(LY::kTmemCols));
}

struct MassPlan {
  int nsplit;
  size_t bytes;
};
MassPlan mass_plan(const cast_ctx* c, int B, int n_layers, int max_rows, int Hq, int Hkv, const Paging& g) {
  MassPlan pl;
  const long long base = (long long)B * n_layers * Hkv, tiles = (g.max_pos() + kTile - 1) / kTile;
  long long n = (8ll * c->num_sms + base - 1) / base;  // two rounds of resident CTAs: sequences differ in length
  if (n > kMaxSplit) n = kMaxSplit;
  if (n > tiles) n = tiles;
  pl.nsplit = (int)(n < 1 ? 1 : n);
  pl.bytes = (size_t)base * max_rows * (Hq / Hkv) * pl.nsplit * sizeof(float2);
  return pl;
}
// What every call needs at most that has no more sequences, layers, rows and positions than these: base * n of mass_plan goes up and
// down with base, but stays below 8 SMs + base, and below base times the tiles or kMaxSplit. (By the plan alone a workspace for 5
// sequences of 32 layers of 8 kv-heads, one piece each, did not hold 4 of them, two pieces each.)
size_t mass_workspace(const cast_ctx* c, int B, int n_layers, int max_rows, int Hq, int Hkv, const Paging& g) {
  const long long base = (long long)B * n_layers * Hkv, tiles = (g.max_pos() + kTile - 1) / kTile;
  long long pieces = base * (tiles < kMaxSplit ? tiles : kMaxSplit);
  if (pieces > 8ll * c->num_sms + base - 1) pieces = 8ll * c->num_sms + base - 1;
  return (size_t)pieces * max_rows * (Hq / Hkv) * sizeof(float2);
}

template <int D, bool kQ4>
cast_status launch_mass(const MassParams& p, int n_layers, cudaStream_t s) {
  const size_t smem = (size_t)(kRB * (D + 4) + kPT * (D + 4) + kRB * (kPT + 4)) * sizeof(float);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.Hkv * p.nsplit, p.B, n_layers);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // launched while its predecessor drains; waits for it
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  CAST_CUDA_OK(cudaFuncSetAttribute(mass_kernel<D, kQ4, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  CAST_CUDA_OK(cudaFuncSetAttribute(mass_kernel<D, kQ4, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  cudaError_t e = cudaLaunchKernelEx(&cfg, mass_kernel<D, kQ4, 1>, p);
  if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, mass_kernel<D, kQ4, 2>, p);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return CAST_ERR_CUDA;
  }
  return CAST_OK;
}

template <int HD, bool kPaged, bool kQ4>
cast_status launch_mass_tc(const MassParams& p, int n_layers, cudaStream_t s) {
  const int smem = MassLay<HD, kQ4>::kSmemMisc + (int)sizeof(MassMisc);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.Hkv * p.nsplit, p.B, n_layers);
  cfg.blockDim = dim3(kThreadsTc, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // launched while its predecessor drains; waits for it
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  auto* const k1 = mass_tc_kernel<HD, kPaged, kQ4, 1>;
  auto* const k2 = mass_tc_kernel<HD, kPaged, kQ4, 2>;
  for (auto* k : {k1, k2}) {
    CAST_CUDA_OK(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    CAST_CUDA_OK(cudaFuncSetAttribute(k, cudaFuncAttributePreferredSharedMemoryCarveout, kQ4 ? 40 : 100));
  }
  cudaError_t e = cudaLaunchKernelEx(&cfg, k1, p);
  if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, k2, p);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return CAST_ERR_CUDA;
  }
  return CAST_OK;
}
template <int HD, bool kQ4>
cast_status launch_mass_tc(const MassParams& p, int n_layers, cudaStream_t s) {
  return p.g.page_size > 0 ? launch_mass_tc<HD, true, kQ4>(p, n_layers, s) : launch_mass_tc<HD, false, kQ4>(p, n_layers, s);
}

cast_status mass_call(cast_ctx* c, const void* q, const void* k, const void* range, bool q4, cast_dtype dtype, int B, int n_layers,
                      size_t q_stride, size_t k_stride, size_t range_stride, int Hq, int Hkv, int D, const Paging& g,
                      const int32_t* path, const int32_t* accept_len, const int32_t* kv_len, float scale, float* mass,
                      void* stream) {
  if (!c || !q || !k || !range || !accept_len || !kv_len || !mass || B < 1 || n_layers < 1 || Hq < 1 || Hkv < 1 ||
      g.page_size < 0 || g.seq_capacity < 1 || (g.page_size > 0 && (!g.table || g.num_pages < 1)) || !on_device(c))
    return CAST_ERR_INVALID_ARG;
  if (dtype != CAST_F32 && dtype != CAST_BF16) return CAST_ERR_DTYPE;
  if (B > c->cfg.max_batch || g.max_pos() > kMaxPositions || n_layers > 65535) return CAST_ERR_CAPACITY;
  if (Hq % Hkv != 0 || (D != 64 && D != 128)) return CAST_ERR_SHAPE;
  if (((uintptr_t)q | (uintptr_t)k | q_stride | k_stride) & 15 || ((uintptr_t)range | range_stride) & 3) return CAST_ERR_SHAPE;
  MassParams p;
  p.q = q; p.k = (const unsigned char*)k; p.range = (const uint32_t*)range;
  p.q_stride = q_stride; p.k_stride = k_stride; p.range_stride = range_stride;
  p.B = B; p.Ncap = c->cfg.max_tree; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv;
  p.path_stride = c->cfg.max_depth + 1;
  p.max_rows = path ? p.path_stride : p.Ncap;
  p.g = g; p.path = path; p.accept_len = accept_len; p.kv_len = kv_len;
  p.scale = scale == 0.f ? 1.0f / sqrtf((float)D) : scale;
  p.scale_log2 = p.scale * 1.4426950408889634f;
  p.mass = mass; p.st = c->state;
  if (!fast_paging(g, B, Hkv, &p.fg)) return CAST_ERR_CAPACITY;
  const MassPlan pl = mass_plan(c, B, n_layers, p.max_rows, Hq, Hkv, g);
  // compute calls never allocate: the workspace comes from cast_reserve_attention_mass
  if (pl.bytes > c->mass_ws_bytes) return CAST_ERR_CAPACITY;
  p.nsplit = pl.nsplit;
  p.part = (float2*)c->mass_ws;
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == CAST_BF16) {
    if (q4) return D == 64 ? launch_mass_tc<64, true>(p, n_layers, s) : launch_mass_tc<128, true>(p, n_layers, s);
    return D == 64 ? launch_mass_tc<64, false>(p, n_layers, s) : launch_mass_tc<128, false>(p, n_layers, s);
  }
  if (q4) return D == 64 ? launch_mass<64, true>(p, n_layers, s) : launch_mass<128, true>(p, n_layers, s);
  return D == 64 ? launch_mass<64, false>(p, n_layers, s) : launch_mass<128, false>(p, n_layers, s);
}

}  // namespace

extern "C" cast_status cast_reserve_attention_mass(cast_ctx* c, cast_dtype dtype, int B, int n_layers, int max_rows, int Hq, int Hkv,
                                                   int D, int page_size, int seq_capacity) {
  const Paging g = {nullptr, page_size, seq_capacity, 0};
  if (!c || B < 1 || n_layers < 1 || max_rows < 1 || Hq < 1 || Hkv < 1 || page_size < 0 || seq_capacity < 1 || !on_device(c))
    return CAST_ERR_INVALID_ARG;
  if (dtype != CAST_F32 && dtype != CAST_BF16) return CAST_ERR_DTYPE;
  if (B > c->cfg.max_batch || g.max_pos() > kMaxPositions || max_rows > CAST_MAX_TREE) return CAST_ERR_CAPACITY;
  if (Hq % Hkv != 0 || (D != 64 && D != 128)) return CAST_ERR_SHAPE;
  return grow_workspace(&c->mass_ws, &c->mass_ws_bytes, mass_workspace(c, B, n_layers, max_rows, Hq, Hkv, g), 0);
}

extern "C" cast_status cast_attention_mass(cast_ctx* c, const void* q, const void* k_cache, cast_dtype dtype, int B, int n_layers,
                                           size_t q_stride_bytes, size_t layer_stride_bytes, int Hq, int Hkv, int D, int page_size,
                                           const int32_t* page_table, int seq_capacity, int num_pages, const int32_t* accept_path,
                                           const int32_t* accept_len, const int32_t* kv_len, float scale, float* mass,
                                           void* stream) {
  const Paging g = {page_table, page_size, seq_capacity, num_pages};
  return mass_call(c, q, k_cache, k_cache, false, dtype, B, n_layers, q_stride_bytes, layer_stride_bytes, 0, Hq, Hkv, D, g,
                   accept_path, accept_len, kv_len, scale, mass, stream);
}

extern "C" cast_status cast_attention_mass_q4(cast_ctx* c, const void* q, const void* k_codes, const void* k_range, cast_dtype dtype,
                                              int B, int n_layers, size_t q_stride_bytes, size_t code_stride_bytes,
                                              size_t range_stride_bytes, int Hq, int Hkv, int D, int page_size,
                                              const int32_t* page_table, int seq_capacity, int num_pages,
                                              const int32_t* accept_path, const int32_t* accept_len, const int32_t* kv_len,
                                              float scale, float* mass, void* stream) {
  const Paging g = {page_table, page_size, seq_capacity, num_pages};
  return mass_call(c, q, k_codes, k_range, true, dtype, B, n_layers, q_stride_bytes, code_stride_bytes, range_stride_bytes, Hq, Hkv,
                   D, g, accept_path, accept_len, kv_len, scale, mass, stream);
}
