// cast_chunk_attention and cast_tree_attention_window: attention of new tokens over the cache, causal or under a tree's mask, with an
// optional sliding window and its sinks. Here the entry points and the CUDA-core kernel: fp32 inputs, and the bf16 shapes that the tensor-core
// kernel does not take (chunk_attention_tc.cu).
//
// One CTA works its stretch of the line of tiles (chunk_attn.h) item by item: 32 query rows of one kv-head against tiles of 64 positions,
// both in fp32 in shared memory; S = Q K^T by packed multiply-adds, an online softmax, O += P V in registers. Positions that no row of the
// item sees are neither loaded nor looked up (pages outside the window may be gone) and stand as zeros; a tile that some rows see only in
// part takes the products with hidden positions out one by one, so that no value of a hidden row, NaN or infinity, reaches a row's output.
// Bound by the chain of a tile: products by packed multiply-adds from shared memory, a warp's softmax, three barriers, 5 us in all, so small calls spread over all CTAs tile by tile.
#include <math.h>

#include "chunk_attn.h"

using namespace cast;

namespace cast {
// implemented in chunk_attention_tc.cu
size_t chunk_attention_tc_workspace(const cast_ctx* c, int D);
bool chunk_attention_tc_launch(cast_ctx* c, ChunkParams& p, int D, void* workspace, cudaStream_t s, cast_status* status);
}

namespace {

constexpr int kRB = 32;
constexpr int kPT = 64;
constexpr int kThreads = 256;
constexpr size_t kTicketBytes = 2 * kChunkGrid * sizeof(int32_t);

typedef unsigned long long f32x2;
__device__ __forceinline__ float sum2(f32x2 v) {
  return __uint_as_float((uint32_t)v) + __uint_as_float((uint32_t)(v >> 32));
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ void store4(float* p, const float (&x)[4], float f) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&x)[4], float f) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x[0] * f, x[1] * f), b = __floats2bfloat162_rn(x[2] * f, x[3] * f);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

template <bool V> struct Choice { static constexpr bool value = V; };

template <typename T, int D, bool kTree>
__global__ void __launch_bounds__(kThreads, 2) chunk_attn_cc_kernel(const ChunkParams p) {
  constexpr int KS = D + 4, SS = kPT + 4;     // row strides (floats)
  constexpr int CH = Vec<T>::N, CPR = D / CH; // elements per 16-byte chunk, chunks per row
  constexpr int DC = D / 32;                  // output columns per lane
  extern __shared__ __align__(16) float smem[];
  float* Qs = smem;            // [kRB][KS]
  float* Ks = Qs + kRB * KS;   // [kPT][KS]
  float* Vs = Ks + kPT * KS;   // [kPT][D]
  float* Ss = Vs + kPT * D;    // [kRB][SS]
  __shared__ ChunkPlan plan;
  __shared__ float row_m[kRB], row_l[kRB], row_alpha[kRB];
  __shared__ RowSight sight[kRB];
  __shared__ uint32_t anc_s[kRB][CAST_MAX_TREE / 32];
  __shared__ long long slot_s[2][kPT];
  __shared__ int s_last;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  make_plan<kPT, kTree>(p, plan);
  ChunkWalk w;
  const T* q = reinterpret_cast<const T*>(p.q);
  const T* kc = reinterpret_cast<const T*>(p.k);
  const T* vc = reinterpret_cast<const T*>(p.v);
  T* out = reinterpret_cast<T*>(p.out);
  const int ty = tid / 16, tx = tid % 16, G = p.G;

  for (bool more = walk_begin<kPT, kTree>(p, plan, w, blockIdx.x); more; more = walk_next<kPT, kTree>(p, plan, w)) {
    const Span sp = w.span;
    const bool nothing = sp.n == 0;  // (a sequence past its capacity: its rows see nothing)
    if (w.t1 <= w.t0 && !(nothing && w.at == w.item0)) continue;
    const ChunkSeq s = plan.seq[w.b];
    const int rows_total = (s.n - s.F) * G, row0 = w.rb * kRB, kvh = w.h, b = w.b;
    const int rows_here = min(rows_total - row0, kRB);
    __syncthreads();  // the item before is over
    auto find_slots = [&](int i) {  // cache slots of a tile's positions, a tile ahead of their use
      if (tid >= kPT) return;
      long long slot = -1;
      if (i < w.t1) {
        const int pos = sp.tile(i) * kPT + tid;
        int page, in_page;
        if (pos < sp.hi && (pos >= sp.lo || pos < sp.s_end)) {
          if (find_place(p.g, b, pos, page, in_page)) slot = (long long)page * (p.g.page_size == 0 ? p.g.seq_capacity : p.g.page_size) + in_page;
          else report(p.st, CAST_ERR_BAD_PAGE, b);
        }
      }
      slot_s[i & 1][tid] = slot;
    };
    find_slots(w.t0);
    auto row_at = [&](int r) {  // a row's first element in q and out
      const int row = row0 + r, t = s.F + row / G;
      return (((size_t)s.off + t) * p.Hq + kvh * G + row % G) * D;
    };
    for (int i = tid; i < kRB * CPR; i += kThreads) {
      const int r = i / CPR, ch = i % CPR;
      float f[CH] = {};
      if (r < rows_here) Vec<T>::unpack(*reinterpret_cast<const uint4*>(q + row_at(r) + ch * CH), f);
#pragma unroll
      for (int e = 0; e < CH; ++e) Qs[r * KS + ch * CH + e] = f[e] * p.scale;
    }
    if (tid < kRB) {
      row_m[tid] = -INFINITY;
      row_l[tid] = 0.f;
      RowSight rs = {0, 0, 0};
      uint32_t a[CAST_MAX_TREE / 32] = {};
      if (tid < rows_here) {
        const int t = s.F + (row0 + tid) / G;
        const int depth = kTree ? depth_of(p, s, t) : 0;
        rs = sight_of<kTree>(p, s, t, depth);
        if (kTree)
          for (int wd = 0; wd < CAST_MAX_TREE / 32; ++wd) a[wd] = tree_word(p, s, t, depth, wd);
      }
      sight[tid] = rs;
      for (int wd = 0; wd < CAST_MAX_TREE / 32; ++wd) anc_s[tid][wd] = a[wd];
    }
    float o[4][DC];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < DC; ++e) o[i][e] = 0.f;

    // A tile's rows on their way, in registers: they are read under the softmax and the products of the tile before as far as
    // 128 registers a thread, two CTAs per SM, hold them: of 128 dims the keys alone, in fp32 none.
    constexpr int NL = kPT * CPR / kThreads;
    constexpr bool kAheadK = NL <= 4, kAheadV = D == 64;
    uint4 next_k[NL], next_v[NL];
    auto row_of = [&](int i, int x, const T* cache) {
      const int j = tid + x * kThreads;
      const long long slot = slot_s[i & 1][j / CPR];
      return slot >= 0 ? *reinterpret_cast<const uint4*>(cache + ((size_t)slot * p.Hkv + kvh) * D + j % CPR * CH) : make_uint4(0u, 0u, 0u, 0u);
    };
    auto fetch = [&](int i) {
#pragma unroll
      for (int x = 0; x < NL; ++x) {
        if (kAheadK) next_k[x] = row_of(i, x, kc);
        if (kAheadV) next_v[x] = row_of(i, x, vc);
      }
    };
    __syncthreads();  // the slots, Qs, sight, anc_s
    if (w.t0 < w.t1) fetch(w.t0);
    for (int i = w.t0; i < w.t1; ++i) {
      const int pbase = sp.tile(i) * kPT;
      __syncthreads();  // previous tile consumed
#pragma unroll 4
      for (int x = 0; x < NL; ++x) {
        const int j = tid + x * kThreads, pl = j / CPR, ch = j % CPR;
        float fk[CH], fv[CH];
        Vec<T>::unpack(kAheadK ? next_k[x] : row_of(i, x, kc), fk);
        Vec<T>::unpack(kAheadV ? next_v[x] : row_of(i, x, vc), fv);
#pragma unroll
        for (int e = 0; e < CH; e += 4) {
          *reinterpret_cast<float4*>(Ks + pl * KS + ch * CH + e) = make_float4(fk[e], fk[e + 1], fk[e + 2], fk[e + 3]);
          *reinterpret_cast<float4*>(Vs + pl * D + ch * CH + e) = make_float4(fv[e], fv[e + 1], fv[e + 2], fv[e + 3]);
        }
      }
      find_slots(i + 1);
      __syncthreads();
      {  // S: thread (ty, tx) owns rows 2ty, 2ty+1 and positions tx, tx+16, tx+32, tx+48
        f32x2 acc[2][4] = {};
#pragma unroll 8
        for (int d = 0; d < D; d += 4) {
          const ulonglong2 q0 = *reinterpret_cast<const ulonglong2*>(Qs + (2 * ty) * KS + d);
          const ulonglong2 q1 = *reinterpret_cast<const ulonglong2*>(Qs + (2 * ty + 1) * KS + d);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const ulonglong2 kk = *reinterpret_cast<const ulonglong2*>(Ks + (tx + 16 * j) * KS + d);
            acc[0][j] = fma2(q0.y, kk.y, fma2(q0.x, kk.x, acc[0][j]));
            acc[1][j] = fma2(q1.y, kk.y, fma2(q1.x, kk.x, acc[1][j]));
          }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int r = 2 * ty + u;
          const RowSight rs = sight[r];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int pl = tx + 16 * j, pos = pbase + pl;
            bool vis = pos < rs.hi && (pos >= rs.lo || pos < rs.sinks);
            if (kTree && pos >= s.L && pos - s.L < CAST_MAX_TREE) vis = (anc_s[r][(pos - s.L) >> 5] >> ((pos - s.L) & 31)) & 1u;
            Ss[r * SS + pl] = vis && slot_s[i & 1][pl] >= 0 ? sum2(acc[u][j]) : -INFINITY;
          }
        }
      }
      __syncthreads();
      if (i + 1 < w.t1) fetch(i + 1);
      // online softmax and O += P V: warp w owns rows 4w .. 4w+3
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        const int r = 4 * warp + rr;
        const float s0 = Ss[r * SS + lane], s1 = Ss[r * SS + lane + 32];
        float mx = fmaxf(s0, s1);
#pragma unroll
        for (int of = 16; of > 0; of >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, of));
        const float m_old = row_m[r], m_new = fmaxf(m_old, mx);
        float p0 = 0.f, p1 = 0.f, alpha = 1.f;
        if (m_new > -INFINITY) {
          p0 = expf(s0 - m_new);
          p1 = expf(s1 - m_new);
          alpha = expf(m_old - m_new);
        }
        float sum = p0 + p1;
#pragma unroll
        for (int of = 16; of > 0; of >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, of);
        if (__any_sync(0xffffffffu, s0 != s0 || s1 != s1)) sum = __int_as_float(0x7fffffff);  // (the maximum passes over NaN)
        __syncwarp();
        Ss[r * SS + lane] = p0;
        Ss[r * SS + lane + 32] = p1;
        if (lane == 0) {
          row_m[r] = m_new;
          row_l[r] = row_l[r] * alpha + sum;
          row_alpha[r] = alpha;
        }
      }
      __syncwarp();
#pragma unroll
      for (int rr = 0; rr < 4; ++rr) {
        const float a = row_alpha[4 * warp + rr];
#pragma unroll
        for (int e = 0; e < DC; ++e) o[rr][e] *= a;
      }
      // whether a position of this tile that was loaded is hidden from a row of the item (a bound on it, the same for all)
      const int tf = s.F + row0 / G, tl = s.F + (row0 + rows_here - 1) / G;
      const bool part = kTree ? pbase + kPT > s.L || (p.window > 0 && (long long)pbase < (long long)s.L + CAST_MAX_TREE + 1 - p.window)
                              : (long long)pbase + kPT > (long long)s.L + tf || (p.window > 0 && (long long)pbase <= (long long)s.L + tl - p.window);
      auto products = [&](auto kPart) {
#pragma unroll 4
        for (int pl = 0; pl < kPT; pl += 4) {
          float4 pv[4];
#pragma unroll
          for (int rr = 0; rr < 4; ++rr) pv[rr] = *reinterpret_cast<const float4*>(Ss + (4 * warp + rr) * SS + pl);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            float vv[DC];
            if constexpr (DC == 4) {
              const float4 t4 = *reinterpret_cast<const float4*>(Vs + (pl + x) * D + lane * 4);
              vv[0] = t4.x; vv[1] = t4.y; vv[2] = t4.z; vv[3] = t4.w;
            } else {
              const float2 t2 = *reinterpret_cast<const float2*>(Vs + (pl + x) * D + lane * 2);
              vv[0] = t2.x; vv[1] = t2.y;
            }
#pragma unroll
            for (int rr = 0; rr < 4; ++rr) {
              const float wt = x == 0 ? pv[rr].x : x == 1 ? pv[rr].y : x == 2 ? pv[rr].z : pv[rr].w;
              if (!decltype(kPart)::value || wt != 0.f) {
#pragma unroll
                for (int e = 0; e < DC; ++e) o[rr][e] += wt * vv[e];
              }
            }
          }
        }
      };
      if (part) products(Choice<true>{});
      else products(Choice<false>{});
    }
    __syncthreads();
    // rows to shared memory (the keys' place), then in contiguous pieces: the output, or this CTA's partial
    float* Os = Ks;
#pragma unroll
    for (int rr = 0; rr < 4; ++rr)
#pragma unroll
      for (int e = 0; e < DC; ++e) Os[(4 * warp + rr) * KS + lane * DC + e] = o[rr][e];
    __syncthreads();
    constexpr int C4 = D / 4;
    if (w.t0 == 0 && w.t1 == sp.n) {
      for (int i = tid; i < rows_here * C4; i += kThreads) {
        const int r = i / C4, c = i % C4 * 4;
        const float4 v = *reinterpret_cast<const float4*>(Os + r * KS + c);
        const float x[4] = {v.x, v.y, v.z, v.w};
        store4(out + row_at(r) + c, x, row_l[r] == 0.f ? 0.f : 1.f / row_l[r]);
      }
      continue;
    }
    const int c_lo = owner_of(plan, w.item0 + kItemCost), c_hi = owner_of(plan, w.item0 + kItemCost + sp.n - 1);
    auto place = [&](int c) { return ((size_t)c * 2 + (c == c_lo ? 1 : 0)) * kRB; };
    const size_t mine = place(blockIdx.x);
    for (int i = tid; i < rows_here * C4; i += kThreads) {
      const int r = i / C4, c = i % C4 * 4;
      __stcg(reinterpret_cast<float4*>(p.part_o + (mine + r) * D + c), *reinterpret_cast<const float4*>(Os + r * KS + c));
    }
    if (tid < rows_here) __stcg(p.part_ml + mine + tid, make_float2(row_m[tid], row_l[tid]));
    __syncthreads();
    if (tid == 0) {
      // releases this CTA's partial (the barrier made it this thread's to release), acquires those that came earlier
      int t;
      asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(t) : "l"(p.ticket + c_lo) : "memory");
      s_last = t == c_hi - c_lo;
      if (t == c_hi - c_lo) p.ticket[c_lo] = 0;  // ready for the next launch
    }
    __syncthreads();
    if (!s_last) continue;
    for (int r = warp; r < rows_here; r += kThreads / 32) {
      float M = -INFINITY;
      for (int c = c_lo; c <= c_hi; ++c) M = fmaxf(M, __ldcg(p.part_ml + place(c) + r).x);
      float l = 0.f, acc[DC] = {};
#pragma unroll 4
      for (int c = c_lo; c <= c_hi; ++c) {
        const float2 ml = __ldcg(p.part_ml + place(c) + r);
        // a part that saw nothing weighs nothing; one whose reference is -inf for NaN has its sum say so
        const float wt = ml.x > -INFINITY ? expf(ml.x - M) : ml.y == 0.f ? 0.f : 1.f;
        l += wt * ml.y;
        const float* src = p.part_o + (place(c) + r) * D + lane * DC;
#pragma unroll
        for (int e = 0; e < DC; ++e) acc[e] += wt * __ldcg(src + e);
      }
      const float inv = l == 0.f ? 0.f : 1.f / l;
      T* dst = out + row_at(r) + lane * DC;
#pragma unroll
      for (int e = 0; e < DC; ++e) {
        if constexpr (sizeof(T) == 4) dst[e] = acc[e] * inv;
        else dst[e] = __float2bfloat16(acc[e] * inv);
      }
    }
  }
}

template <typename T, int D, bool kTree>
cast_status launch_cc(cast_ctx* c, ChunkParams& p, cudaStream_t s) {
  p.block_rows = kRB;
  p.block_tokens = kRB % p.G == 0 ? kRB / p.G : 0;
  p.min_units = kItemCost + 1;  // (a tile is 5 us here, more than what a split costs; 3 sequences of 20-131 tokens under a window of 256, 8/8 heads of 64 dims: 38 us, from two tiles on 45)
  p.join = 0.f;  // (tiles are long enough here that every part pays)
  const int grid = 2 * c->num_sms < kChunkGrid ? 2 * c->num_sms : kChunkGrid;
  p.part_o = reinterpret_cast<float*>(reinterpret_cast<char*>(c->chunk_ws) + kTicketBytes);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + (size_t)kChunkGrid * 2 * kRB * D);
  const size_t smem = (size_t)(kRB * (D + 4) + kPT * (D + 4) + kPT * D + kRB * (kPT + 4)) * sizeof(float);
  auto kern = chunk_attn_cc_kernel<T, D, kTree>;
  CAST_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // launched while its predecessor drains; waits for it
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kern, p) != cudaSuccess) {
    cudaGetLastError();
    return CAST_ERR_CUDA;
  }
  return launch_status();
}

// A bf16 call goes either way by its shape: both workspaces fit.
size_t workspace(const cast_ctx* c, cast_dtype dtype, int D) {
  const size_t cc = (size_t)kChunkGrid * 2 * kRB * (D + 2) * sizeof(float);
  const size_t tc = dtype == CAST_BF16 ? chunk_attention_tc_workspace(c, D) : 0;
  return kTicketBytes + (cc > tc ? cc : tc);
}

template <bool kTree>
cast_status attend(cast_ctx* c, ChunkParams& p, cast_dtype dtype, int D, float scale, void* stream) {
  if (!c || !p.q || !p.k || !p.v || !p.kv_len || !p.n_new || !p.out || p.B < 1 || p.rows < 1 || p.Hq < 1 || p.Hkv < 1 || p.window < 0 ||
      p.sinks < 0 || p.g.page_size < 0 || p.g.seq_capacity < 1 || (p.g.page_size > 0 && (!p.g.table || p.g.num_pages < 1)) || !on_device(c))
    return CAST_ERR_INVALID_ARG;
  if (dtype != CAST_F32 && dtype != CAST_BF16) return CAST_ERR_DTYPE;
  if (p.Hq % p.Hkv != 0 || (D != 64 && D != 128)) return CAST_ERR_SHAPE;
  if (((uintptr_t)p.q | (uintptr_t)p.k | (uintptr_t)p.v | (uintptr_t)p.out) & 15) return CAST_ERR_SHAPE;
  // (rows of a sequence and positions are counted in 32 bits)
  if (p.B > c->cfg.max_batch || p.g.max_pos() > kMaxPositions || (long long)p.B * p.rows > kMaxPositions ||
      (long long)p.rows * (p.Hq / p.Hkv) > kMaxPositions || workspace(c, dtype, D) > c->chunk_ws_bytes)
    return CAST_ERR_CAPACITY;
  p.G = p.Hq / p.Hkv;
  p.max_pos = (int)p.g.max_pos();
  p.scale = scale == 0.f ? 1.0f / sqrtf((float)D) : scale;
  p.st = c->state;
  cudaStream_t s = (cudaStream_t)stream;
  p.ticket = reinterpret_cast<int32_t*>(c->chunk_ws);
  cast_status st;
  if (dtype == CAST_BF16 && chunk_attention_tc_launch(c, p, D, reinterpret_cast<char*>(c->chunk_ws) + kTicketBytes, s, &st)) return st;
  if (dtype == CAST_BF16) return D == 64 ? launch_cc<__nv_bfloat16, 64, kTree>(c, p, s) : launch_cc<__nv_bfloat16, 128, kTree>(c, p, s);
  return D == 64 ? launch_cc<float, 64, kTree>(c, p, s) : launch_cc<float, 128, kTree>(c, p, s);
}

}  // namespace

extern "C" cast_status cast_reserve_chunk_attention(cast_ctx* c, cast_dtype dtype, int D) {
  if (!c || !on_device(c)) return CAST_ERR_INVALID_ARG;
  if (dtype != CAST_F32 && dtype != CAST_BF16) return CAST_ERR_DTYPE;
  if (D != 64 && D != 128) return CAST_ERR_SHAPE;
  // tickets start at zero; every merge leaves its ticket at zero again
  return grow_workspace(&c->chunk_ws, &c->chunk_ws_bytes, workspace(c, dtype, D), kTicketBytes);
}

extern "C" cast_status cast_chunk_attention(cast_ctx* c, const void* q, const void* k_cache, const void* v_cache, cast_dtype dtype, int B,
                                            int rows, const int32_t* row_start, int Hq, int Hkv, int D, int page_size,
                                            const int32_t* page_table, int seq_capacity, int num_pages, const int32_t* kv_len,
                                            const int32_t* n_new, int window, int sinks, float scale, void* out, void* stream) {
  ChunkParams p = {};
  p.q = q; p.k = k_cache; p.v = v_cache; p.out = out;
  p.B = B; p.rows = rows; p.Hq = Hq; p.Hkv = Hkv;
  p.window = window; p.sinks = sinks;
  p.row_start = row_start; p.kv_len = kv_len; p.n_new = n_new;
  p.g = {page_table, page_size, seq_capacity, num_pages};
  return attend<false>(c, p, dtype, D, scale, stream);
}

extern "C" cast_status cast_tree_attention_window(cast_ctx* c, const void* q, const void* k_cache, const void* v_cache, cast_dtype dtype,
                                                  int B, int Hq, int Hkv, int D, int page_size, const int32_t* page_table,
                                                  int seq_capacity, int num_pages, const int32_t* kv_len, const uint32_t* anc_mask,
                                                  const int32_t* depth, const int32_t* n_tree, const int32_t* first_row, int window,
                                                  int sinks, float scale, void* out, void* stream) {
  if (!c || !anc_mask || !depth) return CAST_ERR_INVALID_ARG;
  ChunkParams p = {};
  p.q = q; p.k = k_cache; p.v = v_cache; p.out = out;
  p.B = B; p.rows = c->cfg.max_tree; p.Hq = Hq; p.Hkv = Hkv;
  p.Nmax = c->cfg.total_token;
  p.window = window; p.sinks = sinks;
  p.kv_len = kv_len; p.n_new = n_tree; p.first_row = first_row; p.depth = depth; p.anc = anc_mask; p.words = c->words;
  p.g = {page_table, page_size, seq_capacity, num_pages};
  return attend<true>(c, p, dtype, D, scale, stream);
}
