// cast_attention_mass, cast_attention_mass_q4: the attention weight that the accepted rows gave every cached position.
//
//   mass[p] += sum_r e^(s_r(p) - m_r) / l_r,   s_r(p) = scale q_r . k_p,   l_r = sum_p e^(s_r(p) - m_r)
//
// over the rows r = (accepted token, head of the group) of a kv-head. The weights need every row's sum first, so the keys are
// read twice: mass_kernel<.., 1> forms each row's (max, sum) over a piece of the sequence, mass_kernel<.., 2> merges the pieces'
// pairs, forms the scores again and adds the weights of a position over the rows in their order. A position's sum belongs to one
// thread group of one CTA: no atomics, the same bits every time.
#include <math.h>

#include "kv_q4.h"

using namespace cast;

namespace {

constexpr int kRB = 32;   // query rows per block
constexpr int kPT = 64;   // positions per tile
constexpr int kThreads = 256;
constexpr int kMaxSplit = 64;

struct MassParams {
  const void* q;
  const unsigned char* k;    // 16-bit or fp32 rows, or codes
  const uint32_t* range;     // 4-bit caches: the pairs
  size_t q_stride, k_stride, range_stride;  // bytes per layer
  int B, Ncap, Hq, Hkv, G, max_rows, nsplit, path_stride;
  Paging g;
  const int32_t* path;
  const int32_t* accept_len;
  const int32_t* kv_len;
  float scale;
  float* mass;
  float2* part;  // [n_layers][B][Hkv][max_rows * G][nsplit] (max, sum)
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

template <typename T, int D, bool kQ4>
__device__ __forceinline__ void load_key_piece(const MassParams& p, int layer, long long row, int ch, float (&f)[16]) {
  if constexpr (kQ4) {
    const uint32_t r = *(reinterpret_cast<const uint32_t*>(reinterpret_cast<const unsigned char*>(p.range) + p.range_stride * layer) + row);
    const uint2 w = *reinterpret_cast<const uint2*>(p.k + p.k_stride * layer + row * (D / 2) + ch * 8);
    const float step = q4_step(r), low = q4_low(r);
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] = fmaf(step, (float)(((e < 8 ? w.x : w.y) >> (4 * (e % 8))) & 15u), low);
  } else {
    const T* src = reinterpret_cast<const T*>(p.k + p.k_stride * layer) + row * D + ch * 16;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) {
      const uint4 a = reinterpret_cast<const uint4*>(src)[i];
      float x[Vec<T>::N];
      Vec<T>::unpack(a, x);
#pragma unroll
      for (int e = 0; e < Vec<T>::N; ++e) f[i * Vec<T>::N + e] = x[e];
    }
  }
}

template <typename T, int D, bool kQ4, int kPass>
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
    const T* q = reinterpret_cast<const T*>(reinterpret_cast<const unsigned char*>(p.q) + p.q_stride * layer);
    for (int i = tid; i < kRB * D; i += kThreads) {
      const int r = i / D, d = i % D, row = r0 + r;
      float x = 0.f;
      if (row < rows) {
        const int j = row / p.G, t = p.path ? p.path[(size_t)b * p.path_stride + j] : j;
        x = to_float(q[(((size_t)b * p.Ncap + t) * p.Hq + kvh * p.G + row % p.G) * D + d]) * p.scale;
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
        if (slot_s[pl] >= 0) load_key_piece<T, D, kQ4>(p, layer, slot_s[pl], ch, f);
#pragma unroll
        for (int e = 0; e < 16; ++e) Ks[pl * KS + ch * 16 + e] = f[e];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = 2 * ty + i, row = r0 + r;
        float acc[4] = {};
#pragma unroll 8
        for (int d = 0; d < D; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[j] = fmaf(Qs[r * KS + d], Ks[(tx + 16 * j) * KS + d], acc[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int pl = tx + 16 * j, pos = tile * kPT + pl;
          const bool vis = row < rows && slot_s[pl] >= 0 && pos < sq.len - sq.n + row / p.G + 1;
          Ss[r * SS + pl] = vis ? acc[j] : -INFINITY;
        }
      }
      __syncthreads();
      if (kPass == 1) {
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) {
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

struct MassPlan {
  int nsplit;
  size_t bytes;
};
MassPlan mass_plan(const cast_ctx* c, int B, int n_layers, int max_rows, int Hq, int Hkv, const Paging& g) {
  MassPlan pl;
  const long long base = (long long)B * n_layers * Hkv, tiles = (g.max_pos() + kPT - 1) / kPT;
  long long n = (4ll * c->num_sms + base - 1) / base;
  if (n > kMaxSplit) n = kMaxSplit;
  if (n > tiles) n = tiles;
  pl.nsplit = (int)(n < 1 ? 1 : n);
  pl.bytes = (size_t)base * max_rows * (Hq / Hkv) * pl.nsplit * sizeof(float2);
  return pl;
}

template <typename T, int D, bool kQ4>
cast_status launch_mass(cast_ctx* c, const MassParams& p, int n_layers, cudaStream_t s) {
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
  CAST_CUDA_OK(cudaFuncSetAttribute(mass_kernel<T, D, kQ4, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  CAST_CUDA_OK(cudaFuncSetAttribute(mass_kernel<T, D, kQ4, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
  cudaError_t e = cudaLaunchKernelEx(&cfg, mass_kernel<T, D, kQ4, 1>, p);
  if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, mass_kernel<T, D, kQ4, 2>, p);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return CAST_ERR_CUDA;
  }
  return CAST_OK;
}

cast_status mass_call(cast_ctx* c, const void* q, const void* k, const void* range, bool q4, cast_dtype dtype, int B, int n_layers,
                      size_t q_stride, size_t k_stride, size_t range_stride, int Hq, int Hkv, int D, const Paging& g,
                      const int32_t* path, const int32_t* accept_len, const int32_t* kv_len, float scale, float* mass,
                      void* stream) {
  if (!c || !q || !k || !range || !accept_len || !kv_len || !mass || B < 1 || n_layers < 1 || Hq < 1 || Hkv < 1 ||
      g.page_size < 0 || g.seq_capacity < 1 || (g.page_size > 0 && (!g.table || g.num_pages < 1)) || !on_device(c))
    return CAST_ERR_INVALID_ARG;
  if (dtype != CAST_F32 && dtype != CAST_BF16) return CAST_ERR_DTYPE;
  if (B > c->cfg.max_batch || g.max_pos() > 0x7fffffffll || n_layers > 65535) return CAST_ERR_CAPACITY;
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
  p.mass = mass; p.st = c->state;
  const MassPlan pl = mass_plan(c, B, n_layers, p.max_rows, Hq, Hkv, g);
  // compute calls never allocate: the workspace comes from cast_reserve_attention_mass
  if (pl.bytes > c->mass_ws_bytes) return CAST_ERR_CAPACITY;
  p.nsplit = pl.nsplit;
  p.part = (float2*)c->mass_ws;
  cudaStream_t s = (cudaStream_t)stream;
  if (q4) {
    if (dtype == CAST_F32) return D == 64 ? launch_mass<float, 64, true>(c, p, n_layers, s) : launch_mass<float, 128, true>(c, p, n_layers, s);
    return D == 64 ? launch_mass<__nv_bfloat16, 64, true>(c, p, n_layers, s) : launch_mass<__nv_bfloat16, 128, true>(c, p, n_layers, s);
  }
  if (dtype == CAST_F32) return D == 64 ? launch_mass<float, 64, false>(c, p, n_layers, s) : launch_mass<float, 128, false>(c, p, n_layers, s);
  return D == 64 ? launch_mass<__nv_bfloat16, 64, false>(c, p, n_layers, s) : launch_mass<__nv_bfloat16, 128, false>(c, p, n_layers, s);
}

}  // namespace

extern "C" cast_status cast_reserve_attention_mass(cast_ctx* c, cast_dtype dtype, int B, int n_layers, int max_rows, int Hq, int Hkv,
                                                   int D, int page_size, int seq_capacity) {
  const Paging g = {nullptr, page_size, seq_capacity, 0};
  if (!c || B < 1 || n_layers < 1 || max_rows < 1 || Hq < 1 || Hkv < 1 || page_size < 0 || seq_capacity < 1 || !on_device(c))
    return CAST_ERR_INVALID_ARG;
  if (dtype != CAST_F32 && dtype != CAST_BF16) return CAST_ERR_DTYPE;
  if (B > c->cfg.max_batch || g.max_pos() > 0x7fffffffll || max_rows > CAST_MAX_TREE) return CAST_ERR_CAPACITY;
  if (Hq % Hkv != 0 || (D != 64 && D != 128)) return CAST_ERR_SHAPE;
  return grow_workspace(&c->mass_ws, &c->mass_ws_bytes, mass_plan(c, B, n_layers, max_rows, Hq, Hkv, g).bytes, 0);
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
