// cast_store_kv_q4, cast_load_kv_q4, cast_compact_kv_q4: rows into the 4-bit cache, out of it, and to the front of the tree
// region after acceptance. All three are bound by memory.
#include "kv_q4.h"

using namespace cast;

namespace {

constexpr int kThreads = 256;
constexpr int kLane = 16;  // dimensions per thread: 8 bytes of codes, so a row's D / 16 threads write whole 32-byte sectors

struct RowsParams {
  const void* k;  // [n_layers][B][rows][Hkv][D]; load: written
  const void* v;
  unsigned char *kc, *vc;
  uint32_t *kr, *vr;
  size_t code_stride, range_stride;
  int B, rows, Hkv;
  Paging g;
  const int32_t* start;
  const int32_t* n_rows;
  DevState* st;
};

template <typename T>
__device__ __forceinline__ void load16(const T* p, float (&x)[kLane]);
template <>
__device__ __forceinline__ void load16<float>(const float* p, float (&x)[kLane]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 a = __ldcs(reinterpret_cast<const float4*>(p) + i);
    x[4 * i] = a.x; x[4 * i + 1] = a.y; x[4 * i + 2] = a.z; x[4 * i + 3] = a.w;
  }
}
template <>
__device__ __forceinline__ void load16<__nv_bfloat16>(const __nv_bfloat16* p, float (&x)[kLane]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p) + i);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[8 * i + 2 * e] = __uint_as_float(w[e] << 16);
      x[8 * i + 2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ void store16(float* p, const float (&x)[kLane]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) __stcs(reinterpret_cast<float4*>(p) + i, make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]));
}
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float (&x)[kLane]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[8 * i + 2 * e], x[8 * i + 2 * e + 1]);
      w[e] = *reinterpret_cast<const uint32_t*>(&h);
    }
    __stcs(reinterpret_cast<uint4*>(p) + i, make_uint4(w[0], w[1], w[2], w[3]));
  }
}

// The row's codes and its pair, from the D / 16 threads that hold it. The quotient is that of a division, rounded to nearest even,
// everywhere: the product with 1 / step is off by less than 4e-6 there (two roundings, quotients below 16), so it decides
// unless it lies within 1e-4 of a half, or 1 / step is out of range.
template <int LPR>
__device__ __forceinline__ uint2 quantise(const float (&x)[kLane], uint32_t& range) {
  float lo = x[0], hi = x[0], bad = 0.f;
#pragma unroll
  for (int e = 0; e < kLane; ++e) {
    lo = fminf(lo, x[e]);
    hi = fmaxf(hi, x[e]);
    bad = fmaf(x[e], 0.f, bad);  // NaN once a value is not finite (fminf and fmaxf pass over NaN)
  }
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    bad += __shfl_xor_sync(0xffffffffu, bad, o);
  }
  const float span = hi - lo;
  const __nv_bfloat16 step_h = __float2bfloat16_rn(__fdiv_rn(span, 15.f)), low_h = __float2bfloat16_rn(lo);
  if (!(bad == 0.f) || !(span < INFINITY) || !(fabsf(__bfloat162float(low_h)) < INFINITY)) {
    range = 0x7fc07fc0u;
    return make_uint2(0u, 0u);
  }
  range = (uint32_t)__bfloat16_as_ushort(step_h) | ((uint32_t)__bfloat16_as_ushort(low_h) << 16);
  const float step = __bfloat162float(step_h), low = __bfloat162float(low_h);
  if (step == 0.f) return make_uint2(0u, 0u);
  const float inv = __fdiv_rn(1.f, step);
  const bool far = !(inv < 1e37f);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < kLane; ++e) {
    const float d = __fsub_rn(x[e], low);
    float t = d * inv, q = rintf(t);
    if (far || fabsf(t - q) > 0.4999f) q = rintf(__fdiv_rn(d, step));
    w[e / 8] |= (uint32_t)fminf(fmaxf(q, 0.f), 15.f) << (4 * (e % 8));
  }
  return make_uint2(w[0], w[1]);
}

// D / 16 threads per row, K and V of it side by side. kStore: into the cache, else out of it.
template <typename T, int D, bool kStore>
__global__ void __launch_bounds__(kThreads) q4_rows_kernel(const RowsParams p) {
  constexpr int LPR = D / kLane;
  const int b = blockIdx.y, layer = blockIdx.z;
  const long long i = (long long)blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
  const int part = threadIdx.x % LPR;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int n = min(p.n_rows[b], p.rows);
  const int t = (int)(i / p.Hkv), h = (int)(i - (long long)t * p.Hkv);
  const unsigned here = __ballot_sync(0xffffffffu, t < n);
  if (here == 0u) return;  // (a row's threads are in one warp: whole warps leave, the others go on together)
  const bool live = t < n;
  long long pos = live ? (long long)(p.start ? p.start[b] : 0) + t : 0;
  int page = 0, slot = 0;
  const bool ok = live && pos >= 0 && pos < p.g.max_pos() && find_place(p.g, b, (int)pos, page, slot);
  if (live && !ok && part == 0) report(p.st, CAST_ERR_BAD_PAGE, b);
  const long long row = ok ? q4_row(p.g, p.Hkv, h, page, slot) : 0;
  const size_t at = ((((size_t)layer * p.B + b) * p.rows + (live ? t : 0)) * p.Hkv + h) * D + part * kLane;
  unsigned char* const kc = p.kc + p.code_stride * layer + row * (D / 2) + part * 8;
  unsigned char* const vc = p.vc + p.code_stride * layer + row * (D / 2) + part * 8;
  uint32_t* const kr = reinterpret_cast<uint32_t*>(reinterpret_cast<unsigned char*>(p.kr) + p.range_stride * layer) + row;
  uint32_t* const vr = reinterpret_cast<uint32_t*>(reinterpret_cast<unsigned char*>(p.vr) + p.range_stride * layer) + row;
  if (kStore) {
    float xk[kLane] = {}, xv[kLane] = {};
    if (live) {
      load16(reinterpret_cast<const T*>(p.k) + at, xk);
      load16(reinterpret_cast<const T*>(p.v) + at, xv);
    }
    uint32_t rk, rv;
    const uint2 ck = quantise<LPR>(xk, rk), cv = quantise<LPR>(xv, rv);
    if (!ok) return;
    *reinterpret_cast<uint2*>(kc) = ck;
    *reinterpret_cast<uint2*>(vc) = cv;
    if (part == 0) {
      *kr = rk;
      *vr = rv;
    }
  } else {
    if (!ok) return;
    const uint2 c[2] = {*reinterpret_cast<const uint2*>(kc), *reinterpret_cast<const uint2*>(vc)};
    const uint32_t r[2] = {*kr, *vr};
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const float step = q4_step(r[w]), low = q4_low(r[w]);
      float x[kLane];
#pragma unroll
      for (int e = 0; e < kLane; ++e) x[e] = fmaf(step, (float)(((e < 8 ? c[w].x : c[w].y) >> (4 * (e % 8))) & 15u), low);
      store16(reinterpret_cast<T*>(const_cast<void*>(w ? p.v : p.k)) + at, x);
    }
  }
}

template <bool kStore>
cast_status launch_rows(cast_ctx* c, RowsParams& p, cast_dtype dtype, int n_layers, int D, cudaStream_t s) {
  const long long per = kThreads / (D / kLane), blocks = ((long long)p.rows * p.Hkv + per - 1) / per;
  if (blocks > 0x7fffffffll || n_layers > 65535) return CAST_ERR_CAPACITY;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks, p.B, n_layers);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // launched while its predecessor drains; waits for it
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  auto* const kern = dtype == CAST_F32 ? (D == 64 ? q4_rows_kernel<float, 64, kStore> : q4_rows_kernel<float, 128, kStore>)
                                       : (D == 64 ? q4_rows_kernel<__nv_bfloat16, 64, kStore> : q4_rows_kernel<__nv_bfloat16, 128, kStore>);
  if (cudaLaunchKernelEx(&cfg, kern, p) != cudaSuccess) {
    cudaGetLastError();
    return CAST_ERR_CUDA;
  }
  return CAST_OK;
}

template <bool kStore>
cast_status rows_call(cast_ctx* c, const void* k, const void* v, cast_dtype dtype, int B, int n_layers, int rows, int Hkv, int D,
                      const Paging& g, const int32_t* start, const int32_t* n_rows, const void* kc, const void* kr,
                      const void* vc, const void* vr, size_t code_stride, size_t range_stride, void* stream) {
  if (!k || !v || !n_rows || n_layers < 1 || rows < 1) return CAST_ERR_INVALID_ARG;
  if (dtype != CAST_F32 && dtype != CAST_BF16) return CAST_ERR_DTYPE;
  const cast_status st = check_q4(c, B, Hkv, D, g, kc, kr, vc, vr, code_stride, range_stride);
  if (st != CAST_OK) return st;
  if (((uintptr_t)k | (uintptr_t)v) & 15) return CAST_ERR_SHAPE;
  RowsParams p;
  p.k = k; p.v = v;
  p.kc = (unsigned char*)kc; p.vc = (unsigned char*)vc; p.kr = (uint32_t*)kr; p.vr = (uint32_t*)vr;
  p.code_stride = code_stride; p.range_stride = range_stride;
  p.B = B; p.rows = rows; p.Hkv = Hkv; p.g = g; p.start = start; p.n_rows = n_rows; p.st = c->state;
  return launch_rows<kStore>(c, p, dtype, n_layers, D, (cudaStream_t)stream);
}

// ---- compaction: as that of the 16-bit cache (the same conditions on the path, the same publication of the length), a thread
// per 16 bytes of codes or pair of one kv-head.
constexpr int kCompactThreads = 128;
constexpr int kMaxPath = CAST_MAX_DEPTH + 1;

struct CompactParams {
  unsigned char* base[4];  // K codes, V codes, K pairs, V pairs
  size_t code_stride, range_stride;
  int Hkv, D, H1;
  Paging g;
  const int32_t* accept_path;
  const int32_t* accept_len;
  int32_t* kv_len;
  int32_t* ticket;
  DevState* st;
};

// All loads of a column come before its stores, and a path entry is no smaller than its place: a destination is never the
// source of a later entry.
template <typename V>
__device__ __forceinline__ void move_column(unsigned char* at, size_t row_bytes, const long long* src, const long long* dst, int n) {
  V buf[kMaxPath];
#pragma unroll
  for (int j = 0; j < kMaxPath; ++j)
    if (j < n) buf[j] = *reinterpret_cast<const V*>(at + src[j] * row_bytes);
#pragma unroll
  for (int j = 0; j < kMaxPath; ++j)
    if (j < n) *reinterpret_cast<V*>(at + dst[j] * row_bytes) = buf[j];
}

__global__ void __launch_bounds__(kCompactThreads) compact_q4_kernel(const CompactParams p) {
  __shared__ long long src_s[kMaxPath], dst_s[kMaxPath];  // rows of kv-head 0
  __shared__ int n_moves;
  const int layer = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int L = p.kv_len[b];
  bool bad = false;
  int a = 0;
  if (tid < 32) {
    a = p.accept_len[b];
    const int src = tid < p.H1 ? p.accept_path[b * p.H1 + tid] : 0;
    a = a < 0 ? 0 : (a > p.H1 - 1 ? p.H1 - 1 : a);
    long long from = 0, to = 0;
    if (tid <= a) {
      bad = L < 0 || src < tid || (long long)L + src >= p.g.max_pos();
      if (!bad) {
        int page, slot;
        bad = !find_place(p.g, b, L + src, page, slot);
        from = q4_row(p.g, p.Hkv, 0, page, slot);
        bad = !find_place(p.g, b, L + tid, page, slot) || bad;
        to = q4_row(p.g, p.Hkv, 0, page, slot);
      }
    }
    const unsigned moves = __ballot_sync(0xffffffffu, tid <= a && from != to);
    if (tid <= a && from != to) {
      const int at = __popc(moves & ((1u << tid) - 1u));
      src_s[at] = from;
      dst_s[at] = to;
    }
    if (tid == 0) n_moves = __popc(moves);
  }
  const int any_bad = __syncthreads_or(bad ? 1 : 0);
  if (tid == 0) {
    if (any_bad) report(p.st, CAST_ERR_BAD_PAGE, b);
    // every CTA of the sequence has read kv_len[b] once all have taken the ticket: the last one publishes the new length
    const int t = atomicAdd(&p.ticket[b], 1);
    if (t == (int)(gridDim.x * gridDim.y) - 1) {
      p.ticket[b] = 0;
      if (!any_bad) p.kv_len[b] = L + a + 1;
    }
  }
  const int chunks = p.D / 32, per_head = chunks + 1;  // 16-byte pieces of a row's codes, and its pair
  const int i = blockIdx.x * kCompactThreads + tid, n = n_moves;
  if (any_bad || i >= 2 * p.Hkv * per_head) return;
  const int v = i / (p.Hkv * per_head), h = i / per_head % p.Hkv, ch = i % per_head;
  const long long head = (long long)h * (p.g.page_size == 0 ? p.g.seq_capacity : p.g.page_size);
  if (ch < chunks)
    move_column<uint4>(p.base[v] + p.code_stride * layer + head * (p.D / 2) + ch * 16, p.D / 2, src_s, dst_s, n);
  else
    move_column<uint32_t>(p.base[2 + v] + p.range_stride * layer + head * 4, 4, src_s, dst_s, n);
}

}  // namespace

extern "C" cast_status cast_store_kv_q4(cast_ctx* c, const void* k, const void* v, cast_dtype dtype, int B, int n_layers, int rows,
                                        int Hkv, int D, int page_size, const int32_t* page_table, int seq_capacity, int num_pages,
                                        const int32_t* start, const int32_t* n_rows, void* k_codes, void* k_range, void* v_codes,
                                        void* v_range, size_t code_stride_bytes, size_t range_stride_bytes, void* stream) {
  const Paging g = {page_table, page_size, seq_capacity, num_pages};
  return rows_call<true>(c, k, v, dtype, B, n_layers, rows, Hkv, D, g, start, n_rows, k_codes, k_range, v_codes, v_range,
                         code_stride_bytes, range_stride_bytes, stream);
}

extern "C" cast_status cast_load_kv_q4(cast_ctx* c, const void* k_codes, const void* k_range, const void* v_codes,
                                       const void* v_range, size_t code_stride_bytes, size_t range_stride_bytes, cast_dtype dtype,
                                       int B, int n_layers, int rows, int Hkv, int D, int page_size, const int32_t* page_table,
                                       int seq_capacity, int num_pages, const int32_t* start, const int32_t* n_rows, void* k,
                                       void* v, void* stream) {
  const Paging g = {page_table, page_size, seq_capacity, num_pages};
  return rows_call<false>(c, k, v, dtype, B, n_layers, rows, Hkv, D, g, start, n_rows, k_codes, k_range, v_codes, v_range,
                          code_stride_bytes, range_stride_bytes, stream);
}

extern "C" cast_status cast_compact_kv_q4(cast_ctx* c, void* k_codes, void* k_range, void* v_codes, void* v_range,
                                          size_t code_stride_bytes, size_t range_stride_bytes, int B, int n_layers, int Hkv, int D,
                                          int page_size, const int32_t* page_table, int seq_capacity, int num_pages,
                                          const int32_t* accept_path, const int32_t* accept_len, int32_t* kv_len, void* stream) {
  const Paging g = {page_table, page_size, seq_capacity, num_pages};
  if (!accept_path || !accept_len || !kv_len || n_layers < 1) return CAST_ERR_INVALID_ARG;
  const cast_status st = check_q4(c, B, Hkv, D, g, k_codes, k_range, v_codes, v_range, code_stride_bytes, range_stride_bytes);
  if (st != CAST_OK) return st;
  if (n_layers > 65535) return CAST_ERR_CAPACITY;
  c->tree_inputs_fresh = 1;  // kv_len: an attention call that follows reads it after its dependency wait
  CompactParams p;
  p.base[0] = (unsigned char*)k_codes; p.base[1] = (unsigned char*)v_codes;
  p.base[2] = (unsigned char*)k_range; p.base[3] = (unsigned char*)v_range;
  p.code_stride = code_stride_bytes; p.range_stride = range_stride_bytes;
  p.Hkv = Hkv; p.D = D; p.H1 = c->cfg.max_depth + 1; p.g = g;
  p.accept_path = accept_path; p.accept_len = accept_len; p.kv_len = kv_len; p.ticket = c->compact_ticket; p.st = c->state;
  const int cols = 2 * Hkv * (D / 32 + 1);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((cols + kCompactThreads - 1) / kCompactThreads, n_layers, B);
  cfg.blockDim = dim3(kCompactThreads, 1, 1);
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // launched while the walk finishes; waits for it
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, compact_q4_kernel, p) != cudaSuccess) {
    cudaGetLastError();
    return CAST_ERR_CUDA;
  }
  return CAST_OK;
}
