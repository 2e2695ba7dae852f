// cast_store_kv_q4, cast_load_kv_q4, cast_compact_kv_q4: rows into the 4-bit cache, out of it, and to the front of the tree
// region after acceptance.
// Store and load of 4 x 4097 rows, 2 layers of 8 heads of 128 in bf16: 64 us for both (40 to move the bytes); the store alone 38, its issue
// slots 72 % busy with the quantiser. 60 rows of one sequence, both ways: 6.5 us, two launches. The compaction of 32 layers: one sequence
// 11.5 us, the chain length - path - pages - rows - rows; 64 sequences 28.5 (9 for the bytes: rows of 64 bytes and pairs of 4 at scattered places).
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
  FastPaging fg;
  uint32_t head_mul;  // row of the call / Hkv = row * head_mul >> head_shift
  int head_shift;
  const int32_t* start;
  const int32_t* n_rows;
  DevState* st;
};

// Sixteen values as they come, their least and largest (NaN if one is NaN), and the values one by one in fp32.
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
template <typename T>
struct Raw;
template <>
struct Raw<float> {
  float x[kLane];
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 a = __ldcs(reinterpret_cast<const float4*>(p) + i);
      x[4 * i] = a.x; x[4 * i + 1] = a.y; x[4 * i + 2] = a.z; x[4 * i + 3] = a.w;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < kLane; ++e) x[e] = 0.f;
  }
  __device__ __forceinline__ float get(int e) const { return x[e]; }
  __device__ __forceinline__ void range(float& lo, float& hi) const {
    lo = hi = x[0];
#pragma unroll
    for (int e = 1; e < kLane; ++e) {
      lo = min_nan(lo, x[e]);
      hi = max_nan(hi, x[e]);
    }
  }
};
template <>
struct Raw<__nv_bfloat16> {
  uint32_t w[kLane / 2];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p) + i);
      w[4 * i] = a.x; w[4 * i + 1] = a.y; w[4 * i + 2] = a.z; w[4 * i + 3] = a.w;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < kLane / 2; ++e) w[e] = 0u;
  }
  __device__ __forceinline__ float get(int e) const { return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16); }
  __device__ __forceinline__ void range(float& lo, float& hi) const {  // two at a time
    uint32_t a = w[0], b = w[0];
#pragma unroll
    for (int e = 1; e < kLane / 2; ++e) {
      asm("min.NaN.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(w[e]));
      asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(b) : "r"(w[e]));
    }
    lo = min_nan(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u));
    hi = max_nan(__uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u));
  }
};
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

// The row's codes and its pair, from the D / 16 threads that hold it. The code is the quotient of a division, rounded to nearest
// even, without dividing: q = d r with the rounded reciprocal r, corrected once by its exact remainder, q + (d - q step) r, is within
// 2^-46 of the quotient before its last rounding, exact at a tie; and no quotient of a difference and a bf16 step lies nearer than
// 2^-32 to the place where rounding to fp32 would make a tie of it. Reciprocals out of range are divided, and rows whose largest
// value is further from the rounded low than fp32 reaches (hi - lo in range, low below lo): a difference of inf has no remainder.
template <int LPR, typename R>
__device__ __forceinline__ uint2 quantise(const R& x, uint32_t& range) {
  float lo, hi;
  x.range(lo, hi);
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) {
    lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const float span = hi - lo;
  const __nv_bfloat16 step_h = __float2bfloat16_rn(__fdiv_rn(span, 15.f)), low_h = __float2bfloat16_rn(lo);
  if (!(span < INFINITY) || !(fabsf(__bfloat162float(low_h)) < INFINITY)) {  // (NaN among the values: span is NaN; infinities: so, or inf)
    range = 0x7fc07fc0u;
    return make_uint2(0u, 0u);
  }
  range = (uint32_t)__bfloat16_as_ushort(step_h) | ((uint32_t)__bfloat16_as_ushort(low_h) << 16);
  const float step = __bfloat162float(step_h), low = __bfloat162float(low_h);
  if (step == 0.f) return make_uint2(0u, 0u);
  const float inv = __fdiv_rn(1.f, step);
  constexpr float kMagic = 12582912.f;  // 1.5 * 2^23: adding it leaves the nearest integer, ties to even, in the lowest bits
  uint32_t w[2] = {0u, 0u};
  if (!(inv < 1e30f) || !(__fsub_rn(hi, low) < INFINITY)) {
#pragma unroll 1
    for (int e = 0; e < kLane; ++e) {
      float x0 = 0.f;
#pragma unroll
      for (int k = 0; k < kLane; ++k) x0 = k == e ? x.get(k) : x0;
      const float t = rintf(__fdiv_rn(__fsub_rn(x0, low), step));
      const uint32_t c = (uint32_t)fminf(fmaxf(t, 0.f), 15.f) << (4 * (e & 7));
      if (e < 8) w[0] |= c;
      else w[1] |= c;
    }
    return make_uint2(w[0], w[1]);
  }
#pragma unroll
  for (int e = 0; e < kLane; ++e) {
    const float d = __fsub_rn(x.get(e), low), q = __fmul_rn(d, inv), t = fmaf(fmaf(-q, step, d), inv, q);
    w[e / 8] += __float_as_uint(__fadd_rn(fminf(fmaxf(t, 0.f), 15.f), kMagic)) << (4 * (e % 8));
  }
  constexpr uint32_t kBits = 0x4b400000u;  // the magic number's own bits, eight times shifted and added
  constexpr uint32_t kOwn = kBits + (kBits << 4) + (kBits << 8) + (kBits << 12) + (kBits << 16) + (kBits << 20) + (kBits << 24) + (kBits << 28);
  return make_uint2(w[0] - kOwn, w[1] - kOwn);
}

// D / 16 threads per row, K and V of it side by side. kStore: into the cache, else out of it.
template <typename T, int D, bool kStore>
__global__ void __launch_bounds__(kThreads) q4_rows_kernel(const RowsParams p) {
  constexpr int LPR = D / kLane;
  const int b = blockIdx.y, layer = blockIdx.z;
  const uint32_t i = blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
  const int part = threadIdx.x % LPR;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int n = min(p.n_rows[b], p.rows);
  const int t = (int)(((uint64_t)i * p.head_mul) >> p.head_shift), h = (int)i - t * p.Hkv;
  const unsigned here = __ballot_sync(0xffffffffu, t < n);
  if (here == 0u) return;  // (a row's threads are in one warp: whole warps leave, the others go on together)
  const bool live = t < n;
  long long pos = live ? (long long)(p.start ? p.start[b] : 0) + t : 0;
  bool ok = live && pos >= 0 && pos < p.g.max_pos();
  uint32_t page = b, slot = (uint32_t)pos, slots = p.fg.seq_capacity;
  if (p.fg.page_size > 0) {
    slots = p.fg.page_size;
    const uint32_t e = ok ? (uint32_t)(((uint64_t)slot * p.fg.mul) >> p.fg.shift) : 0u;
    page = (uint32_t)p.fg.table[(size_t)b * p.fg.seq_capacity + e];
    slot -= e * slots;
    ok = ok && page < (uint32_t)p.fg.num_pages;
  }
  if (live && !ok && part == 0) report(p.st, CAST_ERR_BAD_PAGE, b);
  const size_t row = ok ? (page * (uint32_t)p.Hkv + h) * slots + slot : 0u;
  const size_t at = ((((size_t)layer * p.B + b) * p.rows + (live ? t : 0)) * p.Hkv + h) * D + part * kLane;
  unsigned char* const kc = p.kc + p.code_stride * layer + row * (D / 2) + part * 8;
  unsigned char* const vc = p.vc + p.code_stride * layer + row * (D / 2) + part * 8;
  uint32_t* const kr = reinterpret_cast<uint32_t*>(reinterpret_cast<unsigned char*>(p.kr) + p.range_stride * layer) + row;
  uint32_t* const vr = reinterpret_cast<uint32_t*>(reinterpret_cast<unsigned char*>(p.vr) + p.range_stride * layer) + row;
  if (kStore) {
    Raw<T> xk, xv;
    xk.clear();
    xv.clear();
    if (live) {
      xk.load(reinterpret_cast<const T*>(p.k) + at);
      xv.load(reinterpret_cast<const T*>(p.v) + at);
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
      for (int e = 0; e < kLane; ++e) {
        // 16 + code, by its bits (the conversion instruction has a quarter of the rate); the difference is exact
        const uint32_t word = e < 8 ? c[w].x : c[w].y, sh = e % 8 < 5 ? word << (19 - 4 * (e % 8)) : word >> (4 * (e % 8) - 19);
        x[e] = fmaf(step, __uint_as_float(and_or(sh, 0x00780000u, 0x41800000u)) - 16.f, low);
      }
      store16(reinterpret_cast<T*>(const_cast<void*>(w ? p.v : p.k)) + at, x);
    }
  }
}

template <bool kStore>
cast_status launch_rows(cast_ctx* c, RowsParams& p, cast_dtype dtype, int n_layers, int D, cudaStream_t s) {
  const long long per = kThreads / (D / kLane), blocks = ((long long)p.rows * p.Hkv + per - 1) / per;
  if ((long long)p.rows * p.Hkv > 0x7fffff00ll || n_layers > 65535 || !fast_paging(p.g, p.B, p.Hkv, &p.fg)) return CAST_ERR_CAPACITY;
  int lg = 0;
  while ((1ll << lg) < p.Hkv) ++lg;
  p.head_shift = 31 + lg;  // (as for the pages: exact below 2^31)
  p.head_mul = (uint32_t)(((1ull << p.head_shift) + p.Hkv - 1) / p.Hkv);
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
  if (!kStore) c->tree_inputs_fresh = 1;  // (k and v may be a 16-bit cache: an attention call that follows reads no row early)
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
