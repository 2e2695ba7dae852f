// cast_append_kv: new rows of queries, keys and values from a projection's output to where the attention reads them, with the norm
// of queries and keys per head and the rotation by their positions on the way.
//
// Formulas: x' = x / sqrt(mean(x^2) + eps) * w over the D dims of a head (fp32), then for every pair (a, b) of rotating dims
// (a, b) -> magnitude (a cos - b sin, b cos + a sin) with the angle position * inv_freq[i]; rounded once, on the way out. The angle is
// formed in turns and in fp64 and only its fraction becomes fp32: in fp32 a position of 100 000 leaves 0.006 of a radian.
//
// One pass: a row is read once and written once, so memory bounds a long call: 10 400 rows of 32/8 heads of 128 dims in bf16 (255 MB in
// and out) take 53 us, 4.8 TB/s, 73 % of a copy's rate (the loop without its arithmetic: the same). What comes next is instructions, 74 % of the issue slots; hence:
// - A warp takes a row, or a part of one where rows are few, 512 bytes of one tensor at a time. It needs no other warp.
// - Loads run ahead by cp.async into a ring of the warp's own, over the ends of rows, so that the loop need not be unrolled over
//   registers in flight (with it: 61 us, and more registers in flight were slower, at 65 to 86, for they cost warps).
// - A lane has two chunks of eight bytes, half a rotation apart in the halves layout, so that a dim meets its partner in the lane; cosine, sine
//   and weight become one factor each for a dim and its partner, in registers, once per row and tensor (formed per head: 124 us; with
//   the head and row found by division: 149). A rotation that is no whole number of chunks reads the partner from the ring
//   (36 of 128 dims, the same rows: 80 us). In fp32 the same rows take 96 us, 87 % of a copy's rate.
// A small call is a chain of two reads of memory behind its launch: 7 us.
// The live rows are enumerated on the device: sequences without rows cost nothing.
#include "kv_q4.h"

using namespace cast;

namespace {

constexpr int kThreadsA = 256;
constexpr int kMaxPairs = 64;

struct AppendParams {
  const unsigned char *q, *k, *v;
  size_t q_stride, k_stride, v_stride;  // bytes from a row to the next
  unsigned char *q_out, *k_cache, *v_cache;
  int B, rows, Hq, Hkv, parts_log2;     // warps per row
  const int32_t *row_start, *first_row, *n_rows, *depth, *position, *start;
  const double* inv_freq;
  int rot_dim, interleaved;
  float magnitude, eps;
  const float *q_weight, *k_weight;
  Paging g;
  DevState* st;
};

// Two fp32 in a register pair, for the packed forms of multiply and fused multiply-add.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{.reg .b64 x, y, z; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mul.rn.f32x2 z, x, y; mov.b64 {%0, %1}, z;}" : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{.reg .b64 x, y, z; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%6, %7}; fma.rn.f32x2 z, x, y, z; mov.b64 {%0, %1}, z;}" : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}

// Eight bytes of a row as pairs of fp32 and back (rounded to nearest even).
template <typename T> struct Chunk;
template <> struct Chunk<float> {
  static constexpr int N = 1;  // pairs
  static __device__ __forceinline__ void unpack(const uint2& a, float2* x) { x[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y)); }
  static __device__ __forceinline__ uint2 pack(const float2* x) { return make_uint2(__float_as_uint(x[0].x), __float_as_uint(x[0].y)); }
};
template <> struct Chunk<__nv_bfloat16> {
  static constexpr int N = 2;
  static __device__ __forceinline__ void unpack(const uint2& a, float2* x) {
    x[0] = make_float2(__uint_as_float(a.x << 16), __uint_as_float(a.x & 0xffff0000u));
    x[1] = make_float2(__uint_as_float(a.y << 16), __uint_as_float(a.y & 0xffff0000u));
  }
  static __device__ __forceinline__ uint2 pack(const float2* x) {
    const __nv_bfloat162 a = __float22bfloat162_rn(x[0]), b = __float22bfloat162_rn(x[1]);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
};

// Where a rotating dim's partner lies: in the same pair of the lane's first or second chunk; at the same place of its other chunk; anywhere.
enum { kBeside, kAcross, kAnywhere };

template <typename T, int D, int MODE>
__global__ void __launch_bounds__(kThreadsA, MODE == kAnywhere ? 2 : 3) append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int N = Chunk<T>::N, C = 2 * N;          // pairs and dims of a chunk of eight bytes; a lane has two
  constexpr int LPH = D / (2 * C), HPW = 32 / LPH;   // lanes per head, heads per piece
  constexpr int kPiece = 512, UN = 4;                // bytes a warp takes at a time; pieces in its ring
  __shared__ float2 cs[kThreadsA / 32][kMaxPairs];
  __shared__ float w_s[2][D];
  __shared__ int before_s[CAST_MAX_BATCH], first_s[CAST_MAX_BATCH], off_s[CAST_MAX_BATCH], live_s;
  __shared__ int start_s[CAST_MAX_BATCH], position_s[CAST_MAX_BATCH];
  __shared__ alignas(16) unsigned char in_s[kThreadsA / 32][UN][kPiece];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, lig = lane % LPH;
  const int half = p.rot_dim / 2;
  // The lane's chunks. Where halves rotate, the lanes of the rotating dims take a chunk of each half, so that partners meet in a lane.
  const bool across = MODE == kAcross && lig * 2 * C < p.rot_dim;
  const int d0 = across ? lig * C : lig * 2 * C, d1 = across ? half + lig * C : d0 + C;
  const bool rotates = MODE != kAnywhere && half > 0 && lig * 2 * C < p.rot_dim;
  auto dim = [&](int e) { return e < C ? d0 + e : d1 + e - C; };
  const int nq = p.q ? (p.Hq + HPW - 1) / HPW : 0, nk = p.k ? (p.Hkv + HPW - 1) / HPW : 0, pieces = nq + 2 * nk;
  const uint32_t q_bytes = (uint32_t)p.Hq * (uint32_t)(D * sizeof(T)), k_bytes = (uint32_t)p.Hkv * (uint32_t)(D * sizeof(T));
  const uint32_t at0 = (uint32_t)((lane / LPH * D + d0) * sizeof(T)), gap = (uint32_t)((d1 - d0) * sizeof(T));
  const long long all_rows = p.row_start ? p.rows : (long long)p.B * p.rows;
  const long long max_pos = p.g.max_pos();

  // what no row changes: frequencies in turns, weights
  double freq[kMaxPairs / 32];
#pragma unroll
  for (int j = 0; j < kMaxPairs / 32; ++j) freq[j] = j * 32 + lane < half ? p.inv_freq[j * 32 + lane] * 0.15915494309189533577 : 0.;
  for (int d = tid; d < 2 * D; d += kThreadsA) {
    const float* w = d < D ? p.q_weight : p.k_weight;
    w_s[d / D][d % D] = w ? w[d % D] : 1.f;
  }

  // The live rows in front of every sequence, its first token, and where that token's row lies. (In shared memory: registers are
  // better spent on warps, which hide this kernel's latency.)
  for (int b = tid; b < p.B; b += kThreadsA) {
    start_s[b] = p.start ? p.start[b] : 0;
    if (p.position) position_s[b] = p.position[b];
  }
  if (warp == 0) {
    int live = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const int b = b0 + lane;
      int n = b < p.B ? min(max(p.n_rows[b], 0), p.rows) : 0;
      const int off = b >= p.B ? 0 : p.row_start ? p.row_start[b] : b * p.rows;
      int first = b < p.B && p.first_row ? p.first_row[b] : 0;
      if (p.row_start && (off < 0 || (long long)off + n > all_rows)) {
        if (n > 0 && blockIdx.x == 0) report(p.st, CAST_ERR_BAD_TREE, b);
        n = 0;
      }
      first = min(max(first, 0), n);
      n -= first;
      int x = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      before_s[b] = live + x - n;
      first_s[b] = first;
      off_s[b] = off;
      live += __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) live_s = live;
  }
  __syncthreads();
  const int live = live_s;

  auto find = [&](int i) {  // the sequence of the i-th live row: the last one with i rows or fewer in front of it
    int b = 0;
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const unsigned hit = __ballot_sync(0xffffffffu, b0 + lane < p.B && before_s[b0 + lane] <= i);
      if (hit) b = b0 + 31 - __clz(hit);
    }
    return b;
  };
  // A piece is 512 bytes of one tensor's row: the rows of q, k and v in that order, a warp's pieces `parts` apart. A cursor walks them:
  // `end` is where its tensor ends, `lim` where the lane's share of it does (the last piece may be a part).
  const int parts = 1 << p.parts_log2, units = (int)gridDim.x * (kThreadsA / 32);
  const int u0 = (int)blockIdx.x * (kThreadsA / 32) + warp, part = warp & (parts - 1);
  const uint32_t stride = (uint32_t)kPiece << p.parts_log2;
  struct Cursor {
    int j, end, lim;
    uint32_t at;
  };
  auto seat = [&](Cursor& c, uint32_t at) {
    const int sec = (c.j >= nq) + (c.j >= nq + nk), from = sec == 0 ? 0 : sec == 1 ? nq : nq + nk;
    const uint32_t bytes = sec == 0 ? q_bytes : k_bytes;
    c.end = sec == 0 ? nq : sec == 1 ? nq + nk : pieces;
    c.at = (uint32_t)(c.j - from) * kPiece + at;
    c.lim = c.j >= pieces ? 0 : c.end - ((uint32_t)(c.end - 1 - from) * kPiece + at < bytes ? 0 : 1);
    return sec;
  };
  // Loads run UN - 1 pieces ahead, over the ends of rows, into shared memory: a warp's own ring.
  int u_load = u0, row_load = -1;
  Cursor in = {0, 0, 0, 0u};
  const unsigned char* from = nullptr;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(&in_s[warp][0][lane * 16]);
  uint32_t slot_load = 0, slot = 0;
  auto load = [&]() {
    if (in.j >= in.end && u_load >> p.parts_log2 < live) {
      if (row_load < 0) {
        const int i = u_load >> p.parts_log2, b = find(i);
        row_load = off_s[b] + first_s[b] + i - before_s[b];
        in.j = part;
      }
      const int sec = seat(in, lane * 16);
      from = sec == 0 ? p.q + (size_t)row_load * p.q_stride : sec == 1 ? p.k + (size_t)row_load * p.k_stride : p.v + (size_t)row_load * p.v_stride;
      from += in.at;
    }
    if (in.j < in.lim) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + slot_load), "l"(from) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
    slot_load = (slot_load + kPiece) % (UN * kPiece);
    in.j += parts;
    from += stride;
    if (in.j >= pieces) {
      in.end = 0;
      in.lim = 0;
      u_load += row_load >= 0 ? units : 0;
      row_load = -1;
    }
  };
#pragma unroll 1
  for (int k = 0; k < UN - 1; ++k) load();
  for (int u = u0; u >> p.parts_log2 < live; u += units) {
    const int i = u >> p.parts_log2, b = find(i), t = i - before_s[b] + first_s[b], row = off_s[b] + t;
    Cursor out = {part, 0, 0, 0u};
    // the row's place in the cache
    long long place = -1;
    const int begin = start_s[b];
    if (p.k) {
      const long long pos = (long long)begin + t;
      int page = 0, slot = 0;
      const bool ok = pos >= 0 && pos < max_pos && find_place(p.g, b, (int)pos, page, slot);
      if (ok) place = (long long)page * (p.g.page_size == 0 ? p.g.seq_capacity : p.g.page_size) + slot;
      else if (lane == 0) report(p.st, CAST_ERR_BAD_PAGE, b);
    }
    // its cosines and sines, a pair or two a lane
    if (half > 0) {
      const long long pos = (long long)(p.position ? position_s[b] : begin) + (p.depth ? p.depth[row] : t);
      __syncwarp();
#pragma unroll
      for (int j = 0; j < kMaxPairs / 32; ++j) {
        const double turns = (double)pos * freq[j];
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        cs[warp][j * 32 + lane] = make_float2(c * p.magnitude, s * p.magnitude);
      }
      __syncwarp();
    }
    // and what they make of the lane's dims, the weights within: out = a x + b partner. A warp's pieces lie in order, so queries'
    // give way to keys' once.
    float2 ca[C], cb[C];
    bool norm = false, changes = false;
    unsigned char* to = nullptr;
    auto enter = [&]() {
      const int sec = seat(out, at0);
      to = sec == 0 ? p.q_out + (size_t)row * q_bytes : (sec == 1 ? p.k_cache : p.v_cache) + (size_t)place * k_bytes;
      to += out.at;
      if (sec > 0 && place < 0) out.lim = 0;
      norm = sec == 0 ? p.q_weight != nullptr : sec == 1 && p.k_weight != nullptr;
      changes = norm || (sec < 2 && half > 0);
      if (!changes) return;
      const float* w = w_s[sec];
#pragma unroll
      for (int e = 0; e < 2 * C; ++e) {
        const int d = dim(e);
        const bool turns = d < p.rot_dim, low = p.interleaved ? (e & 1) == 0 : d < half;
        const int o = !turns ? d : p.interleaved ? d ^ 1 : low ? d + half : d - half;
        const float2 a = turns ? cs[warp][p.interleaved ? d >> 1 : low ? d : o] : make_float2(1.f, 0.f);
        const float x = a.x * w[d], y = (low || !turns ? -a.y : a.y) * w[o];  // (-0 leaves a zero's sign alone)
        if (e & 1) {
          ca[e / 2].y = x; cb[e / 2].y = y;
        } else {
          ca[e / 2].x = x; cb[e / 2].x = y;
        }
      }
    };
#pragma unroll 1
    while (out.j < pieces) {
      load();
      asm volatile("cp.async.wait_group %0;" ::"n"(UN - 1) : "memory");
      __syncwarp();
      const unsigned char* piece = in_s[warp][0] + slot + lane / LPH * (D * sizeof(T));
      uint2 y[2] = {*reinterpret_cast<const uint2*>(piece + d0 * sizeof(T)), *reinterpret_cast<const uint2*>(piece + d1 * sizeof(T))};
      if (out.j >= out.end) enter();
      if (changes) {  // (else the values stay as they are, bit by bit)
        float2 f[C], g[C];
        Chunk<T>::unpack(y[0], f);
        Chunk<T>::unpack(y[1], f + N);
        if (MODE == kAnywhere) {
          const T* head = reinterpret_cast<const T*>(piece);
#pragma unroll
          for (int e = 0; e < 2 * C; ++e) {
            const int d = d0 + e;
            const float o = d < p.rot_dim ? (float)head[p.interleaved ? d ^ 1 : d < half ? d + half : d - half] : 0.f;
            if (e & 1) g[e / 2].y = o; else g[e / 2].x = o;
          }
        }
        float inv = 1.f;
        if (norm) {
          float2 sq = mul2(f[0], f[0]);
#pragma unroll
          for (int e = 1; e < C; ++e) sq = fma2(f[e], f[e], sq);
          float sum = sq.x + sq.y;
#pragma unroll
          for (int o = LPH / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
          inv = rsqrtf(sum * (1.f / D) + p.eps);
        }
#pragma unroll
        for (int e = 0; e < C; ++e) {
          if (MODE == kBeside) g[e] = make_float2(f[e].y, f[e].x);
          if (MODE == kAcross) g[e] = f[e < N ? e + N : e - N];
        }
        if (MODE == kAnywhere || rotates) {
#pragma unroll
          for (int e = 0; e < C; ++e) f[e] = fma2(f[e], ca[e], mul2(g[e], cb[e]));
        } else {
#pragma unroll
          for (int e = 0; e < C; ++e) f[e] = mul2(f[e], ca[e]);
        }
        if (norm) {
#pragma unroll
          for (int e = 0; e < C; ++e) f[e] = mul2(f[e], make_float2(inv, inv));
        }
        y[0] = Chunk<T>::pack(f);
        y[1] = Chunk<T>::pack(f + N);
      }
      if (out.j < out.lim) {
        *reinterpret_cast<uint2*>(to) = y[0];
        *reinterpret_cast<uint2*>(to + gap) = y[1];
      }
      out.j += parts;
      to += stride;
      slot = (slot + kPiece) % (UN * kPiece);
      __syncwarp();  // (the next load takes this slot)
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

template <typename T, int D>
cast_status launch_append(const cast_ctx* c, AppendParams& p, cudaStream_t s) {
  constexpr int C = 2 * Chunk<T>::N, HPW = 32 / (D / (2 * C)), kWarps = kThreadsA / 32;
  const long long rows = p.row_start ? p.rows : (long long)p.B * p.rows;
  const int pieces = (p.q ? (p.Hq + HPW - 1) / HPW : 0) + (p.k ? 2 * ((p.Hkv + HPW - 1) / HPW) : 0);
  // Warps per row: as many as the device has places for (a warp's pieces are a chain, 0.3 us each: 64 rows of 32/8 heads take 9.2 us
  // with two warps a row, 8.2 with four, 7.2 with eight), one from there on (each forms the row's angles for itself).
  const long long most = 3ll * c->num_sms;  // CTAs
  p.parts_log2 = 0;
  while (1 << p.parts_log2 < kWarps && rows << p.parts_log2 < most * kWarps && 2 << p.parts_log2 <= pieces) ++p.parts_log2;
  const long long want = ((rows << p.parts_log2) + kWarps - 1) / kWarps;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(want < most ? want : most), 1, 1);
  cfg.blockDim = dim3(kThreadsA, 1, 1);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  // (a lane's rotating dims have their partners in the lane: chunks of eight bytes are whole)
  const cudaError_t e = p.rot_dim % (2 * C) != 0 ? cudaLaunchKernelEx(&cfg, append_kernel<T, D, kAnywhere>, p)
                        : p.interleaved          ? cudaLaunchKernelEx(&cfg, append_kernel<T, D, kBeside>, p)
                                                 : cudaLaunchKernelEx(&cfg, append_kernel<T, D, kAcross>, p);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return CAST_ERR_CUDA;
  }
  return launch_status();
}

}  // namespace

extern "C" cast_status cast_append_kv(cast_ctx* c, const void* q, size_t q_stride_bytes, const void* k, size_t k_stride_bytes,
                                      const void* v, size_t v_stride_bytes, cast_dtype dtype, int B, int rows, int Hq, int Hkv, int D,
                                      const int32_t* row_start, const int32_t* first_row, const int32_t* n_rows,
                                      const int32_t* depth, const int32_t* position, const double* inv_freq, int rot_dim,
                                      int interleaved, float magnitude, const float* q_weight, const float* k_weight, float eps,
                                      int page_size, const int32_t* page_table, int seq_capacity, int num_pages,
                                      const int32_t* start, void* q_out, void* k_cache, void* v_cache, void* stream) {
  if (!c || B < 1 || rows < 1 || !n_rows || (!q && !k) || (!k != !v) || (q && (!q_out || Hq < 1)) || rot_dim < 0 ||
      (rot_dim > 0 && !inv_freq) || !(eps >= 0.f))
    return CAST_ERR_INVALID_ARG;
  if (k && (!k_cache || !v_cache || Hkv < 1 || page_size < 0 || seq_capacity < 1 || (page_size > 0 && (!page_table || num_pages < 1))))
    return CAST_ERR_INVALID_ARG;
  if (!on_device(c)) return CAST_ERR_INVALID_ARG;
  if (dtype != CAST_F32 && dtype != CAST_BF16) return CAST_ERR_DTYPE;
  const size_t e = dtype == CAST_F32 ? 4 : 2;
  if ((D != 64 && D != 128) || rot_dim > D || rot_dim % 2) return CAST_ERR_SHAPE;
  uintptr_t all = 0;
  if (q) {
    if (q_stride_bytes < (size_t)Hq * D * e) return CAST_ERR_SHAPE;
    all |= (uintptr_t)q | (uintptr_t)q_out | q_stride_bytes | (uintptr_t)q_weight;
  }
  if (k) {
    if (k_stride_bytes < (size_t)Hkv * D * e || v_stride_bytes < (size_t)Hkv * D * e) return CAST_ERR_SHAPE;
    all |= (uintptr_t)k | (uintptr_t)v | k_stride_bytes | v_stride_bytes | (uintptr_t)k_cache | (uintptr_t)v_cache | (uintptr_t)k_weight;
  }
  if (all & 15 || (uintptr_t)inv_freq & 7) return CAST_ERR_SHAPE;
  AppendParams p;
  p.g = {page_table, page_size, seq_capacity, num_pages};
  // (the count of live rows, with a grid's step behind it, is 32-bit)
  if (B > c->cfg.max_batch || (long long)B * rows > kMaxPositions || (k && p.g.max_pos() > kMaxPositions) ||
      (q ? (long long)Hq : 0) + (k ? 2ll * Hkv : 0) > 65536)
    return CAST_ERR_CAPACITY;
  p.q = (const unsigned char*)q; p.k = (const unsigned char*)k; p.v = (const unsigned char*)v;
  p.q_stride = q_stride_bytes; p.k_stride = k_stride_bytes; p.v_stride = v_stride_bytes;
  p.q_out = (unsigned char*)q_out; p.k_cache = (unsigned char*)k_cache; p.v_cache = (unsigned char*)v_cache;
  p.B = B; p.rows = rows; p.Hq = Hq; p.Hkv = Hkv;
  p.row_start = row_start; p.first_row = first_row; p.n_rows = n_rows; p.depth = depth; p.position = position; p.start = start;
  p.inv_freq = inv_freq; p.rot_dim = rot_dim; p.interleaved = interleaved;
  p.magnitude = magnitude == 0.f ? 1.f : magnitude;
  p.eps = eps; p.q_weight = q_weight; p.k_weight = k_weight;
  p.st = c->state;
  cudaStream_t s = (cudaStream_t)stream;
  if (dtype == CAST_F32) return D == 64 ? launch_append<float, 64>(c, p, s) : launch_append<float, 128>(c, p, s);
  return D == 64 ? launch_append<__nv_bfloat16, 64>(c, p, s) : launch_append<__nv_bfloat16, 128>(c, p, s);
}
