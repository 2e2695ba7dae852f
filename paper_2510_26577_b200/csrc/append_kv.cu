// cast_append_kv: new rows of queries, keys and values from a projection's output to where the attention reads them, with the norm
// of queries and keys per head and the rotation by their positions on the way.
//
// Formulas: x' = x / sqrt(mean(x^2) + eps) * w over the D dims of a head (fp32), then for every pair (a, b) of rotating dims
// (a, b) -> magnitude (a cos - b sin, b cos + a sin) with the angle position * inv_freq[i]; rounded once, on the way out. The angle is
// formed in turns and in fp64 and only its fraction becomes fp32: in fp32 a position of 100 000 leaves 0.006 of a radian.
//
// One pass: a row is read once and written once. A CTA takes one or four rows; its threads form the rows' cosines and sines once for all
// heads (shared memory), then every group of D * sizeof / 16 lanes takes a head at a time, 16 bytes a lane, eight heads in flight per
// warp of bf16 rows of 128 dims. The partner of a dim (half a rotation away in the halves layout) comes through shared memory, so any even number of rotating
// dims goes one way. The live rows are enumerated on the device: sequences without rows cost nothing.
#include "kv_q4.h"

using namespace cast;

namespace {

constexpr int kThreadsA = 256;
constexpr int kMaxRows = 4;  // rows per CTA at most
constexpr int kMaxPairs = 64;

struct AppendParams {
  const unsigned char *q, *k, *v;
  size_t q_stride, k_stride, v_stride;  // bytes from a row to the next
  unsigned char *q_out, *k_cache, *v_cache;
  int B, rows, Hq, Hkv, rb;             // rb: rows per CTA
  const int32_t *row_start, *first_row, *n_rows, *depth, *position, *start;
  const double* inv_freq;
  int rot_dim, interleaved;
  float magnitude, eps;
  const float *q_weight, *k_weight;
  Paging g;
  DevState* st;
};

// Sixteen bytes of a row as fp32 and back (rounded to nearest even).
template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& a, float (&x)[4]) { Vec<float>::unpack(a, x); }
  static __device__ __forceinline__ uint4 pack(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <> struct Piece<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& a, float (&x)[8]) { Vec<__nv_bfloat16>::unpack(a, x); }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreadsA) append_kernel(const AppendParams p) {
  constexpr int CH = Piece<T>::N, LPH = D / CH, HPW = 32 / LPH;  // dims per lane, lanes per head, heads per warp at a time
  constexpr int kGroups = kThreadsA / LPH, UN = 4;
  constexpr int KB = CAST_MAX_BATCH / 32;
  __shared__ float2 cs[kMaxRows][kMaxPairs];
  __shared__ long long place_s[kMaxRows];                          // row of the cache, -1: none
  __shared__ alignas(16) float turn_s[kThreadsA / 32][HPW * D];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int group = tid / LPH, lig = tid % LPH;                    // lane in its group
  const int heads = (p.q ? p.Hq : 0) + (p.k ? 2 * p.Hkv : 0), q_heads = p.q ? p.Hq : 0;
  const long long all_rows = p.row_start ? p.rows : (long long)p.B * p.rows;

  // live rows of the sequences: lane b % 32 holds sequence b's
  int cnt[KB], first[KB], off[KB], before[KB];
#pragma unroll
  for (int j = 0; j < KB; ++j) {
    const int b = j * 32 + lane;
    const bool in = b < p.B;
    cnt[j] = in ? p.n_rows[b] : 0;
    first[j] = in && p.first_row ? p.first_row[b] : 0;
    off[j] = !in ? 0 : p.row_start ? p.row_start[b] : b * p.rows;
  }
  int live = 0;
#pragma unroll
  for (int j = 0; j < KB; ++j) {
    int n = min(max(cnt[j], 0), p.rows);
    if (p.row_start && (off[j] < 0 || (long long)off[j] + n > all_rows)) {
      if (n > 0 && blockIdx.x == 0 && warp == 0) report(p.st, CAST_ERR_BAD_TREE, j * 32 + lane);
      n = 0;
    }
    first[j] = min(max(first[j], 0), n);
    cnt[j] = n - first[j];
    int x = cnt[j];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    before[j] = live + x - cnt[j];
    live += __shfl_sync(0xffffffffu, x, 31);
  }
  // row i of the live ones: its sequence and token (the whole warp calls)
  auto find = [&](int i, int& b, int& t, int& row) {
    b = t = row = 0;
#pragma unroll
    for (int j = 0; j < KB; ++j) {
      const unsigned hit = __ballot_sync(0xffffffffu, i >= before[j] && i - before[j] < cnt[j]);
      if (hit) {
        const int l = __ffs(hit) - 1;
        b = j * 32 + l;
        t = i - __shfl_sync(0xffffffffu, before[j], l) + __shfl_sync(0xffffffffu, first[j], l);
        row = __shfl_sync(0xffffffffu, off[j], l) + t;
      }
    }
  };

  const int half = p.rot_dim / 2, d0 = lig * CH;
  const long long max_pos = p.g.max_pos();
  for (int i0 = (int)blockIdx.x * p.rb; i0 < live; i0 += (int)gridDim.x * p.rb) {
    const int here = min(p.rb, live - i0);
    int b[kMaxRows], t[kMaxRows], row[kMaxRows];
#pragma unroll
    for (int r = 0; r < kMaxRows; ++r) {
      b[r] = t[r] = row[r] = 0;
      if (r < here) find(i0 + r, b[r], t[r], row[r]);
    }
    auto pick = [&](const int (&x)[kMaxRows], int r) { return r == 0 ? x[0] : r == 1 ? x[1] : r == 2 ? x[2] : x[3]; };
    // (head, row) pairs, a group of lanes each: the first loads go out before the angles are formed
    const int units = here * heads;
    auto source = [&](int u) {
      const int r = u / heads, h = u - r * heads;
      const size_t at = (size_t)pick(row, r);
      const unsigned char* base = h < q_heads ? p.q + at * p.q_stride + (size_t)h * (D * sizeof(T))
                                  : h < q_heads + p.Hkv ? p.k + at * p.k_stride + (size_t)(h - q_heads) * (D * sizeof(T))
                                                        : p.v + at * p.v_stride + (size_t)(h - q_heads - p.Hkv) * (D * sizeof(T));
      return *reinterpret_cast<const uint4*>(base + lig * 16);
    };
    uint4 x[UN];
#pragma unroll
    for (int k = 0; k < UN; ++k) x[k] = group + k * kGroups < units ? source(group + k * kGroups) : make_uint4(0u, 0u, 0u, 0u);
    for (int a = tid; a < here * half; a += kThreadsA) {
      const int r = a / half, i = a - r * half, bb = pick(b, r);
      const long long pos = (long long)(p.position ? p.position[bb] : p.start ? p.start[bb] : 0) + (p.depth ? p.depth[pick(row, r)] : pick(t, r));
      const double turns = (double)pos * (p.inv_freq[i] * 0.15915494309189533577);
      float s, c;
      sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
      cs[r][i] = make_float2(c * p.magnitude, s * p.magnitude);
    }
    if (p.k && tid >= kThreadsA - kMaxRows) {
      const int r = tid - (kThreadsA - kMaxRows);
      if (r < here) {
        const int bb = pick(b, r);
        const long long pos = (long long)(p.start ? p.start[bb] : 0) + pick(t, r);
        int page = 0, slot = 0;
        const bool ok = pos >= 0 && pos < max_pos && find_place(p.g, bb, (int)pos, page, slot);
        if (!ok) report(p.st, CAST_ERR_BAD_PAGE, bb);
        place_s[r] = ok ? (long long)page * (p.g.page_size == 0 ? p.g.seq_capacity : p.g.page_size) + slot : -1;
      }
    }
    __syncthreads();
    for (int u0 = group; __any_sync(0xffffffffu, u0 < units); u0 += UN * kGroups) {
#pragma unroll
      for (int k = 0; k < UN; ++k) {
        const int u = u0 + k * kGroups;
        const bool on = u < units;
        const int r = on ? u / heads : 0, h = on ? u - r * heads : 0;
        const bool is_q = h < q_heads, is_v = h >= q_heads + p.Hkv;
        uint4 y = x[k];
        if (u + UN * kGroups < units) x[k] = source(u + UN * kGroups);
        const bool rotate = !is_v && half > 0;
        const float* w = is_q ? p.q_weight : is_v ? nullptr : p.k_weight;
        if (__any_sync(0xffffffffu, on && (rotate || w != nullptr))) {
          float f[CH];
          Piece<T>::unpack(y, f);
          float sq = 0.f;
#pragma unroll
          for (int e = 0; e < CH; ++e) sq = fmaf(f[e], f[e], sq);
#pragma unroll
          for (int o = LPH / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
          if (w != nullptr) {
            const float inv = rsqrtf(sq * (1.f / D) + p.eps);
#pragma unroll
            for (int e = 0; e < CH; e += 4) {
              const float4 w4 = __ldg(reinterpret_cast<const float4*>(w + d0 + e));
              f[e] *= inv * w4.x; f[e + 1] *= inv * w4.y; f[e + 2] *= inv * w4.z; f[e + 3] *= inv * w4.w;
            }
          }
          if (p.interleaved) {
            if (rotate && d0 < p.rot_dim) {
#pragma unroll
              for (int e = 0; e < CH; e += 2) {
                if (d0 + e < p.rot_dim) {
                  const float2 a = cs[r][(d0 + e) >> 1];
                  const float lo = f[e], hi = f[e + 1];
                  f[e] = lo * a.x - hi * a.y;
                  f[e + 1] = hi * a.x + lo * a.y;
                }
              }
            }
          } else if (half > 0) {
            // dim e of lane l lies at [e / 4][l][e % 4]: 16-byte stores without bank conflicts
            float* mine = turn_s[warp] + (lane / LPH) * D;
#pragma unroll
            for (int e = 0; e < CH; e += 4)
              *reinterpret_cast<float4*>(mine + (e / 4) * (LPH * 4) + lig * 4) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
            __syncwarp();
            if (rotate && d0 < p.rot_dim) {
#pragma unroll
              for (int e = 0; e < CH; ++e) {
                const int d = d0 + e;
                if (d < p.rot_dim) {
                  const bool low = d < half;
                  const int o = low ? d + half : d - half;
                  const float other = mine[(o % CH / 4) * (LPH * 4) + (o / CH) * 4 + o % 4];
                  const float2 a = cs[r][low ? d : o];
                  f[e] = f[e] * a.x + (low ? -other : other) * a.y;
                }
              }
            }
            __syncwarp();
          }
          if (rotate || w != nullptr) y = Piece<T>::pack(f);  // (values stay as they are, bit by bit)
        }
        if (on) {
          if (is_q) {
            *reinterpret_cast<uint4*>(p.q_out + ((size_t)pick(row, r) * p.Hq + h) * (D * sizeof(T)) + lig * 16) = y;
          } else if (place_s[r] >= 0) {
            unsigned char* cache = is_v ? p.v_cache : p.k_cache;
            const int kh = h - q_heads - (is_v ? p.Hkv : 0);
            *reinterpret_cast<uint4*>(cache + ((size_t)place_s[r] * p.Hkv + kh) * (D * sizeof(T)) + lig * 16) = y;
          }
        }
      }
    }
    __syncthreads();
  }
}

template <typename T, int D>
cast_status launch_append(const cast_ctx* c, AppendParams& p, cudaStream_t s) {
  const long long rows = p.row_start ? p.rows : (long long)p.B * p.rows;
  // Four rows per CTA share its start, one keeps a small call's chain short: four from the count on that gives every SM two CTAs.
  p.rb = rows >= 8ll * c->num_sms ? kMaxRows : 1;
  const long long want = (rows + p.rb - 1) / p.rb, most = 8ll * c->num_sms;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(want < most ? want : most), 1, 1);
  cfg.blockDim = dim3(kThreadsA, 1, 1);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, append_kernel<T, D>, p) != cudaSuccess) {
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
  if (all & 15) return CAST_ERR_SHAPE;
  AppendParams p;
  p.g = {page_table, page_size, seq_capacity, num_pages};
  // (the count of live rows, with a grid's step behind it, is 32-bit)
  if (B > c->cfg.max_batch || (long long)B * rows > kMaxPositions || (k && p.g.max_pos() > kMaxPositions) ||
      (long long)Hq + 2ll * Hkv > 65536)
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
