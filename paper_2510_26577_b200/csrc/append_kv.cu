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

// Where a rotating dim's partner lies: beside it; half a rotation away and that is a whole number of lanes; half a rotation away anywhere.
enum { kBeside, kLanes, kAnywhere };

template <typename T, int D, int MODE>
__global__ void __launch_bounds__(kThreadsA, 3) append_kernel(const __grid_constant__ AppendParams p) {
  constexpr int CH = Piece<T>::N, LPH = D / CH, HPW = 32 / LPH;  // dims per lane, lanes per head, heads per piece
  constexpr int kPiece = 512, UN = 2;                            // bytes a warp takes at a time; pieces in flight
  __shared__ float2 cs[kThreadsA / 32][kMaxPairs];
  __shared__ float w_s[2][D];
  __shared__ int before_s[CAST_MAX_BATCH], first_s[CAST_MAX_BATCH], off_s[CAST_MAX_BATCH], live_s;
  __shared__ alignas(16) unsigned char turn_s[MODE == kAnywhere ? kThreadsA / 32 : 1][kPiece];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int d0 = lane % LPH * CH, half = p.rot_dim / 2;            // first dim of the lane
  const int nq = p.q ? (p.Hq + HPW - 1) / HPW : 0, nk = p.k ? (p.Hkv + HPW - 1) / HPW : 0, pieces = nq + 2 * nk;
  const uint32_t q_bytes = (uint32_t)p.Hq * (uint32_t)(D * sizeof(T)), k_bytes = (uint32_t)p.Hkv * (uint32_t)(D * sizeof(T));
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

  // The live rows in front of every sequence, its first token, and where that token's row lies. (In shared memory: held in registers
  // they took a third of a thread's, and it is warps that hide this kernel's latency.)
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

  const int parts = 1 << p.parts_log2;
  for (int u = (int)blockIdx.x * (kThreadsA / 32) + warp; u >> p.parts_log2 < live; u += (int)gridDim.x * (kThreadsA / 32)) {
    const int i = u >> p.parts_log2;
    int b = 0;  // the i-th live row: the last sequence with i rows or fewer in front of it
    for (int b0 = 0; b0 < p.B; b0 += 32) {
      const unsigned hit = __ballot_sync(0xffffffffu, b0 + lane < p.B && before_s[b0 + lane] <= i);
      if (hit) b = b0 + 31 - __clz(hit);
    }
    const int t = i - before_s[b] + first_s[b], row = off_s[b] + t;
    // A piece is 512 bytes of one tensor's row, sixteen a lane.
    const unsigned char *q_row = p.q + (size_t)row * p.q_stride, *k_row = p.k + (size_t)row * p.k_stride, *v_row = p.v + (size_t)row * p.v_stride;
    auto load = [&](int j) {
      const unsigned char* base = j < nq ? q_row : j < nq + nk ? k_row : v_row;
      const uint32_t o = (uint32_t)(j < nq ? j : j < nq + nk ? j - nq : j - nq - nk) * kPiece + lane * 16;
      return o < (j < nq ? q_bytes : k_bytes) ? __ldcs(reinterpret_cast<const uint4*>(base + o)) : make_uint4(0u, 0u, 0u, 0u);
    };
    uint4 x[UN];
    int j_load = u & (parts - 1), j_now = j_load;
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      x[k] = j_load < pieces ? load(j_load) : make_uint4(0u, 0u, 0u, 0u);
      j_load += parts;
    }
    // the row's place in the cache
    long long place = -1;
    const int begin = p.start ? p.start[b] : 0;
    if (p.k) {
      const long long pos = (long long)begin + t;
      int page = 0, slot = 0;
      const bool ok = pos >= 0 && pos < max_pos && find_place(p.g, b, (int)pos, page, slot);
      if (ok) place = (long long)page * (p.g.page_size == 0 ? p.g.seq_capacity : p.g.page_size) + slot;
      else if (lane == 0) report(p.st, CAST_ERR_BAD_PAGE, b);
    }
    // its cosines and sines, a pair or two a lane
    if (half > 0) {
      const long long pos = (long long)(p.position ? p.position[b] : begin) + (p.depth ? p.depth[row] : t);
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
    float ca[CH], cb[CH];
    bool norm = false, changes = false;
    int sec = -1;
    auto section = [&](int now) {
      sec = now;
      norm = now == 0 ? p.q_weight != nullptr : now == 1 && p.k_weight != nullptr;
      changes = norm || (now < 2 && half > 0);
      if (!changes) return;
#pragma unroll
      for (int e = 0; e < CH; ++e) {
        const int d = d0 + e;
        const bool turns = d < p.rot_dim, low = MODE == kBeside ? (e & 1) == 0 : d < half;
        const int o = !turns ? d : MODE == kBeside ? d ^ 1 : low ? d + half : d - half;
        const float2 a = turns ? cs[warp][MODE == kBeside ? d >> 1 : low ? d : o] : make_float2(1.f, 0.f);
        ca[e] = a.x * w_s[now][d];
        cb[e] = (low || !turns ? -a.y : a.y) * w_s[now][o];  // (-0 leaves a zero's sign alone)
      }
    };

    auto turn = [&](uint4& y) {
      float f[CH], g[CH];
      Piece<T>::unpack(y, f);
      if (MODE == kBeside) {
#pragma unroll
        for (int e = 0; e < CH; ++e) g[e] = d0 + e < p.rot_dim ? f[e ^ 1] : 0.f;
      } else if (MODE == kLanes) {
        const int from = (d0 < half ? d0 + half : d0 - half) / CH;
        uint4 z;
        z.x = __shfl_sync(0xffffffffu, y.x, from, LPH); z.y = __shfl_sync(0xffffffffu, y.y, from, LPH);
        z.z = __shfl_sync(0xffffffffu, y.z, from, LPH); z.w = __shfl_sync(0xffffffffu, y.w, from, LPH);
        if (d0 >= p.rot_dim) z = make_uint4(0u, 0u, 0u, 0u);
        Piece<T>::unpack(z, g);
      } else {
        __syncwarp();
        *reinterpret_cast<uint4*>(turn_s[warp] + lane * 16) = y;
        __syncwarp();
        const T* mine = reinterpret_cast<const T*>(turn_s[warp]) + lane / LPH * D;
#pragma unroll
        for (int e = 0; e < CH; ++e) {
          const int d = d0 + e;
          g[e] = d < p.rot_dim ? (float)mine[d < half ? d + half : d - half] : 0.f;
        }
      }
      float inv = 1.f;
      if (norm) {
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < CH; ++e) sq = fmaf(f[e], f[e], sq);
#pragma unroll
        for (int o = LPH / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
        inv = rsqrtf(sq * (1.f / D) + p.eps);
      }
#pragma unroll
      for (int e = 0; e < CH; ++e) f[e] = fmaf(f[e], ca[e], g[e] * cb[e]) * inv;
      y = Piece<T>::pack(f);
    };
    while (j_now < pieces) {
#pragma unroll
      for (int k = 0; k < UN; ++k) {
        if (j_now >= pieces) break;
        uint4 y = x[k];
        if (j_load < pieces) x[k] = load(j_load);
        j_load += parts;
        const int now = (j_now >= nq) + (j_now >= nq + nk);
        if (now != sec) section(now);
        if (changes) turn(y);  // (else the values stay as they are, bit by bit)
        const uint32_t o = (uint32_t)(j_now - (now > 0 ? nq : 0) - (now > 1 ? nk : 0)) * kPiece + lane * 16;
        unsigned char* to = now == 0 ? p.q_out + (size_t)row * q_bytes : (now == 1 ? p.k_cache : p.v_cache) + (size_t)place * k_bytes;
        if (now == 0 ? o < q_bytes : place >= 0 && o < k_bytes) *reinterpret_cast<uint4*>(to + o) = y;
        j_now += parts;
      }
    }
  }
}

template <typename T, int D>
cast_status launch_append(const cast_ctx* c, AppendParams& p, cudaStream_t s) {
  constexpr int CH = Piece<T>::N, HPW = 32 / (D / CH), kWarps = kThreadsA / 32;
  const long long rows = p.row_start ? p.rows : (long long)p.B * p.rows;
  const int pieces = (p.q ? (p.Hq + HPW - 1) / HPW : 0) + (p.k ? 2 * ((p.Hkv + HPW - 1) / HPW) : 0);
  const long long resident = 3ll * c->num_sms * kWarps;
  p.parts_log2 = 0;
  while (p.parts_log2 < 3 && rows << p.parts_log2 < 1 * resident && 2 << p.parts_log2 <= pieces) ++p.parts_log2;
  const long long want = ((rows << p.parts_log2) + kWarps - 1) / kWarps, most = 3ll * c->num_sms;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(want < most ? want : most), 1, 1);
  cfg.blockDim = dim3(kThreadsA, 1, 1);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const int half = p.rot_dim / 2;
  const cudaError_t e = p.interleaved     ? cudaLaunchKernelEx(&cfg, append_kernel<T, D, kBeside>, p)
                        : half % CH == 0 ? cudaLaunchKernelEx(&cfg, append_kernel<T, D, kLanes>, p)
                                         : cudaLaunchKernelEx(&cfg, append_kernel<T, D, kAnywhere>, p);
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
