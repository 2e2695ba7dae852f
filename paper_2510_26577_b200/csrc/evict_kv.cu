// cast_evict_kv, cast_evict_kv_q4: the positions with the least accumulated attention weight leave the cache.
//
// Two launches. evict_select_kernel, one CTA per (layer, sequence, kv-head), finds the (budget - recent)-th largest weight
// of the positions before the recent ones by a radix selection over the order-preserving integers of the weights (11 + 11 + 10
// bits: three histograms in shared memory), then writes the kept positions in ascending order and moves their weights to the
// front in one pass of block-wide counting. evict_gather_kernel moves the rows: a CTA takes one (layer, sequence, kv-head) of K or V
// and walks the list in order, many rows in flight. A row never moves up, so all sources of a
// group of rows lie at or behind the group's own destinations: its loads come before its stores, and nothing later is lost.
// Bound by memory: the weights once, the moved rows once each way. 32 layers of 4 sequences of 6000 to 8192 cut to 4096, 8 heads of 128
// in bf16: 785 us, 72 of them the selection (bound by its instructions), the gather 695 at 6.1 TB/s. One 4-bit sequence of 4001 cut to
// 1000, 8 layers: 37 us, bound by latency (13 + 12 and two launches; 10 to move the bytes).
#include "kv_q4.h"

using namespace cast;

namespace {

constexpr int kSelThreads = 512;
constexpr int kSelItems = 4;                       // positions per thread and round of the counting pass
constexpr int kBins = 2048;
constexpr int kMoveThreads = 256;

struct EvictParams {
  Paging g;
  int B, Hkv, budget, recent;
  float* mass;   // [n_layers][B][Hkv][max_pos]
  int32_t* kept; // [n_layers][B][Hkv][budget]
  int32_t* kv_len;
  int32_t* ticket;
  DevState* st;
};

// Larger key, larger weight; NaN below everything.
__device__ __forceinline__ uint32_t mass_key(float m) { return m != m ? 0u : ordered_bits(m); }

__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const EvictParams p) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t part_s[kSelThreads / 32];
  __shared__ uint32_t found_s[2];
  __shared__ uint2 count_s[2][kSelThreads / 32];
  const int h = blockIdx.x, b = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const long long max_pos = p.g.max_pos();
  const size_t seg = ((size_t)layer * p.B + b) * p.Hkv + h;
  float* const mass = p.mass + seg * (size_t)max_pos;
  int32_t* const kept = p.kept + seg * (size_t)p.budget;
  const int len = p.kv_len[b];
  bool bad = len < 0 || len > max_pos;
  if (!bad && p.g.page_size > 0) {
    const int pages = (int)(((long long)len + p.g.page_size - 1) / p.g.page_size);
    for (int e = tid; e < pages; e += kSelThreads) {
      const int id = p.g.table[(size_t)b * p.g.seq_capacity + e];
      bad = bad || id < 0 || id >= p.g.num_pages;
    }
  }
  if (__syncthreads_or(bad ? 1 : 0)) {
    if (tid == 0) report(p.st, CAST_ERR_BAD_PAGE, b);
    for (int j = tid; j < p.budget; j += kSelThreads) kept[j] = -1;
    return;
  }
  if (len <= p.budget) {
    for (int j = tid; j < p.budget; j += kSelThreads) kept[j] = j < len ? j : -1;
    return;
  }
  const int cand = len - p.recent;           // positions that compete, more than `want`
  const int want = p.budget - p.recent;
  // the want-th largest key, and how many of the positions that hold it stay
  uint32_t key = 0, ties = 0;
  bool none = want == 0;
  if (!none) {
    uint32_t left = (uint32_t)want, mask = 0;
    const int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = shifts[pass], n = 1 << bits[pass];
      for (int i = tid; i < n; i += kSelThreads) hist[i] = 0;
      __syncthreads();
      for (int i0 = tid; i0 < cand; i0 += 8 * kSelThreads) {  // eight loads in flight
        float m[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = i0 + e * kSelThreads < cand ? mass[i0 + e * kSelThreads] : 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t k = mass_key(m[e]);
          if (i0 + e * kSelThreads < cand && (k & mask) == key) atomicAdd(&hist[(k >> shift) & (n - 1)], 1u);
        }
      }
      __syncthreads();
      // from the top: thread t sums the n / kSelThreads bins below those of thread t - 1
      const int per = n / kSelThreads;
      uint32_t mine = 0;
      for (int i = 0; i < per; ++i) mine += hist[n - 1 - (tid * per + i)];
      uint32_t upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
      }
      if (lane == 31) part_s[warp] = upto;
      __syncthreads();
      for (int w = 0; w < warp; ++w) upto += part_s[w];
      if (upto >= left && upto - mine < left) {  // one thread: the counts add up to at least `left`
        uint32_t above = upto - mine;
        int i = 0;
        while (above + hist[n - 1 - (tid * per + i)] < left) above += hist[n - 1 - (tid * per + i++)];
        found_s[0] = (uint32_t)(n - 1 - (tid * per + i));
        found_s[1] = left - above;
      }
      __syncthreads();
      key |= found_s[0] << shift;
      left = found_s[1];
      mask |= (uint32_t)(n - 1) << shift;
    }
    ties = left;
  }
  // Kept positions in order. Counts so far: of keys above `key` (and of recent positions), and of keys equal to it.
  uint32_t above0 = 0, equal0 = 0;
  int round = 0;
  for (int base = 0; base < len; base += kSelThreads * kSelItems, ++round) {
    float m[kSelItems];
    bool up[kSelItems], eq[kSelItems];
    const int i0 = base + tid * kSelItems;
    uint32_t n_up = 0, n_eq = 0;
#pragma unroll
    for (int e = 0; e < kSelItems; ++e) {
      const int i = i0 + e;
      m[e] = i < len ? mass[i] : 0.f;
      const uint32_t k = mass_key(m[e]);
      up[e] = i < len && (i >= cand || (!none && k > key));
      eq[e] = i < cand && !none && k == key;
      n_up += up[e];
      n_eq += eq[e];
    }
    uint2 upto = make_uint2(n_up, n_eq);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, upto.x, o), y = __shfl_up_sync(0xffffffffu, upto.y, o);
      if (lane >= o) {
        upto.x += x;
        upto.y += y;
      }
    }
    if (lane == 31) count_s[round & 1][warp] = upto;
    __syncthreads();  // (and: every weight of this round is in registers before any is overwritten)
    // lane w: the warps' counts up to w
    uint2 sums = lane < kSelThreads / 32 ? count_s[round & 1][lane] : make_uint2(0u, 0u);
#pragma unroll
    for (int o = 1; o < kSelThreads / 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, sums.x, o), y = __shfl_up_sync(0xffffffffu, sums.y, o);
      if (lane >= o) {
        sums.x += x;
        sums.y += y;
      }
    }
    const uint2 all = make_uint2(__shfl_sync(0xffffffffu, sums.x, kSelThreads / 32 - 1), __shfl_sync(0xffffffffu, sums.y, kSelThreads / 32 - 1));
    uint2 before = make_uint2(__shfl_sync(0xffffffffu, sums.x, (warp + 31) & 31), __shfl_sync(0xffffffffu, sums.y, (warp + 31) & 31));
    before = warp == 0 ? make_uint2(above0, equal0) : make_uint2(above0 + before.x, equal0 + before.y);
    uint32_t nu = before.x + upto.x - n_up, ne = before.y + upto.y - n_eq;
#pragma unroll
    for (int e = 0; e < kSelItems; ++e) {
      const uint32_t at = nu + min(ne, ties);
      if (up[e] || (eq[e] && ne < ties)) {
        kept[at] = i0 + e;
        mass[at] = m[e];
      }
      nu += up[e];
      ne += eq[e];
    }
    above0 += all.x;
    equal0 += all.y;
  }
  __syncthreads();
  for (int i = p.budget + tid; i < len; i += kSelThreads) mass[i] = 0.f;
}

struct MoveParams {
  EvictParams e;
  unsigned char* base[4];   // 16-bit caches: K, V; 4-bit: K codes, V codes, K pairs, V pairs
  size_t stride[4];         // bytes per layer
  FastPaging fg;
};

// The rows of one (layer, sequence, kv-head) of one buffer, VPR threads to a row, ROWS rows at a time: a thread finds the places of
// a row, the next rows' while these rows' loads are out. (Found by every thread for itself the places were most of the work: 32
// layers of 4 sequences cut from 6000-8192 to 4096, 1077 us.)
constexpr int kMoveRows = 512;  // most rows at a time
template <typename V, int VPR, int ROWS, bool kQ4>
__device__ __forceinline__ void move_rows(const MoveParams& p, uint32_t (*src_s)[kMoveRows], uint32_t (*dst_s)[kMoveRows], int which, int layer, int b, int h) {
  constexpr int RPS = kMoveThreads / VPR, U = ROWS / RPS;  // rows per step, steps
  static_assert(ROWS <= kMoveRows && ROWS % RPS == 0, "whole steps");
  const EvictParams& e = p.e;
  const int tid = threadIdx.x, sub = tid % VPR, r = tid / VPR;
  const size_t seg = ((size_t)layer * e.B + b) * e.Hkv + h;
  const int32_t* const kept = e.kept + seg * (size_t)e.budget;
  unsigned char* const base = p.base[which] + p.stride[which] * layer + sub * sizeof(V);
  constexpr int kRow = VPR * (int)sizeof(V);
  auto place = [&](int pos) -> uint32_t {  // (the selection has checked the ids)
    uint32_t page = b, slot = pos, slots = p.fg.seq_capacity;
    if (p.fg.page_size > 0) {
      const uint32_t at = (uint32_t)(((uint64_t)(uint32_t)pos * p.fg.mul) >> p.fg.shift);
      page = __ldg(p.fg.table + (size_t)b * p.fg.seq_capacity + at);
      slots = p.fg.page_size;
      slot = pos - at * slots;
    }
    return kQ4 ? (page * (uint32_t)e.Hkv + h) * slots + slot : (page * slots + slot) * (uint32_t)e.Hkv + h;
  };
  auto find = [&](int j0, int buf) {
#pragma unroll
    for (int i = tid; i < ROWS; i += kMoveThreads)
      if (j0 + i < e.budget) {
        src_s[buf][i] = place(__ldcg(kept + j0 + i));
        dst_s[buf][i] = place(j0 + i);
      }
  };
  // the rows in front of the first that moves lie where they belong (kept[j] - j never falls)
  int lo = 0, hi = e.budget;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (__ldcg(kept + mid) > mid) hi = mid; else lo = mid + 1;
  }
  find(lo, 0);
  __syncthreads();
  int buf = 0;
#pragma unroll 1
  for (int j0 = lo; j0 < e.budget; j0 += ROWS, buf ^= 1) {
    V v[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + u * RPS + r < e.budget) v[u] = __ldcg(reinterpret_cast<const V*>(base + (size_t)src_s[buf][u * RPS + r] * kRow));
    find(j0 + ROWS, buf ^ 1);
    __syncthreads();  // the sources of these rows have been read by all, the next rows' places are known
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + u * RPS + r < e.budget) __stcg(reinterpret_cast<V*>(base + (size_t)dst_s[buf][u * RPS + r] * kRow), v[u]);
    __syncthreads();  // (the places may be overwritten)
  }
}

// blockIdx.x: kv-head and buffer of a (sequence, layer)
template <int RB, bool kQ4>  // bytes of a 16-bit cache's row, or of a 4-bit row's codes
__global__ void __launch_bounds__(kMoveThreads) evict_gather_kernel(const MoveParams p) {
  constexpr int kPieces = kQ4 ? 4 : 2;
  const int piece = blockIdx.x % kPieces, h = blockIdx.x / kPieces, b = blockIdx.y, layer = blockIdx.z;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const EvictParams& e = p.e;
  const int len = e.kv_len[b];
  const size_t seg = ((size_t)layer * e.B + b) * e.Hkv + h;
  const bool cut = len > e.budget && e.kept[seg * (size_t)e.budget] >= 0;
  __syncthreads();  // the whole CTA has read the length
  if (threadIdx.x == 0) {
    // the last CTA of the sequence to have read its length publishes the new one
    const int t = atomicAdd(&e.ticket[b], 1);
    if (t == (int)(gridDim.x * gridDim.z) - 1) {
      e.ticket[b] = 0;
      if (cut) e.kv_len[b] = e.budget;
    }
  }
  if (!cut) return;
  __shared__ uint32_t src_s[2][kMoveRows], dst_s[2][kMoveRows];
  if constexpr (kQ4) {
    if (piece < 2) move_rows<uint4, RB / 16, 512, true>(p, src_s, dst_s, piece, layer, b, h);
    else move_rows<uint32_t, 1, 512, true>(p, src_s, dst_s, piece, layer, b, h);
  } else {
    move_rows<uint4, RB / 16, 32768 / RB, false>(p, src_s, dst_s, piece, layer, b, h);  // 32 KB at a time
  }
}

cast_status launch_evict(cast_ctx* c, MoveParams& p, int n_layers, int B, int Hkv, int pieces, void* kern, cudaStream_t s) {
  if (n_layers > 65535 || (long long)Hkv * pieces > 0x7fffffffll) return CAST_ERR_CAPACITY;
  c->tree_inputs_fresh = 1;  // kv_len and cache rows: an attention call that follows reads them after its dependency wait
  p.e.ticket = c->compact_ticket;
  p.e.st = c->state;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(Hkv, B, n_layers);
  cfg.blockDim = dim3(kSelThreads, 1, 1);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // launched while its predecessor drains; waits for it
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, evict_select_kernel, p.e);
  if (e == cudaSuccess) {
    cfg.gridDim = dim3(Hkv * pieces, B, n_layers);
    cfg.blockDim = dim3(kMoveThreads, 1, 1);
    void* args[] = {&p};
    e = cudaLaunchKernelExC(&cfg, kern, args);
  }
  if (e != cudaSuccess) {
    cudaGetLastError();
    return CAST_ERR_CUDA;
  }
  return CAST_OK;
}

}  // namespace

extern "C" cast_status cast_evict_kv(cast_ctx* c, void* k_cache, void* v_cache, cast_dtype dtype, int B, int n_layers,
                                     size_t layer_stride_bytes, int Hkv, int D, int page_size, const int32_t* page_table,
                                     int seq_capacity, int num_pages, int budget, int recent, float* mass, int32_t* kept,
                                     int32_t* kv_len, void* stream) {
  const Paging g = {page_table, page_size, seq_capacity, num_pages};
  if (!c || !k_cache || !v_cache || !mass || !kept || !kv_len || B < 1 || n_layers < 1 || Hkv < 1 || page_size < 0 ||
      seq_capacity < 1 || (page_size > 0 && (!page_table || num_pages < 1)) || budget < 1 || recent < 0 || recent > budget ||
      !on_device(c))
    return CAST_ERR_INVALID_ARG;
  if (dtype != CAST_F32 && dtype != CAST_BF16) return CAST_ERR_DTYPE;
  if (B > c->cfg.max_batch || g.max_pos() > kMaxPositions) return CAST_ERR_CAPACITY;
  if (D != 64 && D != 128) return CAST_ERR_SHAPE;
  if (((uintptr_t)k_cache | (uintptr_t)v_cache | layer_stride_bytes) & 15) return CAST_ERR_SHAPE;
  const int rb = D * (dtype == CAST_F32 ? 4 : 2);
  MoveParams p = {};
  p.e.g = g; p.e.B = B; p.e.Hkv = Hkv; p.e.budget = budget; p.e.recent = recent;
  p.e.mass = mass; p.e.kept = kept; p.e.kv_len = kv_len;
  p.base[0] = (unsigned char*)k_cache; p.base[1] = (unsigned char*)v_cache;
  p.stride[0] = p.stride[1] = layer_stride_bytes;
  if (!fast_paging(g, B, Hkv, &p.fg)) return CAST_ERR_CAPACITY;
  void* kern = rb == 128 ? (void*)evict_gather_kernel<128, false> : rb == 256 ? (void*)evict_gather_kernel<256, false>
                                                                              : (void*)evict_gather_kernel<512, false>;
  return launch_evict(c, p, n_layers, B, Hkv, 2, kern, (cudaStream_t)stream);
}

extern "C" cast_status cast_evict_kv_q4(cast_ctx* c, void* k_codes, void* k_range, void* v_codes, void* v_range,
                                        size_t code_stride_bytes, size_t range_stride_bytes, int B, int n_layers, int Hkv, int D,
                                        int page_size, const int32_t* page_table, int seq_capacity, int num_pages, int budget,
                                        int recent, float* mass, int32_t* kept, int32_t* kv_len, void* stream) {
  const Paging g = {page_table, page_size, seq_capacity, num_pages};
  if (!mass || !kept || !kv_len || n_layers < 1 || budget < 1 || recent < 0 || recent > budget) return CAST_ERR_INVALID_ARG;
  const cast_status st = check_q4(c, B, Hkv, D, g, k_codes, k_range, v_codes, v_range, code_stride_bytes, range_stride_bytes);
  if (st != CAST_OK) return st;
  MoveParams p = {};
  p.e.g = g; p.e.B = B; p.e.Hkv = Hkv; p.e.budget = budget; p.e.recent = recent;
  p.e.mass = mass; p.e.kept = kept; p.e.kv_len = kv_len;
  p.base[0] = (unsigned char*)k_codes; p.base[1] = (unsigned char*)v_codes;
  p.base[2] = (unsigned char*)k_range; p.base[3] = (unsigned char*)v_range;
  p.stride[0] = p.stride[1] = code_stride_bytes;
  p.stride[2] = p.stride[3] = range_stride_bytes;
  if (!fast_paging(g, B, Hkv, &p.fg)) return CAST_ERR_CAPACITY;
  void* kern = D == 64 ? (void*)evict_gather_kernel<32, true> : (void*)evict_gather_kernel<64, true>;
  return launch_evict(c, p, n_layers, B, Hkv, 4, kern, (cudaStream_t)stream);
}
