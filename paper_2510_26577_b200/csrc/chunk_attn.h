// What the two kernels of cast_chunk_attention and cast_tree_attention_window share: which positions a row sees, the line of tiles
// that is cut into the CTAs' pieces, and where the pieces of an item meet again.
//
// A query row is a (new token, head of the GQA group) pair; an item is a block of rows of one (sequence, kv-head). Row t of a chunk
// stands at position L + t and sees the positions p <= L + t, with a window those of them with p > L + t - window or p < sinks. Row t of
// a tree stands at L + depth[t]; of the prefix it sees the same, of the tree its ancestors that lie in the window (by depth) or among the sinks.
// An item walks the tiles that some row of it sees: those of the sinks, then those from the window's start on.
//
// The line: items one behind the other (sequence, row block, kv-head fastest), each as long as its tiles plus kItemCost for its queries and
// output; CTA c of n takes the stretch [c U / n, (c + 1) U / n) of it, so ragged batches load the machine evenly. An item that lies across
// CTAs leaves partials in the workspace, two places per CTA (the item that its stretch begins inside of, the item that it ends inside of);
// the last CTA to finish an item (an atomic ticket, nothing spins) merges them in CTA order, so the same inputs give the same bits.
#pragma once

#include "kv_q4.h"

namespace cast {

constexpr int kItemCost = 2;   // tiles that an item's start and end are worth
constexpr int kChunkGrid = 512;  // CTAs of a launch at most

struct ChunkParams {
  const void *q, *k, *v;
  void* out;
  int B, rows, Hq, Hkv, G;  // rows: of a sequence in q and out, or of all where row_start is given
  int block_rows;           // rows of an item at most
  int min_units;            // a CTA's stretch at least
  int Nmax;                 // tree: most tokens
  int window, sinks;        // window 0: none
  const int32_t *row_start, *kv_len, *n_new, *first_row, *depth;
  const uint32_t* anc;      // null: a chunk
  int words;
  Paging g;
  float scale;
  int32_t* ticket;          // [kChunkGrid]
  float* part_o;            // [grid][2][block rows][D]
  float2* part_ml;          // [grid][2][block rows] reference, sum
  DevState* st;
};

// A sequence's live rows and what its items walk.
struct ChunkSeq {
  int L, n, off;          // prefix, tokens, row of token 0
  unsigned short F, d0;   // tree: first output token, least depth of an output token
};

// The tiles of an item.
struct Span {
  int lo, hi, s_end;   // positions [0, s_end) and [lo, hi)
  int st, wt;          // tiles 0..st-1, then wt, wt + 1, ...
  int n;
  __device__ __forceinline__ int tile(int i) const { return i < st ? i : wt + (i - st); }
};

template <int PT, bool kTree>
__device__ __forceinline__ Span span_of(const ChunkParams& p, const ChunkSeq& s, int tf, int tl) {
  const long long max_pos = p.g.max_pos();
  Span x;
  const long long end = (long long)s.L + (kTree ? s.n : tl + 1);
  x.hi = (int)(end < max_pos ? end : max_pos);
  const long long first = (long long)s.L + (kTree ? s.d0 : tf);
  const long long lo = p.window > 0 ? first - p.window + 1 : 0;
  x.lo = lo < 0 ? 0 : lo > x.hi ? x.hi : (int)lo;
  x.s_end = x.lo > 0 ? (p.sinks < x.lo ? p.sinks : x.lo) : 0;
  x.st = (x.s_end + PT - 1) / PT;
  x.wt = x.lo / PT;
  if (x.wt < x.st) x.wt = x.st;
  const int wt1 = (x.hi + PT - 1) / PT;
  x.n = x.st + (wt1 > x.wt ? wt1 - x.wt : 0);
  return x;
}

// A tree token's depth as the masks use it.
__device__ __forceinline__ int depth_of(const ChunkParams& p, const ChunkSeq& s, int t) {
  const int d = p.depth[s.off + t];
  return d < 0 ? 0 : d > CAST_MAX_TREE ? CAST_MAX_TREE : d;
}

// The schedule, in shared memory.
struct ChunkPlan {
  ChunkSeq seq[CAST_MAX_BATCH];
  long long pre[CAST_MAX_BATCH + 1];  // units of the sequences before
  long long units;
  int workers;
};

template <int PT, bool kTree>
__device__ __forceinline__ Span block_span(const ChunkParams& p, const ChunkSeq& s, int rb) {
  const int r0 = rb * p.block_rows, rows = (s.n - s.F) * p.G;
  const int r1 = min(r0 + p.block_rows, rows);
  return span_of<PT, kTree>(p, s, (int)s.F + r0 / p.G, (int)s.F + (r1 - 1) / p.G);
}

// All threads of the CTA call; ends with a barrier.
template <int PT, bool kTree>
__device__ __forceinline__ void make_plan(const ChunkParams& p, ChunkPlan& pl) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  for (int b = tid; b < CAST_MAX_BATCH; b += blockDim.x) {
    ChunkSeq s = {0, 0, 0, 0, 0};
    int F = 0;
    if (b < p.B) {
      const long long all = p.row_start ? p.rows : (long long)p.B * p.rows;
      s.L = max(p.kv_len[b], 0);
      s.n = p.n_new[b];
      if (p.first_row) F = p.first_row[b];
      s.off = p.row_start ? p.row_start[b] : b * p.rows;
      const int most = kTree ? p.Nmax : p.rows;
      bool bad = false;
      if (s.n > most) {
        bad = kTree;  // (a chunk's count past its rows is cut to them)
        s.n = most;
      }
      s.n = max(s.n, 0);
      if (p.row_start && (s.off < 0 || (long long)s.off + s.n > all)) {
        bad = s.n > 0;
        s.n = 0;
      }
      if (bad && blockIdx.x == 0) report(p.st, CAST_ERR_BAD_TREE, b);
      F = min(max(F, 0), s.n);  // (with a tree, so it fits)
      s.F = (unsigned short)(kTree ? F : 0);
      if ((long long)s.L + s.n > p.g.max_pos() && s.n > s.F) {
        if (blockIdx.x == 0) report(p.st, CAST_ERR_BAD_PAGE, b);
        if (s.L > p.g.max_pos()) s.L = (int)p.g.max_pos();
      }
    }
    pl.seq[b] = s;
  }
  __syncthreads();
  for (int b = warp; b < CAST_MAX_BATCH; b += warps) {
    long long u = 0;
    if (b < p.B) {
      ChunkSeq s = pl.seq[b];
      if (kTree) {
        int d = CAST_MAX_TREE;
        for (int t = s.F + lane; t < s.n; t += 32) d = min(d, depth_of(p, s, t));
        s.d0 = (unsigned short)__reduce_min_sync(0xffffffffu, d);
        if (lane == 0) pl.seq[b].d0 = s.d0;
      }
      const int blocks = (int)(((long long)(s.n - s.F) * p.G + p.block_rows - 1) / p.block_rows);
      for (int rb = lane; rb < blocks; rb += 32) u += block_span<PT, kTree>(p, s, rb).n + kItemCost;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) u += __shfl_xor_sync(0xffffffffu, u, o);
    }
    if (lane == 0) pl.pre[b + 1] = u * p.Hkv;
  }
  __syncthreads();
  if (warp == 0) {
    long long run = 0;
#pragma unroll
    for (int j = 0; j < CAST_MAX_BATCH / 32; ++j) {
      long long x = pl.pre[j * 32 + lane + 1];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      x += run;
      __syncwarp();
      pl.pre[j * 32 + lane + 1] = x;
      run = __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) {
      pl.pre[0] = 0;
      pl.units = run;
      const long long w = run / p.min_units;
      pl.workers = (int)(w < 1 ? 1 : w < (long long)gridDim.x ? w : (long long)gridDim.x);
    }
  }
  __syncthreads();
}

__device__ __forceinline__ long long bound_of(const ChunkPlan& pl, int c) { return pl.units * c / pl.workers; }
__device__ __forceinline__ int owner_of(const ChunkPlan& pl, long long u) { return (int)(((u + 1) * pl.workers - 1) / pl.units); }

// A CTA's way along its stretch, item by item; every warp that follows it computes the same (all 32 lanes call).
struct ChunkWalk {
  long long at, end;    // the rest of the stretch
  int b, rb, h;         // the item
  int blocks;           // row blocks of the sequence
  long long item0;      // the item's first unit
  Span span;
  int t0, t1;           // tiles of the item in this stretch
};

template <int PT, bool kTree>
__device__ __forceinline__ void walk_item(const ChunkParams& p, const ChunkPlan& pl, ChunkWalk& w) {
  const long long a = w.at - w.item0 - kItemCost, z = w.end - w.item0 - kItemCost;
  w.t0 = a < 0 ? 0 : (int)a;
  w.t1 = z < 0 ? 0 : z < w.span.n ? (int)z : w.span.n;
}
template <int PT, bool kTree>
__device__ __forceinline__ void walk_block(const ChunkParams& p, const ChunkPlan& pl, ChunkWalk& w) {
  w.span = block_span<PT, kTree>(p, pl.seq[w.b], w.rb);
}
template <int PT, bool kTree>
__device__ __forceinline__ bool walk_begin(const ChunkParams& p, const ChunkPlan& pl, ChunkWalk& w, int c) {
  const int lane = threadIdx.x & 31;
  w.at = w.end = 0;
  if (c >= pl.workers || pl.units == 0) return false;
  w.at = bound_of(pl, c);
  w.end = bound_of(pl, c + 1);
  w.b = 0;
  for (int j = 0; j < CAST_MAX_BATCH / 32; ++j)
    w.b += __popc(__ballot_sync(0xffffffffu, pl.pre[j * 32 + lane + 1] <= w.at));
  long long left = w.at - pl.pre[w.b], base = pl.pre[w.b];
  const ChunkSeq s = pl.seq[w.b];
  w.blocks = (int)(((long long)(s.n - s.F) * p.G + p.block_rows - 1) / p.block_rows);
  for (int rb0 = 0;; rb0 += 32) {  // the row block that the stretch begins in
    const int rb = rb0 + lane;
    const long long own = rb < w.blocks ? (long long)(block_span<PT, kTree>(p, s, rb).n + kItemCost) * p.Hkv : 0;
    long long x = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    const int hit = __popc(__ballot_sync(0xffffffffu, x <= left));
    if (hit < 32) {
      w.rb = rb0 + hit;
      const long long skip = __shfl_sync(0xffffffffu, x - own, hit);
      left -= skip;
      base += skip;
      break;
    }
    const long long skip = __shfl_sync(0xffffffffu, x, 31);
    left -= skip;
    base += skip;
  }
  walk_block<PT, kTree>(p, pl, w);
  const int len = w.span.n + kItemCost;
  w.h = (int)(left / len);
  w.item0 = base + (long long)w.h * len;
  walk_item<PT, kTree>(p, pl, w);
  return true;
}
// The next item; false behind the stretch.
template <int PT, bool kTree>
__device__ __forceinline__ bool walk_next(const ChunkParams& p, const ChunkPlan& pl, ChunkWalk& w) {
  w.item0 += w.span.n + kItemCost;
  w.at = w.item0;
  if (w.at >= w.end) return false;
  if (++w.h == p.Hkv) {
    w.h = 0;
    if (++w.rb == w.blocks) {
      w.rb = 0;
      do ++w.b;
      while (pl.pre[w.b + 1] == pl.pre[w.b]);  // (units are left, so a sequence with rows follows)
      const ChunkSeq s = pl.seq[w.b];
      w.blocks = (int)(((long long)(s.n - s.F) * p.G + p.block_rows - 1) / p.block_rows);
    }
    walk_block<PT, kTree>(p, pl, w);
  }
  walk_item<PT, kTree>(p, pl, w);
  return true;
}

// What a row sees: prefix and chunk positions [lo, hi) and, below hi, [0, sinks); a tree's positions behind L by its mask.
struct RowSight {
  int lo, hi, sinks;
};
template <bool kTree>
__device__ __forceinline__ RowSight sight_of(const ChunkParams& p, const ChunkSeq& s, int t, int depth) {
  const long long pos = (long long)s.L + (kTree ? depth : t), max_pos = p.g.max_pos();
  RowSight r;
  const long long hi = kTree ? s.L : pos + 1;
  r.hi = (int)(hi < max_pos ? hi : max_pos);
  const long long lo = p.window > 0 ? pos - p.window + 1 : 0;
  r.lo = lo < 0 ? 0 : lo > 0x7fffffffll ? 0x7fffffff : (int)lo;
  r.sinks = p.window > 0 ? p.sinks : 0;
  return r;
}
// Word w of a tree row's mask without the ancestors that the window hides.
__device__ __forceinline__ uint32_t tree_word(const ChunkParams& p, const ChunkSeq& s, int t, int depth, int w) {
  uint32_t a = w < p.words ? p.anc[((size_t)s.off + t) * p.words + w] : 0u;
  if (p.window > 0) {
    for (uint32_t left = a; left; left &= left - 1) {
      const int bit = __ffs(left) - 1, j = w * 32 + bit;
      const int dj = j < s.n ? depth_of(p, s, j) : 0;
      if (depth - dj >= p.window && (long long)s.L + dj >= p.sinks) a &= ~(1u << bit);
    }
  }
  // bits past the tree see nothing
  const int valid = s.n - w * 32;
  return valid >= 32 ? a : valid <= 0 ? 0u : a & ((1u << valid) - 1u);
}

}  // namespace cast
