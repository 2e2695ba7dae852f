// What the two kernels of cast_chunk_attention and cast_tree_attention_window share: which positions a row sees, the line of tiles
// that is cut into the CTAs' pieces, and where the pieces of an item meet again.
//
// A query row is a (new token, head of the GQA group) pair; an item is a block of rows of one (sequence, kv-head). Row t of a chunk
// stands at position L + t and sees the positions p <= L + t, with a window those of them with p > L + t - window or p < sinks. Row t of
// a tree stands at L + depth[t]; of the prefix it sees the same, of the tree its ancestors that lie in the window (by depth) or among the sinks.
// An item walks the tiles that some row of it sees: those of the sinks, then those from the window's start on. (A tree's token j lies at L + j but
// stands at L + depth[j], so as a sink it may lie behind the sinks and before the window: a tree's own places are walked whatever the window.)
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
  int block_tokens;         // where they are whole tokens: how many; else 0
  int max_pos;              // capacity of a sequence
  int min_units;            // a CTA's stretch at least
  float join;               // partials that are joined in the time of a tile (0: any number)
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
  int L, n, off;          // prefix (up to 2^31 - 1, whatever the capacity), tokens, row of token 0
  unsigned short F, d0;   // tree: first output token, least depth of an output token
};

// The tiles of an item.
struct Span {
  int lo, hi, s_end;   // positions [0, s_end) and [lo, hi)
  int st, wt;          // tiles 0..st-1, then wt, wt + 1, ...
  int n;
  __host__ __device__ __forceinline__ int tile(int i) const { return i < st ? i : wt + (i - st); }
  // Whether some row sees a position of half `f` of tile i (tiles of PT positions).
  template <int PT>
  __host__ __device__ __forceinline__ bool half_seen(int i, int f) const {
    const int pos0 = tile(i) * PT + f * (PT / 2);
    return pos0 < s_end || (pos0 < hi && pos0 + PT / 2 > lo);
  }
  // Of the tiles [tile0, stop), counted from tile0: one whose first half no row sees, two whose second half none does (-1: none). Only at the edges: the
  // sinks' last tile, the window's first, the last. Some row sees one half of every tile at least: the other roles of a kernel count on a step in each.
  template <int PT>
  __host__ __device__ __forceinline__ void unseen_halves(int tile0, int stop, int& no0, int& no1a, int& no1b) const {
    const int a1 = st - 1 - tile0, b0 = st - tile0, c1 = n - 1 - tile0, here = stop - tile0;
    no1a = a1 >= 0 && a1 < here && !half_seen<PT>(tile0 + a1, 1) ? a1 : -1;
    no0 = b0 >= 0 && b0 < here && !half_seen<PT>(tile0 + b0, 0) ? b0 : -1;
    no1b = c1 > a1 && c1 < here && !half_seen<PT>(tile0 + c1, 1) ? c1 : -1;
  }
};

template <int PT, bool kTree>
__host__ __device__ __forceinline__ Span span_of(const ChunkParams& p, const ChunkSeq& s, int tf, int tl) {
  Span x;
  const long long end = (long long)s.L + (kTree ? s.n : tl + 1);
  x.hi = (int)(end < p.max_pos ? end : p.max_pos);
  x.lo = 0;
  if (p.window > 0) {
    long long lo = (long long)s.L + (kTree ? s.d0 : tf) - p.window + 1;
    if (kTree && lo > s.L) lo = s.L;
    x.lo = lo < 0 ? 0 : lo > x.hi ? x.hi : (int)lo;
  }
  x.s_end = x.lo > 0 ? (p.sinks < x.lo ? p.sinks : x.lo) : 0;
  x.st = (int)((uint32_t)(x.s_end + PT - 1) / PT);
  x.wt = (int)((uint32_t)x.lo / PT);
  if (x.wt < x.st) x.wt = x.st;
  const int wt1 = (int)((uint32_t)(x.hi + PT - 1) / PT);
  x.n = x.st + (x.lo < x.hi && wt1 > x.wt ? wt1 - x.wt : 0);  // (rows wholly past the capacity: lo = hi, and a tile they both lie in is none)
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

// First and last token of a row block.
__device__ __forceinline__ int first_token(const ChunkParams& p, const ChunkSeq& s, int rb) {
  return s.F + (p.block_tokens ? rb * p.block_tokens : rb * p.block_rows / p.G);
}
__device__ __forceinline__ int last_token(const ChunkParams& p, const ChunkSeq& s, int rb) {
  if (p.block_tokens) return min((int)s.F + (rb + 1) * p.block_tokens, s.n) - 1;
  return s.F + (min((rb + 1) * p.block_rows, (s.n - s.F) * p.G) - 1) / p.G;
}
__device__ __forceinline__ int blocks_of(const ChunkParams& p, const ChunkSeq& s) {
  return (int)(p.block_tokens ? (uint32_t)(s.n - s.F + p.block_tokens - 1) / (uint32_t)p.block_tokens
                              : ((uint32_t)(s.n - s.F) * p.G + p.block_rows - 1) / (uint32_t)p.block_rows);
}
template <int PT, bool kTree>
__device__ __forceinline__ Span block_span(const ChunkParams& p, const ChunkSeq& s, int rb) {
  return span_of<PT, kTree>(p, s, first_token(p, s, rb), last_token(p, s, rb));
}

// a * b / c for c >= 1, in 32 bits where they hold it (a division in 64 is a chain of some hundred cycles, and this is on the way to the first tile).
__device__ __forceinline__ long long mul_div(long long a, int b, long long c) {
  const long long x = a * b;
  return x < 0xffffffffll && c <= 0xffffffffll ? (long long)((uint32_t)x / (uint32_t)c) : x / c;
}

// A warp's plan, a lane per two sequences (lane l: sequences l and l + 32): the sequences, the units up to and including each, all units, all items. Between the kernel's start and its
// first load there is one round trip to memory and one scan. (A warp per sequence, with a barrier in front and behind, took 2.6 us for one sequence and 5.7 for 64.)
constexpr int kPerLane = CAST_MAX_BATCH / 32;
template <int PT, bool kTree>
__device__ __forceinline__ void plan_warp(const ChunkParams& p, ChunkSeq (&seq)[kPerLane], long long (&upto)[kPerLane], long long& units, long long& items) {
  const int lane = threadIdx.x & 31;
  int L[kPerLane], n[kPerLane], F[kPerLane], off[kPerLane];
#pragma unroll
  for (int j = 0; j < kPerLane; ++j) {  // all loads first
    const int b = j * 32 + lane;
    const bool in = b < p.B;
    L[j] = in ? p.kv_len[b] : 0;
    n[j] = in ? p.n_new[b] : 0;
    F[j] = in && p.first_row ? p.first_row[b] : 0;
    off[j] = in && p.row_start ? p.row_start[b] : 0;
  }
  long long run = 0;
  items = 0;
#pragma unroll
  for (int j = 0; j < kPerLane; ++j) {
    const int b = j * 32 + lane;
    ChunkSeq s = {max(L[j], 0), n[j], p.row_start ? off[j] : b * p.rows, 0, 0};
    const int most = kTree ? p.Nmax : p.rows;
    bool bad = kTree && s.n > most;  // (a chunk's count past its rows is cut to them)
    s.n = min(max(s.n, 0), most);
    if (p.row_start && s.n > 0 && (s.off < 0 || (long long)s.off + s.n > p.rows)) {
      bad = true;
      s.n = 0;
    }
    if (bad && blockIdx.x == 0) report(p.st, CAST_ERR_BAD_TREE, b);
    s.F = (unsigned short)(kTree ? min(max(F[j], 0), s.n) : 0);
    if (s.n > s.F && (long long)s.L + s.n > p.max_pos && blockIdx.x == 0) report(p.st, CAST_ERR_BAD_PAGE, b);  // (L stays: windows hang on it)
    if (kTree && p.first_row) {  // (a whole tree has its root, at depth 0)
      for (unsigned left = __ballot_sync(0xffffffffu, s.n > s.F); left; left &= left - 1) {
        const int l = __ffs(left) - 1;
        ChunkSeq x = s;
        x.n = __shfl_sync(0xffffffffu, s.n, l);
        x.off = __shfl_sync(0xffffffffu, s.off, l);
        int d = CAST_MAX_TREE;
        for (int t = __shfl_sync(0xffffffffu, (int)s.F, l) + lane; t < x.n; t += 32) d = min(d, depth_of(p, x, t));
        d = __reduce_min_sync(0xffffffffu, d);
        if (lane == l) s.d0 = (unsigned short)d;
      }
    }
    const int blocks = blocks_of(p, s);
    items += (long long)__reduce_add_sync(0xffffffffu, (unsigned)blocks) * p.Hkv;
    long long u = 0;
    if (blocks <= 4) {
      for (int rb = 0; rb < blocks; ++rb) u += block_span<PT, kTree>(p, s, rb).n + kItemCost;
    }
    for (unsigned left = __ballot_sync(0xffffffffu, blocks > 4); left; left &= left - 1) {  // many row blocks: a lane each
      const int l = __ffs(left) - 1, nb = __shfl_sync(0xffffffffu, blocks, l);
      ChunkSeq x;
      x.L = __shfl_sync(0xffffffffu, s.L, l);
      x.n = __shfl_sync(0xffffffffu, s.n, l);
      x.F = (unsigned short)__shfl_sync(0xffffffffu, (int)s.F, l);
      x.d0 = (unsigned short)__shfl_sync(0xffffffffu, (int)s.d0, l);
      long long y = 0;
      for (int rb = lane; rb < nb; rb += 32) y += block_span<PT, kTree>(p, x, rb).n + kItemCost;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) y += __shfl_xor_sync(0xffffffffu, y, o);
      if (lane == l) u = y;
    }
    u *= p.Hkv;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, u, o);
      if (lane >= o) u += y;
    }
    u += run;
    run = __shfl_sync(0xffffffffu, u, 31);
    seq[j] = s;
    upto[j] = u;
  }
  units = run;
}
// CTAs that get a stretch. One CTA joins the partials of an item, one behind the other, so n stretches of an item of A tiles take A / n + n / join tiles' time: n is
// sqrt(join A) at most, over all items sqrt(join units items).
__device__ __forceinline__ int workers_of(const ChunkParams& p, long long units, long long items) {
  long long w = mul_div(units, 1, p.min_units);
  if (p.join > 0.f) w = min(w, (long long)fminf(sqrtf(p.join * (float)units * (float)items), 1e6f));
  return (int)(w < 1 ? 1 : w < (long long)gridDim.x ? w : (long long)gridDim.x);
}

// The plan in shared memory. All threads of the CTA call; ends with a barrier.
template <int PT, bool kTree>
__device__ __forceinline__ void make_plan(const ChunkParams& p, ChunkPlan& pl) {
  const int lane = threadIdx.x & 31;
  if (threadIdx.x < 32) {
    ChunkSeq seq[kPerLane];
    long long upto[kPerLane], units, items;
    plan_warp<PT, kTree>(p, seq, upto, units, items);
#pragma unroll
    for (int j = 0; j < kPerLane; ++j) {
      pl.seq[j * 32 + lane] = seq[j];
      pl.pre[j * 32 + lane + 1] = upto[j];
    }
    if (lane == 0) {
      pl.pre[0] = 0;
      pl.units = units;
      pl.workers = workers_of(p, units, items);
    }
  }
  __syncthreads();
}

__device__ __forceinline__ long long bound_of(long long units, int workers, int c) { return mul_div(units, c, workers); }
__device__ __forceinline__ int owner_of(long long units, int workers, long long u) { return (int)mul_div((u + 1) * workers - 1, 1, units); }
__device__ __forceinline__ long long bound_of(const ChunkPlan& pl, int c) { return bound_of(pl.units, pl.workers, c); }
__device__ __forceinline__ int owner_of(const ChunkPlan& pl, long long u) { return owner_of(pl.units, pl.workers, u); }

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
  w.blocks = blocks_of(p, s);
  w.rb = 0;
  for (int rb0 = 0; w.blocks > 1; rb0 += 32) {  // the row block that the stretch begins in
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
  w.h = (int)mul_div(left, 1, len);
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
      w.blocks = blocks_of(p, s);
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
  const long long pos = (long long)s.L + (kTree ? depth : t);
  RowSight r;
  const long long hi = kTree ? s.L : pos + 1;
  r.hi = (int)(hi < p.max_pos ? hi : p.max_pos);
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
  // bits past the tree or the capacity see nothing
  const int valid = min(s.n, max(p.max_pos - s.L, 0)) - w * 32;
  return valid >= 32 ? a : valid <= 0 ? 0u : a & ((1u << valid) - 1u);
}

}  // namespace cast
