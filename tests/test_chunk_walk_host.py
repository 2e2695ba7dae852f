"""The tiles that the chunk attention walks, on the host: the kernels' own arithmetic, compiled for the CPU, against the definition of
what a row sees."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2510_26577_b200 import build

HARNESS = r"""
#include "cast.h"
#include "chunk_attn.h"
using namespace cast;
template <int PT, bool kTree>
static void walk(const int* a, int* out) {
  ChunkParams p = {};
  p.max_pos = a[0]; p.window = a[1]; p.sinks = a[2];
  ChunkSeq s = {};
  s.L = a[3]; s.n = a[4]; s.d0 = (unsigned short)a[5];
  const Span x = span_of<PT, kTree>(p, s, a[6], a[7]);
  out[0] = x.lo; out[1] = x.hi; out[2] = x.s_end; out[3] = x.n;
  for (int i = 0; i < x.n && i < 64; ++i) out[4 + i] = x.tile(i);
  x.template unseen_halves<PT>(a[8], a[9] < 0 ? x.n : a[9], out[68], out[69], out[70]);
}
extern "C" CAST_API int page(int page_size, int pos) {
  FastPaging f;
  fast_paging({nullptr, page_size, 1, 1}, 1, 1, &f);
  return (int)(((unsigned long long)(uint32_t)pos * f.mul) >> f.shift);
}
extern "C" CAST_API void span(int tile, int tree, const int* a, int* out) {
  if (tile == 64) tree ? walk<64, true>(a, out) : walk<64, false>(a, out);
  else tree ? walk<128, true>(a, out) : walk<128, false>(a, out);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("walk")
    src, out = d / "walk.cu", d / "walk.so"
    src.write_text(HARNESS)
    subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-shared", "-o", str(out), str(src)], check=True, capture_output=True, text=True)
    return ctypes.CDLL(str(out))


def span(lib, tile, tree, max_pos, window, sinks, L, n, d0, tf, tl, cut=(0, -1), halves=False):
    a, out = np.array([max_pos, window, sinks, L, n, d0, tf, tl, *cut], np.int32), np.zeros(71, np.int32)
    lib.span(tile, int(tree), a.ctypes.data_as(ctypes.c_void_p), out.ctypes.data_as(ctypes.c_void_p))
    assert out[3] <= 64
    return (out[0], out[1], out[2], out[4:4 + out[3]]) + ((out[68:],) if halves else ())


def walked(positions, lo, hi, s_end, tiles, tile):
    """Whether each position is loaded: in a tile of the walk and in the ranges that some row sees."""
    return np.isin(positions // tile, tiles) & (((positions >= lo) & (positions < hi)) | (positions < s_end))


@pytest.mark.parametrize("tile", [64, 128])
def test_every_token_that_a_trees_row_sees_is_walked(lib, tile):
    """Random trees, their later rows, short windows, sinks that reach into the tree."""
    rng = np.random.default_rng(tile)
    lost = 0
    for _ in range(20000):
        n = int(rng.integers(1, 40))
        L, window, sinks = int(rng.integers(0, 150)), int(rng.integers(1, 8)), int(rng.integers(0, 170))
        parent = [-1] + [int(rng.integers(max(0, t - 3), t)) for t in range(1, n)]
        depth = np.zeros(n, np.int64)
        for t in range(1, n):
            depth[t] = depth[parent[t]] + 1
        first = int(rng.integers(0, n))
        seen = np.zeros(L + n, bool)
        pos = np.arange(L)
        for t in range(first, n):
            seen[:L] |= (L + depth[t] - pos < window) | (pos < sinks)
            j = t
            while j >= 0:
                seen[L + j] |= depth[t] - depth[j] < window or L + depth[j] < sinks
                j = parent[j]
        d0 = int(depth[first:].min()) if first else 0
        lo, hi, s_end, tiles = span(lib, tile, True, 1 << 20, window, sinks, L, n, d0, first, n - 1)
        at = np.flatnonzero(seen)
        lost += not walked(at, lo, hi, s_end, tiles, tile).all()
    assert lost == 0


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("edge", [0, 1, 63, 64, 65, 127])
def test_every_tile_has_a_half_that_some_row_sees(lib, tree, edge):
    """Around and past the capacity too, wherever it lies in a tile: a tile both of whose halves are passed over is one whose place in the ring
    nobody gives back. And what is passed over is what no row sees, by the definition."""
    rng = np.random.default_rng(edge)
    for _ in range(6000):
        max_pos = 128 * int(rng.integers(1, 6)) + edge
        n = int(rng.integers(1, 129 if tree else 700))
        L = int(rng.integers(0, 2 * max_pos))
        window, sinks = int(rng.integers(0, 400)), int(rng.choice([0, 1, 4, 64, 130, 1000]))
        tf = int(rng.integers(0, n))
        tl = n - 1 if tree else min(n - 1, tf + int(rng.integers(0, 200)))
        d0 = int(rng.integers(0, tf + 1)) if tree else 0
        lo, hi, s_end, tiles, _ = span(lib, 128, tree, max_pos, window, sinks, L, n, d0, tf, tl, halves=True)
        tile0 = int(rng.integers(0, len(tiles) + 1))
        stop = int(rng.integers(tile0, len(tiles) + 1))
        *_, (no0, no1a, no1b) = span(lib, 128, tree, max_pos, window, sinks, L, n, d0, tf, tl, cut=(tile0, stop), halves=True)
        for i, t in enumerate(tiles[tile0:stop]):
            pos = 128 * int(t) + np.arange(128)
            if tree:  # (a bound on what the rows see: all that any tree's could)
                seen = (pos < L + n) & ((pos < sinks) | (pos > L + d0 - window) | (pos >= L)) if window else pos < L + n
            else:
                seen = (pos <= L + tl) & ((pos < sinks) | (pos > L + tf - window)) if window else pos <= L + tl
            half = (seen & (pos < max_pos)).reshape(2, 64).any(1)
            skipped = np.array([i == no0, i in (no1a, no1b)])
            assert not skipped.all(), (max_pos, n, L, window, sinks, tf, tl)
            assert not (half & skipped).any() and half.any()


def test_pages_of_any_size_divide_exactly(lib):
    """The constants that stand for a division by the page size, up to pages of 2^31 - 2^16 positions."""
    rng = np.random.default_rng(1)
    sizes = {1, 2, 3, 2 ** 31 - 2 ** 16} | {(1 << e) + d for e in range(1, 31) for d in (-1, 0, 1, 8)} - {0}
    for size in sorted(sizes | set(rng.integers(1, 2 ** 31 - 2 ** 16, 200).tolist())):
        most = 2 ** 31 - 1
        k = int(rng.integers(1, most // size + 1))
        for pos in {0, size - 1, size, k * size - 1, k * size, most - 1, most, int(rng.integers(0, most))}:
            if 0 <= pos <= most:
                assert lib.page(size, pos) == pos // size, (size, pos)


def test_the_kernels_wait_before_they_read_and_release_behind_their_allocation():
    """What test_dependent_launch_host.py asks of the other kernels: a wait before anything is read, tensor memory behind it, and the
    dependents released by the warp that has it."""
    from test_dependent_launch_host import _body, _source
    kernel = _body(_source("chunk_attention_tc.cu"), "chunk_attn_tc_kernel(const __grid_constant__ ChunkParams p")
    steps = ("griddepcontrol.wait", "if (warp == 10) {", "tcgen05.alloc", "tcgen05.relinquish_alloc_permit", "griddepcontrol.launch_dependents")
    at = [kernel.index(x) for x in steps]
    assert at == sorted(at) and all(kernel.count(x) == 1 for x in (steps[0], *steps[2:]))
    assert at[-1] < at[1] + len(_body(kernel[at[1]:], "if (warp == 10)"))
    for name, head, inputs in (("chunk_attention_tc.cu", "chunk_attn_tc_kernel(const", ("p.kv_len[", "plan_warp<", "depth_of(")),
                               ("chunk_attention.cu", "chunk_attn_cc_kernel(const", ("make_plan<", "depth_of(")),
                               ("append_kv.cu", "append_kernel(const", ("p.n_rows[", "p.start[", "p.inv_freq[", "p.q_weight", "p.position["))):
        body = _body(_source(name), head)
        wait = body.index("griddepcontrol.wait")
        assert "return" not in body[:wait] and body.count("griddepcontrol.wait") == 1
        assert all(x not in body[:wait] for x in inputs) and any(x in body[wait:] for x in inputs)
        assert wait < body.index("griddepcontrol.launch_dependents")
