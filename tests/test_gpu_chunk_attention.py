"""cast_chunk_attention and cast_tree_attention_window against 64 bits."""
import numpy as np
import pytest
import torch

import chunk_oracle as co
import q4_oracle as o4

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step, relative to the value
POISON = [float("nan"), float("inf"), -float("inf")]


@pytest.fixture(scope="module")
def binding():
    from paper_2510_26577_b200 import build
    build.build()
    from paper_2510_26577_b200 import binding as b
    b.load_library()
    return b


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Batch:
    """Sequences of L cached and n new positions over a paged cache, whose rows nobody may see hold NaN and infinities, and
    whose pages outside of the window are gone from the table."""

    def __init__(self, seed, dtype, Hq, Hkv, D, page, L, n, window=0, sinks=0, packed=False, tree=False, first=None, scale=0.0, spread=1.0):
        rng = self.rng = np.random.default_rng(seed)
        self.dtype, self.Hq, self.Hkv, self.D, self.page, self.window, self.sinks, self.scale = dtype, Hq, Hkv, D, page, window, sinks, scale
        self.L, self.n = np.array(L, np.int32), np.array(n, np.int32)
        self.B, self.rows = len(L), max(1, int(self.n.max()))
        self.first = None if first is None else np.array(first, np.int32)
        self.paged = p = o4.Paged(rng, self.B, int((self.L + self.n).max()) + 3, page)
        gen = torch.Generator("cuda").manual_seed(seed)
        self.k, self.v = (torch.randn((*p.shape, Hkv, D), generator=gen, device="cuda").to(DT[dtype]) for _ in range(2))
        self.k *= spread
        self.row0 = np.arange(self.B) * self.rows
        self.total, self.row_start = self.B * self.rows, None
        if packed:
            at = 1
            for b in rng.permutation(self.B):
                self.row0[b] = at
                at += self.n[b] + 1
            self.total, self.row_start = at + 2, self.row0.astype(np.int32)
        self.q = torch.randn((self.total, Hq, D), generator=gen, device="cuda").to(DT[dtype])
        self.tree = None
        if tree:
            self.tree, self.anc, self.depth = [], np.zeros((self.B, self.rows, (self.rows + 31) // 32), np.uint32), np.full((self.B, self.rows), -1, np.int32)
            for b in range(self.B):
                vis = np.zeros((self.n[b], self.n[b]), bool)
                for t in range(self.n[b]):
                    parent = int(min(rng.integers(0, t), rng.integers(0, t))) if t else -1
                    if t:
                        vis[t] = vis[parent]
                    vis[t, t] = True
                    self.depth[b, t] = 0 if t == 0 else self.depth[b, parent] + 1
                    for j in np.flatnonzero(vis[t]):
                        self.anc[b, t, j >> 5] |= np.uint32(1 << (j & 31))
                self.tree.append(vis)
        dead = torch.ones(self.total, dtype=torch.bool)
        for b in range(self.B):
            dead[self.rows_of(b)] = False
        self.q[dead.cuda()] = float("nan")
        self.table = None if p.table is None else p.table.copy()
        self.poison()

    def rows_of(self, b):
        F = min(int(self.first[b]), int(self.n[b])) if self.first is not None else 0
        return self.row0[b] + np.arange(F, self.n[b])

    def seen(self, b):
        F = min(int(self.first[b]), int(self.n[b])) if self.first is not None else 0
        n, L = int(self.n[b]), int(self.L[b])
        stands = L + (self.depth[b, :n] if self.tree is not None else np.arange(n))
        return co.sight(L, stands, self.window, self.sinks, None if self.tree is None else self.tree[b])[F:]

    def poison(self):
        live = np.zeros(self.paged.shape, bool)
        for b in range(self.B):
            pos = np.flatnonzero(self.seen(b).any(0))
            live[self.paged.at(b, pos)] = True
            if self.table is not None:  # entries that no row needs (a tree's own tokens are stored)
                stored = int(self.L[b]) + np.arange(int(self.n[b]) if self.tree is not None else 0)
                gone = np.setdiff1d(np.arange(self.paged.cap), np.concatenate([pos, stored]) // self.page)
                self.table[b, gone] = self.rng.choice([-1, self.paged.pages, 2 ** 31 - 1, -2 ** 31], len(gone))
        dead = dev(~live)
        bad = torch.tensor(POISON, device="cuda")
        for x in (self.k, self.v):
            at = torch.arange(int(dead.sum()), device="cuda") % 3
            x[dead] = bad[at][:, None, None].to(x.dtype)

    def run(self, binding, ctx=None, out=None, check=True):
        tokens = self.rows if self.tree is not None else 8
        ctx = ctx or binding.CastContext(max_batch=self.B, vocab=1000, top_k=4, max_depth=6, total_token=tokens, max_tree=tokens)
        ctx.cast_reserve_chunk_attention(DT[self.dtype], self.D)
        out = torch.full_like(self.q, float("nan")) if out is None else out
        where = (self.page, dev(self.table), self.paged.cap, self.paged.pages)
        if self.tree is not None:
            ctx.cast_tree_attention_window(self.q, self.k, self.v, self.B, self.Hq, self.Hkv, self.D, *where, dev(self.L), dev(self.anc.view(np.int32)),
                                           dev(self.depth), dev(self.n), dev(self.first), self.window, self.sinks, self.scale, out)
        else:
            ctx.cast_chunk_attention(self.q, self.k, self.v, self.B, self.total if self.row_start is not None else self.rows, dev(self.row_start), self.Hq,
                                     self.Hkv, self.D, *where, dev(self.L), dev(self.n), self.window, self.sinks, self.scale, out)
        if check:
            assert ctx.cast_poll_status()[0] == 0
        return out

    def check(self, out, sample=400):
        """Within: half a step of the output; with bf16, half a step of every weight, which moves an output by sum_p w_p |v_p| of it (2^-8 of it;
        a weight in bf16 is off by 2^-9 of itself, and the cubic that forms a quarter of them by 2^-13.7); and in 32 bits: a score by D half steps of sum_d |q_d k_d|, its exponent in powers of two by 3 half steps of it (up to 1.5 times the score) and
        the exponential by 2^-21, so the weights by e, an output by 2 e sum_p w_p |v_p| (numerator and sum), and the sums over P positions
        by P half steps of the same."""
        got = out.double().cpu().numpy()
        x = self.q.double().cpu().numpy()
        sc, G = self.scale or self.D ** -0.5, self.Hq // self.Hkv
        touched = np.zeros(self.total, bool)
        for b in range(self.B):
            rows = self.rows_of(b)
            touched[rows] = True
            seen = self.seen(b)
            if len(rows) == 0:
                continue
            pick = np.arange(len(rows)) if len(rows) <= sample else np.unique(np.concatenate([[0, 1, len(rows) - 1], self.rng.integers(0, len(rows), sample)]))
            pg, sl = self.paged.at(b, np.arange(seen.shape[1]))
            for h in range(self.Hkv):
                k, v = (c[dev(pg).long(), dev(sl).long(), h].double().cpu().numpy() for c in (self.k, self.v))
                want, spread, size = co.attend(x[rows[pick], h * G:(h + 1) * G], k, v, seen[pick], sc)
                have = got[rows[pick], h * G:(h + 1) * G]
                np.testing.assert_array_equal(np.isnan(have), np.isnan(want))
                np.testing.assert_array_equal(have[np.isinf(want)], want[np.isinf(want)])
                e = (self.D + 5) * 2.0 ** -24 * size[..., None] + 2.0 ** -21
                tol = HALF[self.dtype] * np.abs(want) + ((HALF["bf16"] if self.dtype == "bf16" else 0) + 2 * e + seen.shape[1] * 2.0 ** -24) * spread
                with np.errstate(invalid="ignore"):
                    err = np.abs(have - want)
                bad = err > tol * 1.01 + 1e-30
                assert not bad.any(), (b, h, np.argwhere(bad)[0], err[bad][0], tol[bad][0], want[bad][0])
        assert np.isnan(got[~touched]).all()  # left as they were


CHUNKS = [  # dtype, Hq, Hkv, D, page, prefix lengths, new tokens, window, sinks, packed
    ("bf16", 32, 8, 128, 16, [70, 200, 0, 1], [1, 1, 1, 1], 0, 0, False),         # one token each
    ("bf16", 4, 4, 64, 0, [63, 64, 65, 127], [1, 65, 64, 1], 0, 0, False),
    ("bf16", 28, 4, 128, 24, [300, 0, 129, 511], [33, 130, 0, 18], 0, 0, True),
    ("bf16", 14, 2, 64, 1, [5, 17, 40], [20, 1, 3], 0, 0, False),
    ("bf16", 16, 2, 128, 64, [900, 1], [128, 300], 0, 0, True),
    ("bf16", 32, 8, 128, 0, [0], [1000], 0, 0, False),                             # a prompt
    ("bf16", 8, 1, 128, 128, [2048, 77], [1, 260], 0, 0, False),
    ("bf16", 8, 8, 128, 8, [1000, 31, 0, 2, 400, 7], [1, 2, 3, 0, 200, 5], 0, 0, True),
    ("bf16", 130, 1, 64, 16, [90], [3], 0, 0, False),
    ("bf16", 6, 2, 128, 256, [255, 256, 257], [1, 1, 300], 0, 0, False),
    ("bf16", 32, 8, 128, 16, [700, 0, 90, 1500], [1, 300, 40, 1], 100, 4, True),   # a window and sinks
    ("bf16", 8, 2, 64, 8, [700, 0, 90, 1500], [70, 300, 40, 1], 128, 130, False),  # sinks past a tile
    ("bf16", 4, 1, 128, 48, [400, 3], [200, 500], 1, 0, False),                    # every row sees itself alone
    ("bf16", 4, 4, 64, 32, [300, 600], [200, 10], 37, 0, True),
    ("bf16", 16, 2, 128, 16, [3000, 100], [64, 64], 700, 1, False),
    ("bf16", 8, 4, 128, 0, [260, 10], [300, 1], 256, 1000, False),                 # more sinks than positions
    ("f32", 8, 8, 64, 24, [300, 1111, 0], [33, 1, 5], 0, 0, False),
    ("f32", 6, 2, 128, 0, [64, 1, 200], [9, 100, 1], 0, 0, True),
    ("f32", 8, 2, 64, 16, [500, 40, 900], [1, 100, 30], 64, 3, False),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,L,n,window,sinks,packed", CHUNKS)
def test_chunk(binding, dtype, Hq, Hkv, D, page, L, n, window, sinks, packed):
    x = Batch(Hq * 100 + sum(n), dtype, Hq, Hkv, D, page, L, n, window, sinks, packed)
    out = x.run(binding)
    x.check(out)
    assert torch.equal(out.view(torch.uint8), x.run(binding).view(torch.uint8))  # the same bits every time


TREES = [  # dtype, Hq, Hkv, D, page, prefix lengths, tokens, window, sinks
    ("bf16", 32, 8, 128, 16, [2048], [60], 512, 4),
    ("bf16", 8, 2, 128, 16, [70, 900, 0, 1], [12, 3, 12, 7], 64, 4),
    ("bf16", 28, 4, 128, 24, [300, 0, 129, 511], [96, 20, 0, 96], 200, 0),
    ("bf16", 4, 4, 64, 0, [63, 64, 65, 640], [7, 7, 1, 7], 3, 1),     # ancestors fall out of the window
    ("bf16", 64, 8, 128, 32, [0, 700], [128, 128], 2, 5),             # and among the sinks
    ("bf16", 32, 8, 64, 16, [1000, 200, 30], [40, 1, 12], 0, 0),      # no window
    ("bf16", 7, 7, 128, 1, [400, 20], [33, 5], 130, 10),
    ("f32", 8, 8, 64, 24, [300, 1111, 0], [33, 10, 33], 100, 2),
    ("f32", 6, 2, 128, 0, [64, 1, 200], [9, 9, 9], 4, 0),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,L,n,window,sinks", TREES)
def test_tree_window(binding, dtype, Hq, Hkv, D, page, L, n, window, sinks):
    x = Batch(Hq * 100 + sum(n), dtype, Hq, Hkv, D, page, L, n, window, sinks, tree=True)
    out = x.run(binding)
    x.check(out)
    assert torch.equal(out.view(torch.uint8), x.run(binding).view(torch.uint8))
    first = np.minimum(n, [3, 0, 50, 1, 2][:len(n)])  # a layer of a growing tree
    y = Batch(Hq * 100 + sum(n), dtype, Hq, Hkv, D, page, L, n, window, sinks, tree=True, first=first)
    y.check(y.run(binding))


@pytest.mark.parametrize("seed", range(16))
def test_mixes(binding, seed):
    """Prompts, single tokens, empty sequences and trees side by side, windows and sinks anywhere within a tile, and the same bits again."""
    rng = np.random.default_rng(1000 + seed)
    tree = seed % 4 == 3
    D, G, Hkv = int(rng.choice([64, 128])), int(rng.choice([1, 3, 4, 7, 8, 16])), int(rng.choice([1, 2, 8, 24]))
    B, page = int(rng.integers(1, 9)), int(rng.choice([0, 8, 16, 24, 40, 128]))
    n = np.where(rng.random(B) < 0.4, rng.integers(0, 2, B), rng.integers(2, 125 if tree else 400, B))
    n[rng.integers(0, B)] = max(1, int(n.max()))
    L = rng.integers(0, 600, B) * rng.integers(0, 4, B)
    window, sinks = (int(rng.integers(1, 500)), int(rng.integers(0, 200))) if seed % 3 else (0, 0)
    x = Batch(seed, "bf16", G * Hkv, Hkv, D, page, L.tolist(), n.tolist(), window, sinks, packed=seed % 2 == 0 and not tree, tree=tree)
    out = x.run(binding)
    x.check(out, sample=60)
    assert torch.equal(x.run(binding).view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("G,Hkv,D,n,page", [(128, 1, 128, 3, 16), (100, 2, 64, 2, 136), (43, 4, 128, 50, 384), (5, 40, 64, 70, 512), (16, 148, 128, 9, 8),
                                            (127, 3, 128, 1, 0), (1, 75, 64, 300, 0), (64, 1, 128, 200, 1000)])
@pytest.mark.parametrize("tree", [False, True])
def test_groups_and_pages(binding, G, Hkv, D, n, page, tree):
    """Groups that fill a block of rows or leave most of it empty, more kv-heads than SMs, pages around and above a tile."""
    n = min(n, 128) if tree else n
    x = Batch(G * 7 + n, "bf16", G * Hkv, Hkv, D, page, [333, 0], [n, max(1, n // 2)], 150, 5, tree=tree)
    x.check(x.run(binding), sample=12)


@pytest.mark.parametrize("lo", [0, 1, 63, 64, 65, 127])
@pytest.mark.parametrize("length,sinks", [(64, 0), (65, 64), (300, 65), (1, 300)])
def test_edges_of_half_tiles(binding, lo, length, sinks):
    """The window's first position, the sinks' and the chunk's last in each half of a tile, for two blocks of rows that share their tiles."""
    window = 100
    x = Batch(lo + length, "bf16", 160, 40, 128, 16, [window - 1 + 256 + lo - length % 64] * 2, [length] * 2, window, sinks)
    x.check(x.run(binding), sample=40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("scale,spread", [(0.4, 1.0), (3.0, 2.0), (-0.5, 1.0), (1e-30, 1.0)])
def test_scales(binding, dtype, tree, scale, spread):
    """Scores far from zero, and turned around."""
    x = Batch(7, dtype, 8, 2, 128, 16, [300, 5, 131], [70, 20, 1], 90 if tree else 0, 2, tree=tree, scale=scale, spread=spread)
    x.check(x.run(binding))


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("n", [1, 200])
def test_scores_that_climb(binding, dtype, D, n):
    """Keys that grow along the sequence by hundreds, and fall again: the running reference has to follow both ways."""
    for sign in (1, -1):
        x = Batch(3, dtype, 4, 2, D, 0, [1500, 700], [n, n])
        ramp = torch.linspace(-12, 12, x.k.shape[1], device="cuda")[None, :, None, None] * sign
        x.q[..., 0] = 20.0
        x.k[..., 0] = (ramp * torch.ones_like(x.k[..., :1]))[..., 0].to(x.k.dtype)
        x.poison()
        x.check(x.run(binding))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("G,n", [(1, 90), (4, 90), (8, 5)])
def test_values_without_a_number_reach_only_who_sees_them(binding, dtype, tree, G, n):
    """NaN and infinities in single dims of values of the prefix's edge, of new tokens and of the window's first positions."""
    x = Batch(5, dtype, 2 * G, 2, 128, 16, [333, 0, 1000], [n, n, n], 120, 3, tree=tree)
    for b in range(3):
        for i, at in enumerate((int(x.L[b]) + n // 2, int(x.L[b]) + n - 1, max(0, int(x.L[b]) - 119 + n // 3))):
            pg, sl = x.paged.at(b, np.array(at))
            x.v[int(pg), int(sl), i % 2, 5 + i] = POISON[(i + b) % 3]
    x.check(x.run(binding))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 100])
def test_nan_queries_and_keys(binding, dtype, n):
    """A query row of NaN gives NaN, and no other row does; a key of NaN gives NaN to the rows that see it."""
    x = Batch(9, dtype, 8, 2, 128, 16, [700, 40], [n, n])
    clean = x.run(binding)
    x.q[x.row0[0] + n // 2, 3] = float("nan")
    pg, sl = x.paged.at(1, np.array(40 + n // 2))
    x.k[int(pg), int(sl), 1, 7] = float("nan")
    out = x.run(binding)
    want = clean.clone()
    want[x.row0[0] + n // 2, 3] = float("nan")
    want[x.row0[1] + n // 2:, 4:] = float("nan")
    assert torch.equal(torch.isnan(out), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(out[ok], clean[ok])


@pytest.mark.parametrize("dtype,Hq,Hkv,D", [("bf16", 32, 8, 128), ("bf16", 8, 8, 64), ("f32", 4, 4, 64)])
def test_many_ragged_sequences(binding, dtype, Hq, Hkv, D):
    """More items than thread blocks, pieces of items on several, sequences without work, prompts beside single tokens."""
    rng = np.random.default_rng(1)
    L, n = rng.integers(0, 900, 64), rng.integers(0, 4, 64)
    n[:6] = [150, 0, 33, 1, 70, 300]
    L[3:5] = [3000, 0]
    x = Batch(2, dtype, Hq, Hkv, D, 16, L, n, packed=True)
    x.check(x.run(binding))
    y = Batch(2, dtype, Hq, Hkv, D, 16, L, n, 200, 5, packed=True)
    y.check(y.run(binding))
    z = Batch(2, dtype, Hq, Hkv, D, 16, L, np.minimum(n, 100), 200, 5, tree=True)
    z.check(z.run(binding))


def test_one_long_sequence_over_all_blocks(binding):
    """A token over 40 000 positions: partial results of every thread block meet."""
    for dtype, Hkv in (("bf16", 1), ("bf16", 8), ("f32", 1)):
        x = Batch(4, dtype, 4 * Hkv, Hkv, 128, 16, [40000], [1])
        x.check(x.run(binding))


def test_no_work(binding):
    for tree in (False, True):
        x = Batch(4, "bf16", 8, 2, 128, 16, [50, 0], [0, 0], tree=tree, window=5)
        assert bool(torch.isnan(x.run(binding)).all())


def test_a_row_that_sees_nothing_gives_zeros(binding):
    x = Batch(6, "bf16", 4, 2, 128, 16, [0, 0], [5, 40], tree=True)
    y = Batch(6, "f32", 4, 2, 128, 16, [0, 0], [5, 40], tree=True)
    for z in (x, y):
        z.anc[1, 7:9] = 0
        out = z.run(binding)
        assert bool((out[z.row0[1] + 7:z.row0[1] + 9] == 0).all())
        z.tree[1][7:9] = False
        z.check(out)


def test_counts_and_places_out_of_range(binding):
    """Counts past the buffer are cut, rows outside it leave their sequence out, positions past the capacity are not seen; each is
    reported, and the other sequences come out as they do alone."""
    for dtype in ("bf16", "f32"):
        x = Batch(8, dtype, 8, 2, 128, 16, [40, 100, 9], [20, 20, 20])
        good = x.run(binding)
        ctx = binding.CastContext(max_batch=3, vocab=1000, top_k=4, max_depth=6, total_token=8, max_tree=8)
        n = x.n
        x.n = np.array([20, 25, 20], np.int32)  # rows is 20: cut, and no error (as for the append)
        assert torch.equal(x.run(binding, ctx), good)
        x.n = np.array([20, -4, 20], np.int32)
        out = x.run(binding, ctx)
        assert torch.equal(out[:20], good[:20]) and torch.equal(out[40:], good[40:]) and bool(torch.isnan(out[20:40]).all())
        x.n = n
        for start in ([0, 41, 40], [0, -1, 40]):
            x.row_start = np.array(start, np.int32)
            out = x.run(binding, ctx, check=False)
            assert ctx.cast_poll_status() == (6, 1)
            assert torch.equal(out[:20], good[:20]) and torch.equal(out[40:], good[40:]) and bool(torch.isnan(out[20:40]).all())
        x.row_start = None
        keep = x.L.copy()
        for past in (x.paged.positions - 5, x.paged.positions, 2 ** 31 - 1):
            x.L = keep.copy()
            x.L[1] = past
            x.table = x.paged.table
            out = x.run(binding, ctx, check=False)
            assert ctx.cast_poll_status() == (7, 1)
            assert torch.equal(out[:20], good[:20]) and torch.equal(out[40:], good[40:])
        x.L = keep
        x.table = x.paged.table.copy()
        x.table[1, 3] = x.paged.pages
        out = x.run(binding, ctx, check=False)
        assert ctx.cast_poll_status() == (7, 1)
        assert torch.equal(out[:20], good[:20]) and torch.equal(out[40:], good[40:])


def test_refusals(binding):
    ctx = binding.CastContext(max_batch=2, vocab=1000, top_k=4, max_depth=6, total_token=4, max_tree=4)
    B, rows, Hq, Hkv, D = 2, 4, 4, 2, 64
    q, k = torch.randn((B, rows, Hq, D), device="cuda"), torch.randn((B, 16, Hkv, D), device="cuda")
    i2 = dev(np.zeros(2, np.int32))
    base = dict(q=q, k=k, v=k, B=B, rows=rows, Hq=Hq, Hkv=Hkv, D=D, page=0, table=None, cap=16, pages=0, kv_len=i2, n=i2, window=0, sinks=0, out=q.clone(),
                anc=torch.zeros((B, rows, 1), dtype=torch.int32, device="cuda"), depth=torch.zeros((B, rows), dtype=torch.int32, device="cuda"))

    def call(tree, **kw):
        a = {**base, **kw}
        where = (a["page"], a["table"], a["cap"], a["pages"], a["kv_len"])
        if tree:
            ctx.cast_tree_attention_window(a["q"], a["k"], a["v"], a["B"], a["Hq"], a["Hkv"], a["D"], *where, a["anc"], a["depth"], a["n"], None,
                                           a["window"], a["sinks"], 0.0, a["out"])
        else:
            ctx.cast_chunk_attention(a["q"], a["k"], a["v"], a["B"], a["rows"], None, a["Hq"], a["Hkv"], a["D"], *where, a["n"], a["window"], a["sinks"],
                                     0.0, a["out"])

    for tree in (False, True):
        with pytest.raises(binding.CastError) as e:  # nothing reserved
            call(tree)
        assert e.value.code == 3
    for bad, code in (((torch.float32, 32), 2), ((torch.bfloat16, 256), 2)):
        with pytest.raises(binding.CastError) as e:
            ctx.cast_reserve_chunk_attention(*bad)
        assert e.value.code == code
    ctx.cast_reserve_chunk_attention(torch.float32, D)
    b16 = {w: base[w].bfloat16() for w in ("q", "k", "v", "out")}
    for tree in (False, True):
        call(tree)
        for code, kw in ((1, dict(kv_len=None)), (1, dict(n=None)), (1, dict(window=-1)), (1, dict(sinks=-1)), (1, dict(B=0)), (1, dict(cap=0)),
                         (1, dict(page=16)), (1, dict(page=-1)), (2, dict(Hkv=3)), (2, dict(D=32)), (3, dict(B=3)), (3, dict(cap=2 ** 31 - 1)),
                         (3, dict(page=1 << 20, table=i2, cap=1 << 20, pages=1)), (4, dict(k=k.bfloat16())), (4, dict(out=q.bfloat16())),
                         (4, dict(q=q.half(), k=k.half(), v=k.half(), out=q.half()))):
            with pytest.raises(binding.CastError) as e:
                call(tree, **kw)
            assert e.value.code == code, (tree, kw, e.value)
    for code, kw in ((1, dict(rows=0)), (3, dict(rows=1 << 30))):
        with pytest.raises(binding.CastError) as e:
            call(False, **kw)
        assert e.value.code == code
    for kw in (dict(anc=None), dict(depth=None)):
        with pytest.raises(binding.CastError) as e:
            call(True, **kw)
        assert e.value.code == 1
    flat = torch.zeros(q.numel() + 1, device="cuda")
    with pytest.raises(binding.CastError) as e:  # not aligned to 16 bytes
        call(False, out=flat[1:])
    assert e.value.code == 2
    with pytest.raises(binding.CastError) as e:  # the workspace of fp32 calls is not that of bf16 calls
        call(False, **b16)
    assert e.value.code == 3
    assert ctx.cast_poll_status()[0] == 0


def test_rows_past_32_bits(binding):
    """Pages, and a run of positions, more than 2^32 elements from the cache's beginning: the same bits as in a small cache."""
    for dtype in ("bf16", "f32"):
        x = Batch(12, dtype, 8, 2, 128, 16, [300, 77], [40, 1])
        good = x.run(binding)
        pages = (1 << 32) // (16 * 2 * 128) + x.paged.pages
        far = [torch.zeros((pages, 16, 2, 128), dtype=DT[dtype], device="cuda") for _ in range(2)]
        for big, small in zip(far, (x.k, x.v)):
            big[pages - x.paged.pages:] = small
        live = (x.table >= 0) & (x.table < x.paged.pages)
        x.table = np.where(live, x.table.astype(np.int64) + pages - x.paged.pages, -1).astype(np.int32)
        x.k, x.v = far
        x.paged.pages = pages
        assert torch.equal(x.run(binding).nan_to_num(nan=7.0), good.nan_to_num(nan=7.0))
        del far, x
        torch.cuda.empty_cache()


def test_another_stream_and_a_captured_graph(binding):
    for tree in (False, True):
        x = Batch(21, "bf16", 32, 8, 128, 16, [900, 40, 0], [40, 1, 40], 300, 4, tree=tree)
        good = x.run(binding)
        tokens = x.rows if tree else 8
        ctx = binding.CastContext(max_batch=3, vocab=1000, top_k=4, max_depth=6, total_token=tokens, max_tree=tokens)
        ctx.cast_reserve_chunk_attention(torch.bfloat16, 128)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            out = x.run(binding, ctx)
        side.synchronize()
        assert torch.equal(out.view(torch.int16), good.view(torch.int16))
        args = (8, 128, 16, dev(x.table), x.paged.cap, x.paged.pages, dev(x.L))
        ints = [dev(a) for a in ((x.anc.view(np.int32), x.depth, x.n) if tree else (x.n,))]
        out = torch.full_like(x.q, float("nan"))

        def call():
            if tree:
                ctx.cast_tree_attention_window(x.q, x.k, x.v, 3, 32, *args, *ints, None, 300, 4, 0.0, out)
            else:
                ctx.cast_chunk_attention(x.q, x.k, x.v, 3, x.rows, None, 32, *args, *ints, 300, 4, 0.0, out)

        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            call()
            call()
        for _ in range(3):
            out.fill_(float("nan"))
            g.replay()
            assert torch.equal(out.view(torch.int16), good.view(torch.int16))
        ints[-1].fill_(1)  # sizes are read when the graph runs
        out.fill_(float("nan"))
        g.replay()
        assert torch.equal(torch.isnan(out).any(-1).any(-1).view(3, -1)[:, 1:], torch.ones((3, x.rows - 1), dtype=torch.bool, device="cuda"))
        assert not bool(torch.isnan(out.view(3, x.rows, 32, 128)[:, 0]).any())
        assert ctx.cast_poll_status()[0] == 0


@pytest.mark.parametrize("dtype,window", [("bf16", 0), ("bf16", 100), ("f32", 48)])
def test_a_prompt_in_chunks_then_trees(binding, dtype, window):
    """A program's run: a prompt appended and attended chunk by chunk (each row against the whole sequence so far, in 64 bits), then a
    verification step under the window on the same cache: rows appended at their depths, attention, acceptance, compaction, and a
    decoding step on what is kept."""
    rng = np.random.default_rng(17)
    B, Hq, Hkv, D, page, tokens, sinks, rot = 2, 8, 2, 128, 16, 12, 3, 96
    total, cap = 300, 24
    ctx = binding.CastContext(max_batch=B, vocab=1000, top_k=4, max_depth=6, total_token=tokens, max_tree=tokens)
    ctx.cast_reserve_chunk_attention(DT[dtype], D)
    paged = o4.Paged(rng, B, cap * page, page)
    where = (page, dev(paged.table), paged.cap, paged.pages)
    kc, vc = (torch.full((paged.pages, page, Hkv, D), float("nan"), device="cuda").to(DT[dtype]) for _ in range(2))
    inv = 10000.0 ** (-np.arange(0, rot, 2) / rot)
    w = [dev((1 + 0.3 * rng.normal(size=D)).astype(np.float32)) for _ in range(2)]
    kv_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    hist_k, hist_v = [np.zeros((0, Hkv, D))] * B, [np.zeros((0, Hkv, D))] * B
    gen = torch.Generator("cuda").manual_seed(1)

    def rows_of(n):
        return torch.randn((B, n, (Hq + 2 * Hkv) * D), generator=gen, device="cuda").to(DT[dtype])

    def append(x, n, depth, q_out):
        q, k, v = x.split([Hq * D, Hkv * D, Hkv * D], -1)
        stride = x.stride(1) * x.element_size()
        ctx.cast_append_kv(q.unflatten(-1, (Hq, D)), stride, k.unflatten(-1, (Hkv, D)), stride, v.unflatten(-1, (Hkv, D)), stride, B, x.shape[1], Hq, Hkv, D,
                           None, None, n, depth, None, dev(inv), rot, 0, 0.0, *w, 1e-6, *where, kv_len, q_out, kc, vc)

    def read(b, start, n):  # what the cache holds now, so that a test of the attention is one of the attention
        pg, sl = (dev(a).long() for a in paged.at(b, start + np.arange(n)))
        return kc[pg, sl].double().cpu().numpy(), vc[pg, sl].double().cpu().numpy()

    def check(out, q, b, n, stands, tree=None):
        L = len(hist_k[b])
        nk, nv = read(b, L, n)
        k, v = np.concatenate([hist_k[b], nk]), np.concatenate([hist_v[b], nv])
        seen = co.sight(L, stands, window, sinks, tree)
        G = Hq // Hkv
        for h in range(Hkv):
            want, spread, size = co.attend(q[b, :n, h * G:(h + 1) * G].double().cpu().numpy(), k[:, h], v[:, h], seen, D ** -0.5)
            err = np.abs(out[b, :n, h * G:(h + 1) * G].double().cpu().numpy() - want)
            e = (D + 5) * 2.0 ** -24 * size[..., None] + 2.0 ** -21
            tol = HALF[dtype] * np.abs(want) + ((HALF["bf16"] if dtype == "bf16" else 0) + 2 * e + len(k) * 2.0 ** -24) * spread
            assert (err <= tol * 1.01).all(), (b, h, err.max())
        return nk, nv

    done = 0
    while done < total:
        n = min(int(rng.choice([1, 37, 64, 130])), total - done)
        x = rows_of(n)
        q, out = torch.zeros((B, n, Hq, D), device="cuda").to(DT[dtype]), torch.zeros((B, n, Hq, D), device="cuda").to(DT[dtype])
        counts = dev(np.full(B, n, np.int32))
        append(x, counts, None, q)
        ctx.cast_chunk_attention(q, kc, vc, B, n, None, Hq, Hkv, D, *where, kv_len, counts, window, sinks, 0.0, out)
        for b in range(B):
            nk, nv = check(out, q, b, n, done + np.arange(n))
            want, pair = co.rotated(co.normalised(x[b, :, Hq * D:(Hq + Hkv) * D].double().cpu().numpy().reshape(n, Hkv, D), w[1].cpu().numpy(), 1e-6),
                                    done + np.arange(n), inv, False, 1.0), None
            assert np.abs(nk - want).max() < (HALF[dtype] + 2.0 ** -17) * 2 * np.abs(want).max()
            hist_k[b], hist_v[b] = np.concatenate([hist_k[b], nk]), np.concatenate([hist_v[b], nv])
        kv_len += n
        done += n
    # a verification step
    parent = np.array([-1, 0, 0, 1, 1, 2, 3, 3, 5, 6, 6, 8])
    depth = np.zeros(tokens, np.int32)
    vis = np.eye(tokens, dtype=bool)
    for t in range(1, tokens):
        depth[t] = depth[parent[t]] + 1
        vis[t] |= vis[parent[t]]
    anc = (vis * (1 << np.arange(tokens))).sum(-1).astype(np.int32)
    x = rows_of(tokens)
    q, out = torch.zeros((B, tokens, Hq, D), device="cuda").to(DT[dtype]), torch.zeros((B, tokens, Hq, D), device="cuda").to(DT[dtype])
    d2, n2 = dev(np.tile(depth, (B, 1))), dev(np.full(B, tokens, np.int32))
    append(x, n2, d2, q)
    ctx.cast_tree_attention_window(q, kc, vc, B, Hq, Hkv, D, *where, kv_len, dev(np.tile(anc[:, None], (B, 1, 1))), d2, n2, None, window, sinks, 0.0, out)
    rows = [check(out, q, b, tokens, total + depth, vis) for b in range(B)]
    path = np.full((B, 7), -1, np.int32)
    path[0, :5], path[1, :3] = [0, 1, 3, 6, 9], [0, 2, 5]
    alen = np.array([4, 2], np.int32)
    ctx.cast_compact_kv(kc, vc, B, 1, kc.numel() * kc.element_size(), Hkv, D, *where, dev(path), dev(alen), kv_len)
    for b in range(B):
        nodes = path[b, :alen[b] + 1]
        nk, nv = read(b, total, len(nodes))
        np.testing.assert_array_equal(nk, rows[b][0][nodes])  # rotated by depth: the places they have moved to are their positions
        hist_k[b], hist_v[b] = np.concatenate([hist_k[b], nk]), np.concatenate([hist_v[b], nv])
    assert kv_len.tolist() == [total + 5, total + 3]
    x = rows_of(1)
    q, out = torch.zeros((B, 1, Hq, D), device="cuda").to(DT[dtype]), torch.zeros((B, 1, Hq, D), device="cuda").to(DT[dtype])
    one = dev(np.ones(B, np.int32))
    append(x, one, None, q)
    ctx.cast_chunk_attention(q, kc, vc, B, 1, None, Hq, Hkv, D, *where, kv_len, one, window, sinks, 0.0, out)
    for b in range(B):
        check(out, q, b, 1, np.array([len(hist_k[b])]))
    assert ctx.cast_poll_status()[0] == 0
