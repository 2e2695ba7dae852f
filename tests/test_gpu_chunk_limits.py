"""cast_chunk_attention and cast_tree_attention_window where windows, sinks and capacities meet: against 64 bits, and the same bits again."""
import numpy as np
import pytest
import torch

import chunk_oracle as co
from test_gpu_chunk_attention import HALF, Batch, binding, dev  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


class Tree(Batch):
    """The same over given trees: parents[b][t] is the parent of token t of sequence b."""

    def __init__(self, seed, dtype, Hq, Hkv, D, page, L, parents, window, sinks, first):
        self.parents = parents
        super().__init__(seed, dtype, Hq, Hkv, D, page, L, [len(x) for x in parents], window, sinks, tree=True, first=first)

    def poison(self):
        self.anc[:], self.depth[:] = 0, -1
        for b, parent in enumerate(self.parents):
            vis = np.eye(len(parent), dtype=bool)
            for t, at in enumerate(parent):
                self.depth[b, t] = 0 if at < 0 else self.depth[b, at] + 1
                if at >= 0:
                    vis[t] |= vis[at]
                for j in np.flatnonzero(vis[t]):
                    self.anc[b, t, j >> 5] |= np.uint32(1 << (j & 31))
            self.tree[b] = vis
        super().poison()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sinks_among_a_trees_tokens_under_a_later_window(binding, dtype):  # noqa: F811
    """Row 7 stands at 1 + 5 and sees, under a window of 3, what stands at 4 or later, and the sinks 0, 1 and 2: token 2 stands at 2, but
    lies at place 3, behind the sinks' places and before the window's."""
    x = Tree(3, dtype, 4, 2, 64, 16, [1], [[-1, 0, 0, 2, 2, 4, 5, 6]], 3, 3, [7])
    assert x.seen(0)[0].tolist() == [True, True, False, True, False, False, True, True, True]
    out = x.run(binding)
    x.check(out)
    assert torch.equal(out.view(torch.uint8), x.run(binding).view(torch.uint8))


@pytest.mark.parametrize("seed", range(8))
def test_deep_trees_later_rows_short_windows(binding, seed):  # noqa: F811
    """Trees deeper than the window whose first tokens are sinks, output rows far down."""
    rng = np.random.default_rng(70 + seed)
    sinks, D, G = int(rng.integers(1, 200)), [64, 128][seed % 2], [1, 4, 8, 3][seed % 4]
    L, parents, first = [], [], []
    for _ in range(6):
        n = int(rng.integers(8, 120))
        L.append(max(0, sinks - int(rng.integers(0, 6))))
        parents.append([-1] + [int(rng.integers(max(0, t - 3), t)) for t in range(1, n)])
        first.append(int(rng.integers(n // 2, n)))
    x = Tree(seed, "f32" if seed % 4 == 3 else "bf16", 2 * G, 2, D, [16, 0, 24, 8][seed % 4], L, parents, int(rng.integers(1, 6)), sinks, first)
    x.check(x.run(binding))


class Past(Batch):
    """The same in a cache that ends at position `cut`, before some sequences do: what lies behind it is not seen."""

    def __init__(self, cut, *args, **kw):
        self.cut = cut
        super().__init__(*args, **kw)
        p = self.paged
        p.positions = cut
        if self.page:
            assert cut % self.page == 0
            p.cap = cut // self.page
            p.table, self.table = p.table[:, :p.cap], self.table[:, :p.cap]
        else:
            p.cap, p.shape = cut, (self.B, cut)
            self.k, self.v = self.k[:, :cut].contiguous(), self.v[:, :cut].contiguous()

    def seen(self, b):
        return super().seen(b)[:, :self.cut]

    def attend(self, binding):
        tokens = self.rows if self.tree is not None else 8
        ctx = binding.CastContext(max_batch=self.B, vocab=1000, top_k=4, max_depth=6, total_token=tokens, max_tree=tokens)
        outs = []
        for _ in range(2):
            outs.append(self.run(binding, ctx, check=False))
            status, b = ctx.cast_poll_status()
            assert status == 7 and self.L[b] + self.n[b] > self.cut
        assert torch.equal(outs[0].view(torch.uint8), outs[1].view(torch.uint8))
        return outs[0]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,cut,L,n,window,sinks,packed", [
    ("bf16", 32, 8, 128, 16, 192, [100, 50, 128, 10], [512, 60, 1, 100], 64, 0, False),   # the capacity in the middle of a tile
    ("bf16", 32, 8, 128, 64, 320, [300, 0, 200, 319], [500, 320, 100, 40], 100, 0, True),
    ("bf16", 16, 16, 64, 8, 128 * 3 + 8, [380, 100, 0, 391], [300, 290, 10, 1], 33, 4, False),
    ("bf16", 8, 8, 128, 0, 190, [100, 0, 189, 5], [400, 189, 300, 1], 65, 130, False),
    ("bf16", 8, 8, 64, 0, 256 + 64, [100, 0, 189, 300], [400, 300, 400, 90], 1, 3, True),
    ("bf16", 28, 4, 128, 16, 128, [100, 127, 64], [30, 5, 600], 64, 0, False),
    ("f32", 4, 2, 64, 16, 96, [70, 10, 95], [60, 40, 9], 20, 2, False),
    ("f32", 4, 2, 128, 0, 100, [90, 10, 95], [130, 40, 9], 32, 0, True),
])
def test_chunks_past_the_capacity_under_a_window(binding, dtype, Hq, Hkv, D, page, cut, L, n, window, sinks, packed):  # noqa: F811
    """Rows whose windows begin behind the capacity see the sinks alone, or nothing and give zeros; every other row what it should."""
    x = Past(cut, cut, dtype, Hq, Hkv, D, page, L, n, window, sinks, packed)
    out = x.attend(binding)
    x.check(out)
    for b in range(x.B):
        blind = x.rows_of(b)[~x.seen(b).any(1)]
        assert bool((out[blind] == 0).all())


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,cut,L,n,window,sinks", [
    ("bf16", 8, 2, 128, 16, 160, [150, 100, 160, 155], [40, 60, 12, 5], 0, 0),    # some tokens of the tree, all, one
    ("bf16", 8, 8, 64, 0, 100, [95, 0, 100, 30], [10, 100, 7, 90], 0, 0),         # the next sequence's rows lie behind
    ("bf16", 64, 8, 128, 24, 192, [191, 190, 10], [64, 20, 3], 7, 3),
    ("bf16", 28, 4, 64, 8, 64, [60, 40, 3], [90, 70, 2], 2, 70),
    ("bf16", 32, 8, 128, 16, 96, [96, 110, 200, 20], [12, 30, 9, 4], 40, 0),      # the prefix itself past the capacity
    ("f32", 4, 2, 64, 16, 96, [90, 60, 120], [20, 40, 9], 0, 0),
    ("f32", 4, 2, 128, 0, 100, [90, 110, 95], [20, 40, 3], 32, 5),
])
def test_trees_past_the_capacity(binding, dtype, Hq, Hkv, D, page, cut, L, n, window, sinks):  # noqa: F811
    x = Past(cut, cut + window, dtype, Hq, Hkv, D, page, L, n, window, sinks, tree=True)
    x.check(x.attend(binding))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,window,sinks", [(16, 60, 0), (0, 60, 5), (16, 0, 0), (0, 1000, 0)])
def test_a_prefix_past_the_capacity_keeps_its_windows(binding, dtype, page, window, sinks):  # noqa: F811
    """Rows at kv_len + t, wherever the cache ends: a window of 60 from position 230 on reaches back to 171 and no further."""
    x = Past(192, 5, dtype, 8, 2, 128, page, [230, 100, 192, 700], [20, 40, 33, 3], window, sinks)
    x.check(x.attend(binding))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree", [False, True])
def test_lengths_up_to_the_largest_int(binding, dtype, tree):  # noqa: F811
    for window in (0, 50, 2 ** 31 - 1):
        x = Batch(4, dtype, 8, 2, 128, 16, [100, 60, 9], [20, 20, 20], window, tree=tree)
        x.table = x.paged.table  # (every entry is looked at below)
        x.k.nan_to_num_(nan=1.0, posinf=2.0, neginf=3.0)
        x.v.nan_to_num_(nan=1.0, posinf=2.0, neginf=3.0)
        good = x.run(binding)
        x.L[1] = 2 ** 31 - 1
        ctx = binding.CastContext(max_batch=3, vocab=1000, top_k=4, max_depth=6, total_token=20, max_tree=20)
        out = x.run(binding, ctx, check=False)
        assert ctx.cast_poll_status() == (7, 1)
        assert torch.equal(out[:20], good[:20]) and torch.equal(out[40:], good[40:])
        mine = out[20:40]
        assert bool(torch.isfinite(mine).all())
        if window == 50:
            assert bool((mine == 0).all())
        if window == 0:  # every row sees the whole cache; the tolerance is Batch.check's
            pos = np.arange(x.paged.positions)
            pg, sl = (dev(a).long() for a in x.paged.at(1, pos))
            for h in range(2):
                k, v = (c[pg, sl, h].double().cpu().numpy() for c in (x.k, x.v))
                want, spread, size = co.attend(x.q[20:40, 4 * h:4 * h + 4].double().cpu().numpy(), k, v, np.ones((20, len(pos)), bool), 128 ** -0.5)
                e = 133 * 2.0 ** -24 * size[..., None] + 2.0 ** -21
                tol = HALF[dtype] * np.abs(want) + ((HALF["bf16"] if dtype == "bf16" else 0) + 2 * e + len(pos) * 2.0 ** -24) * spread
                assert (np.abs(mine[:, 4 * h:4 * h + 4].double().cpu().numpy() - want) <= tol * 1.01).all()


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("page", [2 ** 30 + 8, 2 ** 30 + 128, 2 ** 31 - 2 ** 16])
def test_pages_beyond_2_to_the_30(binding, page, tree):  # noqa: F811
    """One page per cache, of which a part is there and a part of that is read: as the same rows without pages."""
    x = Batch(6, "bf16", 8, 2, 64, 0, [200], [40], 60, 3, tree=tree)
    x.k, x.v = (torch.cat([c, c.new_full((1, 512, 2, 64), float("nan"))], 1) for c in (x.k, x.v))
    x.paged.cap = x.k.shape[1]
    good = x.run(binding)
    x.page, x.table, x.paged.cap, x.paged.pages = page, np.zeros((1, 1), np.int32), 1, 1
    assert torch.equal(x.run(binding).view(torch.int16), good.view(torch.int16))


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("score,size", [(37.25, 42), (37.25, -42), (-45.0, 42), (-45.0, -42)])
def test_values_of_any_size_that_is_promised(binding, tree, score, size):  # noqa: F811
    """Scores that keep a step's weights just within 2^60 of the reference (64 weights of 2^53.7, or of 2^-64.9, over 40 000 positions), and
    values of 2^42 and 2^-42."""
    x = Batch(8, "bf16", 4, 2, 64, 16, [40000, 300], [3, 40], 0, 0, tree=tree, scale=1.0)
    x.q[~torch.isnan(x.q)] = 0.0
    x.q[..., 0] = torch.where(torch.isnan(x.q[..., 0]), x.q[..., 0], torch.ones_like(x.q[..., 0]))
    x.k[..., 0] = score
    x.v *= 2.0 ** size
    x.poison()
    x.check(x.run(binding))


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("order", [1, -1])
def test_scores_of_any_size_that_is_promised(binding, dtype, D, tree, order):  # noqa: F811
    """Scores of 2^28 and -2^28, exact in 32 bits: the weights are equal among the largest that a row sees and zero elsewhere, also where
    all that it sees stands at -2^28."""
    x = Batch(9, dtype, 8, 2, D, 16, [500, 70, 300], [40, 30, 5], 0, 0, tree=tree, scale=1.0)
    x.q[~torch.isnan(x.q)] = 0.0
    x.q[..., 0] = torch.where(torch.isnan(x.q[..., 0]), x.q[..., 0], torch.full_like(x.q[..., 0], 2.0 ** 14))
    x.k.zero_()
    for b, (top, first, last) in enumerate(((2.0 ** 14, 100, 230), (-2.0 ** 14, 0, 100), (2.0 ** 14, 3, 4))):
        pos = np.arange(int(x.L[b] + x.n[b]))
        pg, sl = (dev(a).long() for a in x.paged.at(b, pos))
        inside = dev((pos >= first) & (pos < last))
        x.k[pg, sl, :, 0] = torch.where(inside, top, -2.0 ** 14 if order > 0 else 0.0).to(x.k.dtype)[:, None]
        x.v[pg, sl] = torch.randn((len(pos), 2, D), device="cuda").to(x.v.dtype)
    out = x.run(binding)
    got = out.double().cpu().numpy()
    for b in range(3):
        seen = x.seen(b)
        pos = np.arange(seen.shape[1])
        pg, sl = (dev(a).long() for a in x.paged.at(b, pos))
        s, v = x.k[pg, sl, 0, 0].double().cpu().numpy(), x.v[pg, sl].double().cpu().numpy()
        for r, row in enumerate(x.rows_of(b)):
            at = seen[r] & (s == s[seen[r]].max())
            want, spread = v[at].mean(0), np.abs(v[at]).mean(0)  # the tolerance: half a step of the output and of a weight, sums in 32 bits
            tol = HALF[dtype] * np.abs(want) + (HALF["bf16"] if dtype == "bf16" else 0) * spread + (len(pos) + 8) * 2.0 ** -24 * spread
            err = np.abs(got[row].reshape(2, 4, D) - want[:, None])
            assert (err <= tol[:, None] * 1.01).all(), (b, r, err.max())
