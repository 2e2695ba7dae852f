"""cast_chunk_attention and cast_tree_attention_window where windows, sinks and capacities meet: against 64 bits, and the same bits again."""
import numpy as np
import pytest
import torch

from test_gpu_chunk_attention import Batch, binding  # noqa: F401  (the fixture)

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
