"""bf16 heads of 64 dims: the weights enter the product as two bf16 terms, so an output is the exact one rounded, but for what 32 bits lose."""
import numpy as np
import pytest
import torch

import chunk_oracle as co
from test_gpu_chunk_attention import Batch, binding, dev  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


def within(x, out):
    """Half a step of the output, of its own binade. A weight p of binade 2^e: its first term leaves less than 2^(e - 8) or is exact to a power of two,
    the second half a step of what is left, 2^(e - 17): 2^-17 of p at most. Its score: D half steps of sum_d |q_d k_d|, its exponential 2^-21 as in Batch.check,
    so outputs 2 e sum_p w_p |v_p|; sums over P positions P half steps."""
    got, q = out.double().cpu().numpy(), x.q.double().cpu().numpy()
    sc, G = x.scale or x.D ** -0.5, x.Hq // x.Hkv
    for b in range(x.B):
        rows, seen = x.rows_of(b), x.seen(b)
        if len(rows) == 0:
            continue
        pg, sl = (dev(a).long() for a in x.paged.at(b, np.arange(seen.shape[1])))
        for h in range(x.Hkv):
            k, v = (c[pg, sl, h].double().cpu().numpy() for c in (x.k, x.v))
            want, spread, size = co.attend(q[rows, h * G:(h + 1) * G], k, v, seen, sc)
            e = (x.D + 5) * 2.0 ** -24 * size[..., None] + 2.0 ** -21
            half = 2.0 ** (np.frexp(want)[1] - 9.0)
            tol = half + (2.0 ** -17 + 2 * e + seen.shape[1] * 2.0 ** -24) * spread
            err = np.abs(got[rows, h * G:(h + 1) * G] - want)
            assert (err <= tol).all(), (b, h, float((err > tol).mean()), float((err / tol).max()))


@pytest.mark.parametrize("Hq,Hkv,page,L,n,window,sinks,packed,tree", [
    (32, 8, 16, [70, 20, 0, 55], [1, 1, 40, 1], 0, 0, False, False),
    (8, 8, 0, [60, 0, 30], [1, 60, 33], 0, 0, False, False),
    (4, 1, 8, [0, 64], [100, 1], 20, 3, True, False),
    (96, 24, 16, [0, 10, 30, 5, 9], [90, 70, 80, 66, 90], 0, 0, True, False),   # pairs of row blocks
    (32, 8, 16, [60, 40], [30, 12], 0, 0, False, True),
    (64, 8, 24, [60, 5], [64, 20], 25, 2, False, True),
])
def test_outputs_are_the_exact_ones_rounded(binding, Hq, Hkv, page, L, n, window, sinks, packed, tree):  # noqa: F811
    x = Batch(sum(n), "bf16", Hq, Hkv, 64, page, L, n, window, sinks, packed, tree)
    out = x.run(binding)
    x.check(out)
    within(x, out)


def test_scores_that_move_the_reference(binding):  # noqa: F811
    """Sums beyond 2^60 and below 2^-60 of the first reference: steps that are formed again."""
    for scale, spread in ((1.0, 12.0), (2.0, 8.0)):
        x = Batch(11, "bf16", 8, 2, 64, 16, [60, 33], [40, 1], scale=scale, spread=spread)
        out = x.run(binding)
        x.check(out)
        within(x, out)


def test_without_a_window_as_precise_as_the_tree_attention(binding):  # noqa: F811
    x = Batch(5, "bf16", 32, 8, 64, 16, [70, 9, 31], [24, 24, 24], tree=True)
    within(x, x.run(binding))
    ctx = binding.CastContext(max_batch=3, vocab=1000, top_k=4, max_depth=6, total_token=24, max_tree=24)
    ctx.cast_reserve_attention(torch.bfloat16, 3, 32, 8, 64, 16, x.paged.cap)
    out = torch.full_like(x.q, float("nan"))
    x.k.nan_to_num_(nan=0.0, posinf=0.0, neginf=0.0)
    x.v.nan_to_num_(nan=0.0, posinf=0.0, neginf=0.0)
    ctx.cast_tree_attention(x.q, x.k, x.v, 3, 32, 8, 64, 16, dev(x.paged.table), x.paged.cap, x.paged.pages, dev(x.L), dev(x.anc.view(np.int32)), dev(x.n), 0.0, out)
    assert ctx.cast_poll_status()[0] == 0
    within(x, out)
