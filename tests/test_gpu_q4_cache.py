"""The cache held in 4 bits: rows in and out bit by bit, attention and compaction over it against 64 bits."""
import numpy as np
import pytest
import torch

import q4_oracle as o4

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step, relative to the value


@pytest.fixture(scope="module")
def binding():
    from paper_2510_26577_b200 import build
    build.build()
    from paper_2510_26577_b200 import binding as b
    b.load_library()
    return b


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def context(binding, B, tokens=8, depth=6):
    return binding.CastContext(max_batch=B, vocab=1000, top_k=4, max_depth=depth, total_token=tokens, max_tree=tokens)


class Cache:
    """A 4-bit cache of random rows, on the host (codes [layers, pages, Hkv, slots, D], pairs fp32) and on the device."""

    def __init__(self, rng, paged, nl, Hkv, D):
        pages, slots = paged.shape
        self.paged, self.nl, self.Hkv, self.D = paged, nl, Hkv, D
        self.code, self.pair = {}, {}
        for w in "kv":
            self.code[w] = rng.integers(0, 16, (nl, pages, Hkv, slots, D)).astype(np.uint8)
            step = o4.bf16(rng.uniform(0.05, 0.4, (nl, pages, Hkv, slots, 1)).astype(np.float32))
            self.pair[w] = np.concatenate([step, o4.bf16(-7.5 * step + rng.normal(0, 0.1, step.shape).astype(np.float32))], -1)
        self.upload()

    def upload(self):
        self.kc, self.vc = (dev(o4.pack(self.code[w])) for w in "kv")
        self.kr, self.vr = (dev(self.pair[w]).to(torch.bfloat16) for w in "kv")
        self.strides = (self.kc[0].numel(), self.kr[0].numel() * 2)

    def where(self):
        p = self.paged
        return (p.page, dev(p.table), p.cap, p.pages)

    def bits(self):
        return [t.view(torch.int16).cpu().numpy() if t.dtype == torch.bfloat16 else t.cpu().numpy()
                for t in (self.kc, self.kr, self.vc, self.vr)]

    def host_bits(self):
        pairs = {w: (self.pair[w].view(np.uint32) >> 16).astype(np.uint16).view(np.int16) for w in "kv"}
        return [o4.pack(self.code["k"]), pairs["k"], o4.pack(self.code["v"]), pairs["v"]]

    def rows(self, which, layer, b, h, n):
        """Values and |step (code - 8)| of the first n positions of a sequence."""
        page, slot = self.paged.at(b, np.arange(n))
        code, pair = self.code[which][layer][page, h, slot], self.pair[which][layer][page, h, slot]
        return o4.values(code, pair), np.abs(pair[..., :1].astype(np.float64) * (code.astype(np.float64) - 8))


# ------------------------------------------------------------------------------------------------ rows in and out
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,page,Hkv,rows", [(128, 16, 8, 61), (64, 24, 3, 17), (128, 0, 1, 5), (64, 1, 2, 130), (128, 7, 2, 1)])
def test_store_and_load(binding, dtype, D, page, Hkv, rows):
    rng = np.random.default_rng(D + page + rows)
    B, nl = 4, 2
    paged = o4.Paged(rng, B, rows + 40, page)
    cache = Cache(rng, paged, nl, Hkv, D)
    x = {w: dev(rng.normal(0, 2, (nl, B, rows, Hkv, D)).astype(np.float32)).to(DT[dtype]) for w in "kv"}
    x["k"][0, 0, 0] = 3.0                     # a constant row: step 0
    x["v"][1, 1, 0, 0, 3] = float("inf")      # rows without a value
    x["v"][0, 1, 0, 0, 5] = float("nan")
    x["k"][1, 0, 0, 0, :] = torch.arange(D, device="cuda").to(DT[dtype]) / 2  # quotients that lie halfway
    x["k"][0, 1, 0, 0, :] *= 1e-39            # steps far below the normal numbers
    x["v"][0, 0, 0, 0, :2] = torch.tensor([3.3e38, -3.3e38])  # a span out of range
    start = np.array([0, 37, 5, 11], np.int32)
    n_rows = np.array([rows, rows + 9, 0, rows // 2], np.int32)
    for w in "kv":
        code, pair = o4.quantise(x[w].float().cpu().numpy())
        for b in range(B):
            n = min(n_rows[b], rows)
            pg, sl = paged.at(b, start[b] + np.arange(n))
            cache.code[w][:, pg, :, sl] = code[:, b, :n].swapaxes(0, 1)
            cache.pair[w][:, pg, :, sl] = pair[:, b, :n].swapaxes(0, 1)
    ctx = context(binding, B)
    ctx.cast_store_kv_q4(x["k"], x["v"], B, nl, rows, Hkv, D, *cache.where(), dev(start), dev(n_rows), cache.kc, cache.kr, cache.vc,
                         cache.vr, *cache.strides)
    back = {w: torch.full_like(x[w], -77.0) for w in "kv"}
    ctx.cast_load_kv_q4(cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides, B, nl, rows, Hkv, D, *cache.where(), dev(start),
                        dev(n_rows), back["k"], back["v"])
    assert ctx.cast_poll_status()[0] == 0
    for got, want in zip(cache.bits(), cache.host_bits()):  # everything else in the cache included
        np.testing.assert_array_equal(got, want) if got.dtype != np.int16 else np.testing.assert_array_equal(
            np.where((got & 0x7FFF) > 0x7F80, 0x7FC0, got), np.where((want & 0x7FFF) > 0x7F80, 0x7FC0, want))
    for w in "kv":
        for b in range(B):
            n = min(n_rows[b], rows)
            pg, sl = paged.at(b, start[b] + np.arange(n))
            want = o4.values(cache.code[w][:, pg, :, sl], cache.pair[w][:, pg, :, sl]).swapaxes(0, 1)
            want = torch.from_numpy(want.astype(np.float32)).to(DT[dtype])  # (4 + 8 bits plus 8: one rounding each)
            np.testing.assert_allclose(back[w][:, b, :n].float().cpu().numpy(), want.float().numpy(), rtol=2 * HALF[dtype], atol=1e-44)
            assert bool((back[w][:, b, n:] == -77.0).all())


def test_store_without_start_and_twice(binding):
    rng = np.random.default_rng(3)
    paged = o4.Paged(rng, 2, 33, 8)
    cache = Cache(rng, paged, 1, 2, 64)
    ctx = context(binding, 2)
    n = dev(np.array([33, 20], np.int32))
    for seed in range(2):  # the second call's rows replace the first's
        x = torch.randn((1, 2, 33, 2, 64), generator=torch.Generator("cuda").manual_seed(seed), device="cuda")
        ctx.cast_store_kv_q4(x, x, 2, 1, 33, 2, 64, *cache.where(), None, n, cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides)
    back = torch.zeros_like(x)
    ctx.cast_load_kv_q4(cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides, 2, 1, 33, 2, 64, *cache.where(), None, n, back, back.clone())
    code, pair = o4.quantise(x.cpu().numpy())
    want = o4.values(code, pair)
    np.testing.assert_allclose(back[0, 0].cpu().numpy(), want[0, 0], rtol=2.0 ** -23, atol=0)
    np.testing.assert_allclose(back[0, 1, :20].cpu().numpy(), want[0, 1, :20], rtol=2.0 ** -23, atol=0)
    assert bool((back[0, 1, 20:] == 0).all()) and ctx.cast_poll_status()[0] == 0


def test_store_refuses_places_outside(binding):
    rng = np.random.default_rng(4)
    paged = o4.Paged(rng, 3, 32, 8)
    paged.table[1, 2], paged.table[2, 0] = paged.pages, -1
    cache = Cache(rng, paged, 1, 2, 64)
    before = cache.bits()
    x = torch.randn((1, 3, 16, 2, 64), device="cuda")
    ctx = context(binding, 3)
    # sequence 0 runs past its capacity, 1 into a page id beyond the pool, 2 into a negative one
    ctx.cast_store_kv_q4(x, x, 3, 1, 16, 2, 64, *cache.where(), dev(np.array([24, 12, 2], np.int32)), dev(np.array([16, 8, 4], np.int32)),
                         cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides)
    assert ctx.cast_poll_status()[0] == 7
    code, pair = o4.quantise(x.cpu().numpy())
    for b, first, n in ((0, 24, 8), (1, 12, 4)):
        pg, sl = paged.at(b, first + np.arange(n))
        for w in "kv":
            cache.code[w][:, pg, :, sl] = code[:, b, :n].swapaxes(0, 1)
            cache.pair[w][:, pg, :, sl] = pair[:, b, :n].swapaxes(0, 1)
    for got, want, old in zip(cache.bits(), cache.host_bits(), before):
        np.testing.assert_array_equal(got, want)
        assert not np.array_equal(got, old)
    ctx.cast_load_kv_q4(cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides, 3, 1, 16, 2, 64, *cache.where(),
                        dev(np.array([-1, 0, 0], np.int32)), dev(np.array([1, 0, 0], np.int32)), x, x.clone())
    assert ctx.cast_poll_status()[0] == 7


@pytest.mark.parametrize("D,page", [(128, 16), (64, 0)])
def test_store_at_the_end_of_the_fp32_range(binding, D, page):
    """Rows whose span is finite while a value's distance from the rounded low is not: the definition's quotient is infinite
    there, and its code 15. Bit by bit, with rows just inside of the range beside them."""
    ends = [(-1.7e38, 1.7026e38), (-3.0e38, 0.4e38), (-1.7e38, 1.70e38), (-2.51e38, 0.89e38), (-0.1e38, 3.3e38), (1e38, 3.3e38)]
    rng = np.random.default_rng(D)
    x = np.stack([np.linspace(lo, hi, D).astype(np.float32)[rng.permutation(D)] for lo, hi in ends])
    with np.errstate(over="ignore"):
        low = o4.bf16(x.min(-1))
        assert np.isfinite(x.max(-1) - x.min(-1)).all() and (np.isinf(x.max(-1) - low) == [True, True, False, False, False, False]).all()
    paged = o4.Paged(rng, 1, len(ends) + 3, page)
    cache = Cache(rng, paged, 1, 1, D)
    code, pair = o4.quantise(x)
    assert (code.max(-1) == 15).all()
    pg, sl = paged.at(0, np.arange(len(ends)))
    for w, rows in (("k", slice(None)), ("v", slice(None, None, -1))):
        cache.code[w][0, pg, 0, sl], cache.pair[w][0, pg, 0, sl] = code[rows], pair[rows]
    ctx = context(binding, 1)
    xd = dev(x.reshape(1, 1, len(ends), 1, D))
    ctx.cast_store_kv_q4(xd, xd.flip(2).contiguous(), 1, 1, len(ends), 1, D, *cache.where(), None, dev(np.array([len(ends)], np.int32)),
                         cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides)
    assert ctx.cast_poll_status()[0] == 0
    for got, want in zip(cache.bits(), cache.host_bits()):
        np.testing.assert_array_equal(got, want)


# ------------------------------------------------------------------------------------------------ attention
def random_masks(rng, N, cap):
    anc = np.zeros((cap, (cap + 31) // 32), np.uint32)
    vis = np.zeros((cap, cap), bool)
    for t in range(N):
        if t:
            vis[t] = vis[int(rng.integers(0, t))]
        vis[t, t] = True
        for j in np.flatnonzero(vis[t]):
            anc[t, j >> 5] |= np.uint32(1 << (j & 31))
    return anc, vis


def run_attention(ctx, cache, q, kv_len, anc, n_tree, first=None, scale=0.0, layer=0):
    B, Hq, D = q.shape[0], q.shape[2], q.shape[3]
    out = torch.full_like(q, float("nan"))
    p = cache.paged
    ctx.cast_reserve_attention_q4(q.dtype, B, Hq, cache.Hkv, D, p.page, p.cap)
    ctx.cast_tree_attention_q4(q, cache.kc[layer], cache.kr[layer], cache.vc[layer], cache.vr[layer], B, Hq, cache.Hkv, D,
                               *cache.where(), dev(kv_len), dev(anc.view(np.int32)), dev(n_tree), dev(first), scale, out)
    return out


def check_attention(out, cache, q, kv_len, vis, n_tree, dtype, first=None, scale=0.0, layer=0):
    """Within: half a step of the output; half a bf16 step of every weight (bf16 queries), which moves an output by
    sum_p w_p step_p |code_p - 8| of that; and 32-bit sums: a score is off by at most D 2^-24 sum |q_d k_d| (scaled), twice that is
    the weights' relative error, and weights that are off by e move an output by at most 2 e max |v|."""
    got = out.double().cpu().numpy()
    x = q.double().cpu().numpy()
    B, T, Hq, D = x.shape
    G = Hq // cache.Hkv
    sc = scale or D ** -0.5
    for b in range(B):
        N, L = int(n_tree[b]), int(kv_len[b])
        F = min(int(first[b]), N) if first is not None else 0
        assert np.isnan(got[b, N:]).all() and np.isnan(got[b, :F]).all()  # left untouched
        for h in range(cache.Hkv):
            k, _ = cache.rows("k", layer, b, h, L + N)
            v, spread = cache.rows("v", layer, b, h, L + N)
            qh = x[b, F:N, h * G:(h + 1) * G]
            want, per = o4.attend(qh, k, v, spread, L, vis[b][F:N, :N], sc)
            if not want.size:
                continue
            have = got[b, F:N, h * G:(h + 1) * G]
            np.testing.assert_array_equal(np.isnan(have), np.isnan(want))
            fin = np.abs(np.where(np.isfinite(k), k, 0)).max() if k.size else 0.0
            s_err = D * 2.0 ** -24 * np.abs(qh).sum(-1).max() * fin * abs(sc) + 2.0 ** -20
            vmax = np.abs(np.where(np.isfinite(v), v, 0)).max() if v.size else 0.0
            tol = HALF[dtype] * np.abs(want) + (HALF[dtype] * per if dtype == "bf16" else 0) + 4 * s_err * vmax
            err = np.abs(have - want)
            assert not (err > tol * 1.001 + 1e-30).any(), (b, h, np.nanmax(err - tol), np.nanmax(err))


SHAPES = [  # dtype, Hq, Hkv, D, page, tokens, prefix lengths
    ("bf16", 8, 2, 128, 16, 12, [70, 200, 0, 1]),
    ("bf16", 4, 4, 64, 0, 7, [63, 64, 65, 127]),
    ("bf16", 7, 1, 128, 24, 33, [300, 0, 129, 511]),
    ("bf16", 14, 2, 64, 1, 20, [5, 17, 40]),
    ("bf16", 16, 2, 128, 64, 128, [900, 1]),
    ("bf16", 32, 8, 128, 16, 60, [2048]),
    ("bf16", 8, 8, 128, 8, 1, [1000, 31, 0, 2, 400, 7]),
    ("bf16", 64, 2, 128, 32, 5, [333, 66]),
    ("bf16", 130, 1, 64, 16, 3, [90]),
    ("f32", 8, 8, 64, 24, 33, [300, 1111, 0]),
    ("f32", 6, 2, 128, 0, 9, [64, 1, 200]),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,tokens,lens", SHAPES)
def test_attention(binding, dtype, Hq, Hkv, D, page, tokens, lens):
    rng = np.random.default_rng(Hq * 1000 + tokens)
    B = len(lens)
    cache = Cache(rng, o4.Paged(rng, B, max(lens) + tokens, page), 2, Hkv, D)
    n_tree = rng.integers(1, tokens + 1, B).astype(np.int32)
    n_tree[0] = tokens
    anc, vis = zip(*(random_masks(rng, n_tree[b], tokens) for b in range(B)))
    q = torch.randn((B, tokens, Hq, D), generator=torch.Generator("cuda").manual_seed(tokens), device="cuda").to(DT[dtype])
    for b in range(B):
        q[b, n_tree[b]:] = float("nan")  # rows past the tree may hold anything
    ctx = context(binding, B, tokens)
    kv_len = np.array(lens, np.int32)
    out = run_attention(ctx, cache, q, kv_len, np.stack(anc), n_tree, layer=1)
    assert ctx.cast_poll_status()[0] == 0
    check_attention(out, cache, q, kv_len, vis, n_tree, dtype, layer=1)
    again = run_attention(ctx, cache, q, kv_len, np.stack(anc), n_tree, layer=1)
    assert torch.equal(out.view(torch.uint8), again.view(torch.uint8))  # the same bits every time


@pytest.mark.parametrize("Hq,Hkv,D,tokens,lens", [(32, 8, 128, 60, [2048]), (14, 2, 128, 20, [5, 300, 129]), (8, 8, 128, 1, [400, 0, 7])])
def test_attention_of_unpaged_heads_of_128(binding, Hq, Hkv, D, tokens, lens):
    test_attention(binding, "bf16", Hq, Hkv, D, 0, tokens, lens)


@pytest.mark.parametrize("Hq,Hkv,D,page,tokens,lens", [
    (32, 8, 128, 16, 12, None),
    (32, 8, 64, 0, 12, None),
    (28, 4, 128, 0, 96, [1100, 1150, 1180]),
    (28, 4, 64, 24, 96, [1180, 1110, 1150]),
])
def test_attention_cut_evenly(binding, Hq, Hkv, D, page, tokens, lens):
    """More work than thread blocks: the line of tiles is cut without regard to where items end, so a block holds the end of one
    item and the beginning of another, wide and narrow ones, and hands over two partials. Without lengths: many ragged sequences,
    some with nothing to do; else few items, long enough for several blocks each."""
    rng = np.random.default_rng(D + tokens)
    if lens is None:
        lens = rng.integers(0, 700, 64)
        n_tree = rng.integers(0, tokens + 1, 64).astype(np.int32)
        n_tree[:8] = [12, 4, 0, 1, 5, 0, 0, 12]   # 16 query rows and fewer beside more
        lens[:3] = [0, 1, 650]
    else:
        n_tree = np.full(len(lens), tokens, np.int32)
    B, kv_len = len(lens), np.array(lens, np.int32)
    items = Hkv * (-(-n_tree * (Hq // Hkv) // 48))      # (48 query rows to an item, 128 positions to a tile)
    tiles = np.where(n_tree > 0, -(-(kv_len + n_tree) // 128), 0)
    grid = 2 * torch.cuda.get_device_properties(0).multi_processor_count
    longest = max(3, -(-int((items * tiles).sum()) // grid), -(-int(tiles.max()) // 32)) + 3
    assert (items * -(-tiles // longest)).sum() > grid  # or items would be cut one by one
    cache = Cache(rng, o4.Paged(rng, B, max(lens) + tokens, page), 1, Hkv, D)
    anc, vis = zip(*(random_masks(rng, n_tree[b], tokens) for b in range(B)))
    q = torch.randn((B, tokens, Hq, D), generator=torch.Generator("cuda").manual_seed(tokens), device="cuda").to(torch.bfloat16)
    ctx = context(binding, B, tokens)
    out = run_attention(ctx, cache, q, kv_len, np.stack(anc), n_tree)
    assert ctx.cast_poll_status()[0] == 0
    check_attention(out, cache, q, kv_len, vis, n_tree, "bf16")
    # the same bits again, but for query rows of NaN, in every sequence and so in items that several blocks share
    q2, spoilt = q.clone(), torch.zeros((B, tokens, Hq), dtype=torch.bool)
    for b in range(B):
        if n_tree[b]:
            spoilt[b, int(rng.integers(n_tree[b])), torch.from_numpy(rng.integers(0, Hq, 3))] = True
    q2[spoilt.cuda()] = float("nan")
    again = run_attention(ctx, cache, q2, kv_len, np.stack(anc), n_tree)
    assert ctx.cast_poll_status()[0] == 0
    assert bool(torch.isnan(again[spoilt.cuda()]).all())
    left = ~spoilt.cuda()
    assert torch.equal(again[left].view(torch.int16), out[left].view(torch.int16))
    # and a window of the rows, whose first tokens are context alone
    first = np.minimum(n_tree, rng.integers(0, tokens, B)).astype(np.int32)
    check_attention(run_attention(ctx, cache, q, kv_len, np.stack(anc), n_tree, first, 0.2), cache, q, kv_len, vis, n_tree, "bf16", first, 0.2)
    assert ctx.cast_poll_status()[0] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.3, 4.0, -0.5])
def test_attention_window_scale_and_odd_masks(binding, dtype, scale):
    """Output rows from first_row on; scales that make scores large or turn them around; rows that see nothing, or only a
    later tile; rows without a value in masked places, and one that some rows see."""
    rng = np.random.default_rng(11)
    B, tokens, Hq, Hkv, D = 4, 40, 8, 2, 128
    lens = np.array([0, 100, 0, 513], np.int32)
    cache = Cache(rng, o4.Paged(rng, B, 560, 16), 1, Hkv, D)
    n_tree = np.array([40, 31, 40, 0], np.int32)
    first = np.array([3, 31, 0, 0], np.int32)
    anc, vis = (list(z) for z in zip(*(random_masks(rng, n_tree[b], tokens) for b in range(B))))
    vis[0][5], anc[0][5] = False, 0                     # sees nothing
    vis[0][6], anc[0][6] = False, 0                     # sees the last token alone
    vis[0][6, 39], anc[0][6, 1] = True, np.uint32(1 << 7)
    for b, token in ((0, 20), (2, 39)):                 # masked for most rows
        pg, sl = cache.paged.at(b, np.array([lens[b] + token]))
        cache.pair["v"][:, pg, :, sl] = np.nan
        cache.pair["k"][:, pg, :, sl] = np.nan if b == 2 else 0.5
    for b in range(B):                                  # whatever lies behind the sequence
        pg, sl = cache.paged.at(b, np.arange(lens[b] + n_tree[b], cache.paged.positions))
        cache.pair["v"][:, pg, :, sl], cache.pair["k"][:, pg, :, sl] = np.nan, np.nan
    cache.upload()
    q = torch.randn((B, tokens, Hq, D), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(DT[dtype])
    ctx = context(binding, B, tokens)
    out = run_attention(ctx, cache, q, lens, np.stack(anc), n_tree, first, scale)
    assert ctx.cast_poll_status()[0] == 0
    check_attention(out, cache, q, lens, vis, n_tree, dtype, first, scale)
    assert bool((out[0, 5] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_far_scores(binding, dtype):
    """Scores that climb by hundreds from tile to tile, and fall again: the running reference has to follow."""
    rng = np.random.default_rng(12)
    B, tokens, Hq, Hkv, D = 2, 6, 4, 2, 128
    lens = np.array([1000, 517], np.int32)
    cache = Cache(rng, o4.Paged(rng, B, 1010, 16), 1, Hkv, D)
    for b in range(B):
        pg, sl = cache.paged.at(b, np.arange(1006))
        lift = np.where(np.arange(1006) % 700 < 350, np.arange(1006) % 350, 0) * 0.25
        cache.pair["k"][0, pg, :, sl, 1] += lift[:, None]
        cache.pair["k"] = o4.bf16(cache.pair["k"])
    cache.upload()
    q = torch.rand((B, tokens, Hq, D), generator=torch.Generator("cuda").manual_seed(2), device="cuda").to(DT[dtype])
    anc, vis = zip(*(random_masks(rng, tokens, tokens) for b in range(B)))
    n_tree = np.full(B, tokens, np.int32)
    ctx = context(binding, B, tokens)
    out = run_attention(ctx, cache, q, lens, np.stack(anc), n_tree)
    check_attention(out, cache, q, lens, vis, n_tree, dtype)
    assert ctx.cast_poll_status()[0] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_reports_and_masks_bad_pages(binding, dtype):
    rng = np.random.default_rng(13)
    cache = Cache(rng, o4.Paged(rng, 2, 200, 16), 1, 2, 128)
    q = torch.randn((2, 5, 4, 128), generator=torch.Generator("cuda").manual_seed(3), device="cuda").to(DT[dtype])
    anc, vis = zip(*(random_masks(rng, 5, 5) for b in range(2)))
    lens, n_tree = np.array([150, 90], np.int32), np.array([5, 5], np.int32)
    good = cache.paged.table.copy()
    cache.paged.table[0, 3] = cache.paged.pages + 5
    ctx = context(binding, 2, 5)
    out = run_attention(ctx, cache, q, lens, np.stack(anc), n_tree)
    status = ctx.cast_poll_status()
    assert status[0] == 7 and status[1] == 0
    cache.paged.table = good
    # the other sequence is what it is; of the first, the positions of the bad page count as masked
    keep = np.setdiff1d(np.arange(155), np.arange(48, 64))
    for h in range(2):
        k, _ = cache.rows("k", 0, 0, h, 155)
        v, spread = cache.rows("v", 0, 0, h, 155)
        want, _ = o4.attend(q[0, :, h * 2:h * 2 + 2].double().cpu().numpy(), k[keep], v[keep], spread[keep], 134, vis[0], 128 ** -0.5)
        assert np.abs(out[0, :, h * 2:h * 2 + 2].double().cpu().numpy() - want).max() < 2e-2
    one = np.array([0, 5], np.int32)
    ref = run_attention(ctx, cache, q, lens, np.stack(anc), one)
    assert torch.equal(out[1], ref[1])
    # more positions than the sequence has room for; more tokens than the context verifies
    run_attention(ctx, cache, q, np.array([204, 90], np.int32), np.stack(anc), n_tree)
    assert ctx.cast_poll_status()[0] == 7
    run_attention(ctx, cache, q, lens, np.stack(anc), np.array([5, 6], np.int32))
    assert ctx.cast_poll_status() == (6, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_reports_lengths_past_32_bits(binding, dtype):
    """A length whose sum with the tree leaves the 32-bit integers is past the capacity like any other; the batch's other
    sequence is what it is."""
    rng = np.random.default_rng(25)
    cache = Cache(rng, o4.Paged(rng, 2, 100, 16), 1, 2, 64)
    q = torch.randn((2, 5, 4, 64), generator=torch.Generator("cuda").manual_seed(3), device="cuda").to(DT[dtype])
    anc, vis = zip(*(random_masks(rng, 5, 5) for b in range(2)))
    ctx, n_tree = context(binding, 2, 5), np.array([5, 5], np.int32)
    want = run_attention(ctx, cache, q, np.array([60, 90], np.int32), np.stack(anc), n_tree)
    assert ctx.cast_poll_status()[0] == 0
    for far in (2 ** 31 - 1, 2 ** 31 - 5, 2 ** 31 - 6):
        out = run_attention(ctx, cache, q, np.array([far, 90], np.int32), np.stack(anc), n_tree)
        assert ctx.cast_poll_status() == (7, 0)
        assert torch.equal(out[1], want[1])


@pytest.mark.parametrize("dtype,D,lens", [("bf16", 128, [2100, 3]), ("bf16", 64, [1500, 0]), ("f32", 64, [700, 3]), ("f32", 128, [2100, 0])])
def test_attention_nan_and_infinity(binding, dtype, D, lens):
    """A query row of NaN gives NaN, however its sequence is divided, and so do keys without a value that fill whole tiles; a
    masked row whose pair holds infinities reaches nothing."""
    rng = np.random.default_rng(15)
    tokens, Hq, Hkv = 6, 8, 2
    cache = Cache(rng, o4.Paged(rng, 2, max(lens) + tokens, 16), 1, Hkv, D)
    pg, sl = cache.paged.at(0, np.arange(400))
    cache.pair["k"][0, pg, 1, sl] = np.nan
    anc, vis = (list(z) for z in zip(*(random_masks(rng, tokens, tokens) for b in range(2))))
    for b in range(2):  # token 4 is seen by itself alone
        vis[b][5, 4] = False
        anc[b][5, 0] &= ~np.uint32(1 << 4)
        pg, sl = cache.paged.at(b, np.array([lens[b] + 4]))
        cache.pair["v"][0, pg, 0, sl] = [np.inf, 1.0] if b else [0.25, -np.inf]
    cache.upload()
    q = torch.randn((2, tokens, Hq, D), generator=torch.Generator("cuda").manual_seed(4), device="cuda").to(DT[dtype])
    q[0, 2, 1], q[1, 3, 5] = float("nan"), float("nan")
    q[0, 3, 2, 7] = float("nan")
    ctx = context(binding, 2, tokens)
    n_tree = np.full(2, tokens, np.int32)
    out = run_attention(ctx, cache, q, np.array(lens, np.int32), np.stack(anc), n_tree)
    assert ctx.cast_poll_status()[0] == 0
    got = torch.isnan(out).cpu().numpy()
    want = np.zeros_like(got)
    want[0, :, 4:] = True                        # kv-head 1 of the first sequence
    want[0, 2, 1] = want[0, 3, 2] = want[1, 3, 5] = True
    want[:, 4, :4] = True                        # token 4 sees its own infinity
    out = torch.where(torch.isinf(out), torch.full_like(out, float("nan")), out)
    np.testing.assert_array_equal(got | torch.isnan(out).cpu().numpy(), want)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f32", 64)])
def test_rows_past_four_gigabytes(binding, dtype, D):
    """Pages at the far end of a cache of more than 2^32 bytes: the same bits as from a small one, through every call."""
    rng = np.random.default_rng(22)
    B, Hq, Hkv, page, cap, T, H = 2, 4, 2, 16, 12, 9, 4
    few = B * cap
    far = (1 << 32) // (Hkv * page * D // 2) + 100
    table = rng.permutation(few).reshape(B, cap).astype(np.int32)
    x = torch.randn((2, 1, B, 180, Hkv, D), generator=torch.Generator("cuda").manual_seed(7), device="cuda").to(DT[dtype])
    q = torch.randn((B, T, Hq, D), generator=torch.Generator("cuda").manual_seed(8), device="cuda").to(DT[dtype])
    anc = np.stack([random_masks(rng, T, T)[0] for b in range(B)])
    n_tree, path = dev(np.full(B, T, np.int32)), dev(np.tile(np.array([0, 3, 5, 6, 8], np.int32), (B, 1)))
    ctx = context(binding, B, T, H)
    ctx.cast_reserve_attention_q4(q.dtype, B, Hq, Hkv, D, page, cap)
    ctx.cast_reserve_attention_mass(q.dtype, B, 1, H + 1, Hq, Hkv, D, page, cap)
    results = []
    for pages, first in ((few, 0), (far, far - few)):
        codes = [torch.empty((1, pages, Hkv, page, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
        pairs = [torch.empty((1, pages, Hkv, page, 2), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        cache, strides = (codes[0], pairs[0], codes[1], pairs[1]), (codes[0][0].numel(), pairs[0][0].numel() * 2)
        where, kv_len = (page, dev(table + first), cap, pages), dev(np.array([171, 100], np.int32))
        out, back, mass = torch.zeros_like(q), torch.zeros_like(x), torch.zeros((1, B, Hkv, cap * page), device="cuda")
        kept = torch.zeros((1, B, Hkv, 60), dtype=torch.int32, device="cuda")
        ctx.cast_store_kv_q4(x[0], x[1], B, 1, 180, Hkv, D, *where, None, dev(np.array([180, 109], np.int32)), *cache, *strides)
        ctx.cast_tree_attention_q4(q, *(t[0] for t in cache), B, Hq, Hkv, D, *where, kv_len, dev(anc.view(np.int32)), n_tree, None, 0.0, out)
        ctx.cast_compact_kv_q4(*cache, *strides, B, 1, Hkv, D, *where, path, dev(np.array([4, 2], np.int32)), kv_len)
        ctx.cast_attention_mass_q4(q, codes[0], pairs[0], B, 1, 0, *strides, Hq, Hkv, D, *where, path, dev(np.array([4, 2], np.int32)), kv_len, 0.0, mass)
        ctx.cast_evict_kv_q4(*cache, *strides, B, 1, Hkv, D, *where, 60, 10, mass, kept, kv_len)
        ctx.cast_load_kv_q4(*cache, *strides, B, 1, 180, Hkv, D, *where, None, kv_len, back[0], back[1])
        assert ctx.cast_poll_status()[0] == 0
        results.append((out, back, mass, kept, kv_len))
    for a, b in zip(*results):
        assert torch.equal(a, b) and bool(a.any())


def test_attention_without_work_and_with_a_larger_workspace(binding):
    """No token in any sequence: nothing is written; a call after the workspace has grown for a larger one."""
    rng = np.random.default_rng(23)
    small, large = (Cache(rng, o4.Paged(rng, B, n, 16), 1, 2, 128) for B, n in ((2, 300), (9, 700)))
    ctx = context(binding, 9, 12)
    for cache, kv in ((small, [280, 3]), (large, [680] * 9), (small, [280, 3])):
        B = len(kv)
        q = torch.randn((B, 12, 14, 128), generator=torch.Generator("cuda").manual_seed(B), device="cuda").to(torch.bfloat16)
        anc, vis = zip(*(random_masks(rng, 12, 12) for b in range(B)))
        kv, n_tree = np.array(kv, np.int32), np.full(B, 12, np.int32)
        out = run_attention(ctx, cache, q, kv, np.stack(anc), n_tree)
        check_attention(out, cache, q, kv, vis, n_tree, "bf16")
        none = run_attention(ctx, cache, q, kv, np.stack(anc), np.zeros(B, np.int32))
        assert bool(torch.isnan(none).all())
    assert ctx.cast_poll_status()[0] == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_workspace_serves_fewer_sequences(binding, dtype):
    """Reserved once for the most sequences: every smaller batch runs, those among them that divide a sequence further, with the
    bits that it has after a reservation of its own."""
    rng = np.random.default_rng(24)
    Bmax, tokens, Hq, Hkv, D = 5, 12, 32, 8, 64
    ctx = context(binding, Bmax, tokens)
    ctx.cast_reserve_attention_q4(DT[dtype], Bmax, Hq, Hkv, D, 16, 64)
    anc, vis = zip(*(random_masks(rng, tokens, tokens) for b in range(Bmax)))
    for B in range(Bmax, 0, -1):
        cache = Cache(rng, o4.Paged(rng, B, 1024, 16), 1, Hkv, D)
        q = torch.randn((B, tokens, Hq, D), generator=torch.Generator("cuda").manual_seed(B), device="cuda").to(DT[dtype])
        kv, n_tree = rng.integers(0, 1024 - tokens, B).astype(np.int32), np.full(B, tokens, np.int32)
        out = torch.full_like(q, float("nan"))
        ctx.cast_tree_attention_q4(q, cache.kc[0], cache.kr[0], cache.vc[0], cache.vr[0], B, Hq, Hkv, D, *cache.where(), dev(kv),
                                   dev(np.stack(anc[:B]).view(np.int32)), dev(n_tree), None, 0.0, out)
        assert ctx.cast_poll_status()[0] == 0
        own = context(binding, B, tokens)
        want = run_attention(own, cache, q, kv, np.stack(anc[:B]), n_tree)
        assert torch.equal(out, want)
        if B in (1, 3):
            check_attention(out, cache, q, kv, vis, n_tree, dtype)


def test_attention_needs_its_workspace_and_shapes(binding):
    rng = np.random.default_rng(14)
    cache = Cache(rng, o4.Paged(rng, 1, 4096, 16), 1, 2, 128)
    ctx = context(binding, 1, 8)
    q = torch.zeros((1, 8, 4, 128), dtype=torch.bfloat16, device="cuda")
    anc, n, L = torch.zeros((1, 8, 1), dtype=torch.int32, device="cuda"), dev(np.array([8], np.int32)), dev(np.array([4000], np.int32))

    def call(c=ctx, q=q, codes=cache.kc[0], B=1, Hq=4, Hkv=2, D=128, out=None):
        c.cast_tree_attention_q4(q, codes, cache.kr[0], cache.vc[0], cache.vr[0], B, Hq, Hkv, D, *cache.where(), L, anc, n, None, 0.0,
                                 q.clone() if out is None else out)

    def code(**kw):
        with pytest.raises(binding.CastError) as e:
            call(**kw)
        return e.value.code

    assert code() == 3  # nothing reserved
    ctx.cast_reserve_attention_q4(torch.bfloat16, 1, 4, 2, 128, 16, cache.paged.cap)
    call()
    assert code(B=2) == 3
    assert code(Hq=3) == 2
    assert code(D=96) == 2
    assert code(Hkv=0) == 1
    assert code(out=q.float()) == 4  # another type than the queries'
    assert code(codes=cache.kc[0].reshape(-1)[8:]) == 2  # alignment
    with pytest.raises(TypeError):
        call(codes=cache.kc[0].view(torch.int8))
    with pytest.raises(AssertionError):
        call(q=q.transpose(1, 2))
    with pytest.raises(binding.CastError):
        ctx.cast_reserve_attention_q4(torch.bfloat16, 1, 4, 2, 100, 16, 4)
    assert ctx.cast_poll_status()[0] == 0


def test_sequences_too_long_for_32_bit_positions(binding):
    """The most positions that a sequence may have, and one more, by pages and without: refused by every call, before anything
    runs, since the kernels' indices run past a sequence's end by a tile."""
    B, T, H, D, most = 1, 4, 4, 64, 2 ** 31 - 2 ** 16
    ctx = context(binding, B, T, H)
    x, q = (torch.ones((1, B, T, n, D), device="cuda", dtype=torch.bfloat16) for n in (1, 2))
    kc, vc = (torch.zeros((1, B, 1, 16, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    kr, vr = (torch.zeros((1, B, 1, 16, 2), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    dense = torch.ones((1, B, 16, 1, D), device="cuda", dtype=torch.bfloat16)
    cache, strides = (kc, kr, vc, vr), (kc.numel(), kr.numel() * 2)
    n, one, path = dev(np.array([T], np.int32)), dev(np.array([0], np.int32)), torch.zeros((B, H + 1), dtype=torch.int32, device="cuda")
    anc, table = torch.ones((B, T, 1), dtype=torch.int32, device="cuda"), torch.zeros((B, 16), dtype=torch.int32, device="cuda")
    out, mass, kept = torch.zeros_like(q[0]), torch.zeros(16, device="cuda"), torch.zeros(16, dtype=torch.int32, device="cuda")
    calls = [
        lambda w: ctx.cast_reserve_attention_q4(torch.bfloat16, B, 2, 1, D, w[0], w[2]),
        lambda w: ctx.cast_reserve_attention_q4(torch.float32, B, 2, 1, D, w[0], w[2]),
        lambda w: ctx.cast_reserve_attention_mass(torch.bfloat16, B, 1, H + 1, 2, 1, D, w[0], w[2]),
        lambda w: ctx.cast_store_kv_q4(x, x, B, 1, T, 1, D, *w, None, n, *cache, *strides),
        lambda w: ctx.cast_load_kv_q4(*cache, *strides, B, 1, T, 1, D, *w, None, n, x.clone(), x.clone()),
        lambda w: ctx.cast_tree_attention_q4(q[0], kc, kr, vc, vr, B, 2, 1, D, *w, one, anc, n, None, 0.0, out),
        lambda w: ctx.cast_compact_kv_q4(*cache, *strides, B, 1, 1, D, *w, path, one, n.clone()),
        lambda w: ctx.cast_attention_mass_q4(q, kc, kr, B, 1, 0, *strides, 2, 1, D, *w, path, one, n, 0.0, mass),
        lambda w: ctx.cast_attention_mass(q, dense, B, 1, 0, 0, 2, 1, D, *w, path, one, n, 0.0, mass),
        lambda w: ctx.cast_evict_kv_q4(*cache, *strides, B, 1, 1, D, *w, 8, 2, mass, kept, n),
        lambda w: ctx.cast_evict_kv(dense, dense.clone(), B, 1, 0, 1, D, *w, 8, 2, mass, kept, n),
    ]
    for where in ((0, None, most + 1, 0), (1 << 15, table, (1 << 16) - 1, 1)):
        for i, call in enumerate(calls):
            with pytest.raises(binding.CastError) as e:
                call(where)
            assert e.value.code == 3, i
    for call in calls:  # (a few positions of it are there)
        call((0, None, most, 0))
    assert ctx.cast_poll_status()[0] == 0


# ------------------------------------------------------------------------------------------------ compaction
@pytest.mark.parametrize("D,page,Hkv", [(128, 16, 8), (64, 0, 2), (128, 5, 1)])
def test_compaction(binding, D, page, Hkv):
    rng = np.random.default_rng(page + D)
    B, nl, H = 3, 3, 6
    cache = Cache(rng, o4.Paged(rng, B, 90, page), nl, Hkv, D)
    path = np.full((B, H + 1), -1, np.int32)
    path[0, :4], path[1, :1], path[2] = [0, 2, 5, 9], [0], np.arange(7)
    n = np.array([3, 0, 6], np.int32)
    lens = np.array([60, 31, 47], np.int32)
    for b in range(B):
        src, to = cache.paged.at(b, lens[b] + path[b, :n[b] + 1]), cache.paged.at(b, lens[b] + np.arange(n[b] + 1))
        for w in "kv":
            for a in (cache.code[w], cache.pair[w]):
                a[:, to[0], :, to[1]] = a[:, src[0], :, src[1]]
    ctx = context(binding, B, 16, H)
    kv_len = dev(lens)
    ctx.cast_compact_kv_q4(cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides, B, nl, Hkv, D, *cache.where(), dev(path), dev(n), kv_len)
    assert ctx.cast_poll_status()[0] == 0
    np.testing.assert_array_equal(kv_len.cpu().numpy(), lens + n + 1)
    for got, want in zip(cache.bits(), cache.host_bits()):
        np.testing.assert_array_equal(got, want)
    # a path that goes back, or past the capacity: nothing moves, the length stays
    bad = path.copy()
    bad[0, 2], bad[1, 0] = 1, 80
    before, lens2 = cache.bits(), dev(lens)
    ctx.cast_compact_kv_q4(cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides, B, nl, Hkv, D, *cache.where(), dev(bad),
                           dev(np.array([3, 0, -1], np.int32)), lens2)
    assert ctx.cast_poll_status()[0] == 7
    np.testing.assert_array_equal(lens2.cpu().numpy()[:2], lens[:2])
    for got, want in zip(cache.bits(), before):
        np.testing.assert_array_equal(got, want)


# ------------------------------------------------------------------------------------------------ as a program uses it
@pytest.mark.parametrize("captured", [False, True])
def test_a_step_on_the_4_bit_cache(binding, captured):
    """Prefill, then two steps: the tree's rows stored, attention of two layers, compaction - on another stream, and captured and
    replayed with new inputs."""
    rng = np.random.default_rng(21)
    B, nl, T, Hq, Hkv, D, H = 2, 2, 12, 8, 2, 128, 4
    paged = o4.Paged(rng, B, 260, 16)
    cache = Cache(rng, paged, nl, Hkv, D)
    ctx = context(binding, B, T, H)
    ctx.cast_reserve_attention_q4(torch.bfloat16, B, Hq, Hkv, D, paged.page, paged.cap)
    prompt = torch.randn((2, nl, B, 200, Hkv, D), device="cuda", dtype=torch.bfloat16)
    n0 = np.array([200, 77], np.int32)
    where, kv_len, n_rows = cache.where(), dev(n0), dev(np.array([T, T], np.int32))
    new = torch.randn((2, nl, B, T, Hkv, D), device="cuda", dtype=torch.bfloat16)
    q = torch.randn((nl, B, T, Hq, D), device="cuda", dtype=torch.bfloat16)
    out = torch.full_like(q, float("nan"))
    anc, vis = zip(*(random_masks(rng, T, T) for b in range(B)))
    anc_d = dev(np.stack(anc).view(np.int32))
    path, alen = torch.zeros((B, H + 1), dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")

    def step():
        ctx.cast_store_kv_q4(new[0], new[1], B, nl, T, Hkv, D, *where, kv_len, n_rows, cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides)
        for l in range(nl):
            ctx.cast_tree_attention_q4(q[l], cache.kc[l], cache.kr[l], cache.vc[l], cache.vr[l], B, Hq, Hkv, D, *where, kv_len, anc_d,
                                       n_rows, None, 0.0, out[l])
        ctx.cast_compact_kv_q4(cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides, B, nl, Hkv, D, *where, path, alen, kv_len)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.cast_store_kv_q4(prompt[0], prompt[1], B, nl, 200, Hkv, D, *where, None, kv_len, cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides)
        graph = None
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
    host = {w: [[np.zeros((0, Hkv, D + 2))] * B for _ in range(nl)] for w in "kv"}
    for i, w in enumerate("kv"):  # the rows every sequence holds: codes and pairs side by side
        code, pair = o4.quantise(prompt[i].float().cpu().numpy())
        rows = np.concatenate([code.astype(np.float64), pair], -1)
        host[w] = [[rows[l, b, :n0[b]] for b in range(B)] for l in range(nl)]
    lens = n0.copy()
    for k in range(2):
        g = torch.Generator("cuda").manual_seed(50 + k)
        with torch.cuda.stream(side):
            new.normal_(generator=g)
            q.normal_(generator=g)
            p = np.zeros((B, H + 1), np.int32)
            p[0, :3], p[1, :2] = [0, 3, 7], [0, 1 + k]
            path.copy_(torch.from_numpy(p))
            alen.copy_(torch.from_numpy(np.array([2, 1], np.int32)))
            graph.replay() if captured else step()
        side.synchronize()
        tree = {w: o4.quantise(new[i].float().cpu().numpy()) for i, w in enumerate("kv")}
        for l in range(nl):
            for b in range(B):
                both = {w: np.concatenate([host[w][l][b], np.concatenate([tree[w][0][l, b], tree[w][1][l, b]], -1)]) for w in "kv"}
                for h in range(Hkv):
                    kk, vv = (o4.values(both[w][:, h, :D], both[w][:, h, D:]) for w in "kv")
                    spread = np.abs(both["v"][:, h, D:D + 1] * (both["v"][:, h, :D] - 8))
                    want, per = o4.attend(q[l, b, :, h * 4:h * 4 + 4].double().cpu().numpy(), kk, vv, spread, lens[b], vis[b], D ** -0.5)
                    err = np.abs(out[l, b, :, h * 4:h * 4 + 4].double().cpu().numpy() - want)
                    assert (err <= HALF["bf16"] * (np.abs(want) + per) + 1e-3).all()
                for w in "kv":
                    tr = both[w][lens[b]:]
                    host[w][l][b] = np.concatenate([host[w][l][b], tr[p[b, :(3 if b == 0 else 2)]]])
        lens = lens + np.array([3, 2], np.int32)
        np.testing.assert_array_equal(kv_len.cpu().numpy(), lens)
    assert ctx.cast_poll_status()[0] == 0
