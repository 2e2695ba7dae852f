"""The attention weight that cached positions draw, against 64 bits, and the eviction of those that drew least, row by row."""
import numpy as np
import pytest
import torch

import q4_oracle as o4
from test_gpu_q4_cache import DT, Cache, context, dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    from paper_2510_26577_b200 import build
    build.build()
    from paper_2510_26577_b200 import binding as b
    b.load_library()
    return b


class Dense:
    """A 16-bit or fp32 cache [layers, pages, slots, Hkv, D] of random rows."""

    def __init__(self, rng, paged, nl, Hkv, D, dtype):
        self.paged, self.nl, self.Hkv, self.D = paged, nl, Hkv, D
        g = torch.Generator("cuda").manual_seed(int(rng.integers(1 << 30)))
        self.k, self.v = (torch.randn((nl, *paged.shape, Hkv, D), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
        self.stride = self.k[0].numel() * self.k.element_size()

    def where(self):
        p = self.paged
        return (p.page, dev(p.table), p.cap, p.pages)

    def rows(self, which, layer, b, h, n):
        page, slot = self.paged.at(b, np.arange(n))
        x = (self.k if which == "k" else self.v)[layer].double().cpu().numpy()
        return x[page, slot, h], None


# ------------------------------------------------------------------------------------------------ mass
def run_mass(ctx, cache, q, path, alen, kv_len, mass, scale=0.0, rows=None):
    nl, B, T, Hq, D = q.shape
    p = cache.paged
    ctx.cast_reserve_attention_mass(q.dtype, B, nl, rows or (path.shape[1] if path is not None else T), Hq, cache.Hkv, D, p.page, p.cap)
    qs = q[0].numel() * q.element_size()
    if isinstance(cache, Cache):
        ctx.cast_attention_mass_q4(q, cache.kc, cache.kr, B, nl, qs, *cache.strides, Hq, cache.Hkv, D, *cache.where(), dev(path), dev(alen),
                                   dev(kv_len), scale, mass)
    else:
        ctx.cast_attention_mass(q, cache.k, B, nl, qs, cache.stride, Hq, cache.Hkv, D, *cache.where(), dev(path), dev(alen), dev(kv_len),
                                scale, mass)


def check_mass(mass, before, cache, q, path, alen, kv_len, scale=0.0):
    """Scores are 32-bit sums of D products: off by at most D 2^-24 sum |q_d k_d| (scaled), a weight by twice that relative to
    it plus the exponential's and the quotient's few steps; the sums over rows and with what was there add a step per term."""
    got = mass.double().cpu().numpy()
    nl, B, T, Hq, D = q.shape
    G, sc = Hq // cache.Hkv, scale or D ** -0.5
    x = q.double().cpu().numpy()
    for l in range(nl):
        for b in range(B):
            n, L = int(alen[b]) + 1, int(kv_len[b])
            for h in range(cache.Hkv):
                old = before[l, b, h].double().cpu().numpy()
                if n < 1:
                    np.testing.assert_array_equal(got[l, b, h], old)
                    continue
                k, _ = cache.rows("k", l, b, h, L)
                rows = path[b, :n] if path is not None else np.arange(n)
                qh = x[l, b, rows, h * G:(h + 1) * G]
                add = o4.mass_of(qh, k, L - n + np.arange(n) + 1, sc)
                s_err = D * 2.0 ** -24 * np.einsum("tgd,pd->tgp", np.abs(qh), np.abs(k)).max() * abs(sc)
                tol = add * (2 * s_err + 2.0 ** -19) + (n * G + 2) * 2.0 ** -24 * (np.abs(old[:L]) + add) + 1e-30
                err = np.abs(got[l, b, h, :L] - (old[:L] + add))
                assert (err <= tol).all(), (l, b, h, (err - tol).max(), err.max())
                np.testing.assert_array_equal(got[l, b, h, L:], old[L:])


MASS = [  # cache, dtype, Hq, Hkv, D, page, depth, accepted - 1 per sequence, lengths behind the compaction
    ("16", "bf16", 8, 2, 128, 16, 6, [3, 0, 6, -1], [200, 1, 65, 40]),
    ("4", "bf16", 8, 2, 128, 16, 6, [3, 0, 6, -1], [200, 1, 65, 40]),
    ("16", "bf16", 7, 1, 64, 0, 13, [13, 5], [1100, 517]),
    ("4", "bf16", 7, 1, 64, 24, 13, [13, 5], [1100, 517]),
    ("4", "bf16", 64, 2, 128, 1, 16, [16], [300]),
    ("16", "bf16", 32, 8, 128, 64, 6, [4], [2049]),
    ("4", "bf16", 28, 4, 128, 16, 6, [2, 6], [3000, 127]),
    ("16", "f32", 8, 8, 64, 24, 4, [4, 2], [300, 129]),
    ("16", "f32", 4, 2, 128, 0, 4, [4, 2], [64, 3]),
    ("4", "f32", 4, 1, 128, 8, 4, [1, 4], [100, 64]),
]


@pytest.mark.parametrize("kind,dtype,Hq,Hkv,D,page,depth,accepted,lens", MASS)
def test_mass(binding, kind, dtype, Hq, Hkv, D, page, depth, accepted, lens):
    rng = np.random.default_rng(Hq + D + page)
    B, nl, T = len(lens), 2, 40
    paged = o4.Paged(rng, B, max(lens) + 5, page)
    cache = Cache(rng, paged, nl, Hkv, D) if kind == "4" else Dense(rng, paged, nl, Hkv, D, dtype)
    path = np.full((B, depth + 1), -1, np.int32)
    for b, a in enumerate(accepted):
        path[b, :a + 1] = np.sort(rng.choice(T, a + 1, replace=False))
    alen, kv_len = np.array(accepted, np.int32), np.array(lens, np.int32)
    q = torch.randn((nl, B, T, Hq, D), generator=torch.Generator("cuda").manual_seed(Hq), device="cuda").to(DT[dtype])
    used = torch.zeros((B, T), dtype=torch.bool)
    for b in range(B):
        used[b, path[b, :max(accepted[b] + 1, 0)]] = True
    q[:, ~used.cuda()] = float("nan")  # rows that were not accepted are not read into any sum
    before = torch.rand((nl, B, Hkv, paged.positions), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    ctx = context(binding, B, T, depth)
    mass, again = before.clone(), before.clone()
    run_mass(ctx, cache, q, path, alen, kv_len, mass)
    assert ctx.cast_poll_status()[0] == 0
    check_mass(mass, before, cache, q, path, alen, kv_len)
    run_mass(ctx, cache, q, path, alen, kv_len, again)
    assert torch.equal(mass, again)
    # and once more onto what is there, as the next step does
    run_mass(ctx, cache, q, path, alen, kv_len, again)
    check_mass(again, mass, cache, q, path, alen, kv_len)


@pytest.mark.parametrize("kind,dtype,Hq,Hkv,D,page,depth,accepted,lens", [
    ("4", "bf16", 7, 1, 64, 0, 13, [13, 5], [1100, 517]),
    ("4", "bf16", 8, 2, 128, 0, 6, [3, 0, 6, -1], [200, 1, 65, 40]),
    ("16", "bf16", 28, 4, 128, 0, 6, [2, 6], [2200, 127]),
    ("16", "bf16", 8, 2, 64, 24, 6, [3, 0, 6, -1], [200, 1, 65, 40]),
    ("16", "bf16", 7, 1, 64, 1, 13, [13, 5], [1100, 517]),
    ("4", "f32", 8, 8, 64, 0, 4, [4, 2], [300, 129]),
])
def test_mass_in_other_layouts(binding, kind, dtype, Hq, Hkv, D, page, depth, accepted, lens):
    test_mass(binding, kind, dtype, Hq, Hkv, D, page, depth, accepted, lens)


class Kept(Dense):
    """A cache whose rows are brought to the host once."""

    def rows(self, which, layer, b, h, n):
        if not hasattr(self, "host"):
            self.host = self.k.float().cpu().numpy()
        page, slot = self.paged.at(b, np.arange(n))
        return self.host[layer][page, slot, h].astype(np.float64), None


@pytest.mark.parametrize("D,page", [(128, 16), (64, 0)])
@pytest.mark.parametrize("kind,dtype", [("16", "bf16"), ("4", "bf16"), ("16", "f32"), ("4", "f32")])
def test_mass_far_scores(binding, kind, dtype, D, page):
    """Scores that climb by hundreds from tile to tile and fall again, several tiles to a piece and two pieces to a sequence: a
    row's reference has to follow within a piece, and pieces with references far apart have to meet."""
    rng = np.random.default_rng(16)
    nl, T, Hq, Hkv, H = 16, 6, 16, 8, 2
    lens = np.array([1000, 517, 130, 900, 1003], np.int32)
    B = len(lens)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert 2 <= -(-8 * sms // (B * nl * Hkv)) <= 2  # pieces, of 4 tiles of 128 in the longest
    paged = o4.Paged(rng, B, 1010, page)
    cache = Cache(rng, paged, nl, Hkv, D) if kind == "4" else Kept(rng, paged, nl, Hkv, D, dtype)
    pos = np.arange(1010)
    lift = (np.where(pos % 700 < 350, pos % 350, 0) * 0.25).astype(np.float32)
    for b in range(B):
        pg, sl = paged.at(b, pos)
        if kind == "4":
            cache.pair["k"][:, pg, :, sl, 1] += lift[:, None, None]
        else:
            cache.k[:, torch.from_numpy(pg).cuda(), torch.from_numpy(sl).cuda()] += torch.from_numpy(lift).cuda().to(DT[dtype])[:, None, None]
    if kind == "4":
        cache.pair["k"] = o4.bf16(cache.pair["k"])
        cache.upload()
    q = torch.rand((nl, B, T, Hq, D), generator=torch.Generator("cuda").manual_seed(2), device="cuda").to(DT[dtype])
    path, alen = np.tile(np.array([[0, 2, 5]], np.int32), (B, 1)), np.array([2, 0, 2, 1, 2], np.int32)
    mass = torch.zeros((nl, B, Hkv, paged.positions), device="cuda")
    ctx = context(binding, B, T, H)
    run_mass(ctx, cache, q, path, alen, lens, mass)
    assert ctx.cast_poll_status()[0] == 0
    check_mass(mass, torch.zeros_like(mass), cache, q, path, alen, lens)


@pytest.mark.parametrize("kind,dtype", [("16", "bf16"), ("4", "bf16"), ("16", "f32"), ("4", "f32")])
def test_mass_beside_bad_pages(binding, kind, dtype):
    """Pages that are none: the first tile of a piece, a whole piece and the beginning of the next, a tile in the middle, all of
    a sequence. Their positions count as masked, draw nothing, and the others share what the rows give."""
    rng = np.random.default_rng(17)
    nl, T, Hq, Hkv, D, H, L = 2, 8, 8, 2, 128, 4, 1000
    bad = [np.arange(128), np.arange(304), np.arange(512, 640), np.arange(L + 16), np.zeros(0, int)]
    B = len(bad)
    paged = o4.Paged(rng, B, L + 20, 16)
    cache = Cache(rng, paged, nl, Hkv, D) if kind == "4" else Kept(rng, paged, nl, Hkv, D, dtype)
    good = paged.table.copy()
    q = torch.randn((nl, B, T, Hq, D), generator=torch.Generator("cuda").manual_seed(5), device="cuda").to(DT[dtype])
    path, alen, kv_len = np.tile(np.array([[0, 2, 5, 6, 7]], np.int32), (B, 1)), np.array([4, 2, 0, 3, 1], np.int32), np.full(B, L, np.int32)
    for b, pos in enumerate(bad):
        paged.table[b, pos // 16] = rng.choice([-1, paged.pages, 2 ** 31 - 1], len(pos))
    mass = torch.zeros((nl, B, Hkv, paged.positions), device="cuda")
    ctx = context(binding, B, T, H)
    run_mass(ctx, cache, q, path, alen, kv_len, mass)
    assert ctx.cast_poll_status()[0] == 7
    paged.table = good
    got, x = mass.double().cpu().numpy(), q.double().cpu().numpy()
    for l in range(nl):
        for b in range(B):
            n = int(alen[b]) + 1
            for h in range(Hkv):
                k = cache.rows("k", l, b, h, L)[0]
                keep = np.setdiff1d(np.arange(L), bad[b])
                qh = x[l, b, path[b, :n], h * 4:h * 4 + 4]
                want = np.zeros(L)
                # a row sees the kept positions below its own bound: as many of them as lie there
                if len(keep):
                    want[keep] = o4.mass_of(qh, k[keep], [(keep < L - n + i + 1).sum() for i in range(n)], D ** -0.5)
                s_err = D * 2.0 ** -24 * np.einsum("tgd,pd->tgp", np.abs(qh), np.abs(k)).max() * D ** -0.5
                tol = want * (2 * s_err + 2.0 ** -19 + (n * 4 + 2) * 2.0 ** -24) + 1e-30
                assert (np.abs(got[l, b, h, :L] - want) <= tol).all() and not got[l, b, h, L:].any()


@pytest.mark.parametrize("kind", ["16", "4"])
def test_mass_of_a_window_of_rows(binding, kind):
    """Without a path: the last rows of a prompt chunk, more of them than one block of the kernels."""
    rng = np.random.default_rng(8)
    B, T, Hq, Hkv, D = 2, 100, 8, 2, 128
    paged = o4.Paged(rng, B, 400, 16)
    cache = Cache(rng, paged, 1, Hkv, D) if kind == "4" else Dense(rng, paged, 1, Hkv, D, "bf16")
    q = torch.randn((1, B, T, Hq, D), generator=torch.Generator("cuda").manual_seed(4), device="cuda").to(torch.bfloat16)
    alen, kv_len = np.array([99, 30], np.int32), np.array([399, 31], np.int32)
    mass = torch.zeros((1, B, Hkv, paged.positions), device="cuda")
    ctx = context(binding, B, T)
    run_mass(ctx, cache, q, None, alen, kv_len, mass, scale=0.2)
    assert ctx.cast_poll_status()[0] == 0
    check_mass(mass, torch.zeros_like(mass), cache, q, None, alen, kv_len, scale=0.2)


@pytest.mark.parametrize("kind,dtype", [("16", "bf16"), ("4", "bf16"), ("16", "f32"), ("4", "f32")])
def test_mass_nan(binding, kind, dtype):
    """A query of NaN makes what its row sees NaN, in its layer and kv-head alone; a key without a value likewise, and one
    that no row sees reaches nothing."""
    rng = np.random.default_rng(10)
    B, nl, T, Hq, Hkv, D, L = 3, 2, 8, 4, 2, 128, 1500
    paged = o4.Paged(rng, B, L + 20, 16)
    cache = Cache(rng, paged, nl, Hkv, D) if kind == "4" else Dense(rng, paged, nl, Hkv, D, dtype)
    pos = np.concatenate([np.arange(1498, 1510)])
    for b in (1, 2):  # the last row alone sees position 1499; 1500 and on lie behind the sequence
        pg, sl = paged.at(b, pos if b == 1 else pos[2:])
        if kind == "4":
            cache.pair["k"][1, pg, 1, sl] = np.nan
        else:
            cache.k[1, torch.from_numpy(pg), torch.from_numpy(sl), 1] = float("nan")
    if kind == "4":
        cache.upload()
    q = torch.randn((nl, B, T, Hq, D), generator=torch.Generator("cuda").manual_seed(6), device="cuda").to(DT[dtype])
    q[0, 0, 3, 1] = float("nan")
    path = np.tile(np.array([[1, 3, 6, 0, 0]], np.int32), (B, 1))
    mass = torch.zeros((nl, B, Hkv, paged.positions), device="cuda")
    ctx = context(binding, B, T, 4)
    run_mass(ctx, cache, q, path, np.full(B, 2, np.int32), np.full(B, L, np.int32), mass)
    assert ctx.cast_poll_status()[0] == 0
    want = np.zeros(mass.shape, bool)
    want[0, 0, 0, :L - 1] = True   # row 1 of 3 sees all positions but the last
    want[1, 1, 1, :L] = True       # rows 1 and 2 see 1498; what row 2 gives reaches all
    np.testing.assert_array_equal(np.isnan(mass.cpu().numpy()), want)


def test_16_bit_rows_past_four_gigabytes(binding):
    """As for the 4-bit cache: weights and eviction at the far end of a large cache."""
    rng = np.random.default_rng(11)
    B, Hq, Hkv, D, page, cap, T, H = 2, 4, 2, 128, 16, 12, 9, 4
    few, far = B * cap, (1 << 32) // (Hkv * page * D * 2) + 100
    table = rng.permutation(few).reshape(B, cap).astype(np.int32)
    rows = torch.randn((2, few, page, Hkv, D), generator=torch.Generator("cuda").manual_seed(7), device="cuda").to(torch.bfloat16)
    q = torch.randn((1, B, T, Hq, D), generator=torch.Generator("cuda").manual_seed(8), device="cuda").to(torch.bfloat16)
    ctx = context(binding, B, T, H)
    ctx.cast_reserve_attention_mass(q.dtype, B, 1, T, Hq, Hkv, D, page, cap)
    results = []
    for pages, first in ((few, 0), (far, far - few)):
        k, v = (torch.empty((pages, page, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        k[first:], v[first:] = rows[0], rows[1]
        where, kv_len = (page, dev(table + first), cap, pages), dev(np.array([190, 61], np.int32))
        mass, kept = torch.zeros((1, B, Hkv, cap * page), device="cuda"), torch.zeros((1, B, Hkv, 60), dtype=torch.int32, device="cuda")
        ctx.cast_attention_mass(q, k, B, 1, 0, 0, Hq, Hkv, D, *where, None, dev(np.array([8, 3], np.int32)), kv_len, 0.0, mass)
        ctx.cast_evict_kv(k, v, B, 1, 0, Hkv, D, *where, 60, 10, mass, kept, kv_len)
        assert ctx.cast_poll_status()[0] == 0
        results.append((k[first:].clone(), v[first:].clone(), mass, kept, kv_len))
        del k, v
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert not torch.equal(results[1][0], rows[0])


@pytest.mark.parametrize("kind,dtype", [("16", "bf16"), ("4", "bf16"), ("4", "f32")])
def test_mass_workspace_serves_smaller_calls(binding, kind, dtype):
    """Reserved once for the most sequences, layers and rows, as a server does: calls with fewer of each (among them those
    that divide a sequence into more pieces), shorter caches and fewer kv-heads run, and give the bits they give after a
    reservation of their own."""
    rng = np.random.default_rng(14)
    Bmax, nlmax, T, Hq, Hkv, D, H = 10, 16, 9, 8, 8, 64, 6
    ctx = context(binding, Bmax, T, H)
    ctx.cast_reserve_attention_mass(DT[dtype], Bmax, nlmax, H + 1, Hq, Hkv, D, 16, 20)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    pieces = {b: b * nlmax * Hkv * min(3, -(-8 * sms // (b * nlmax * Hkv))) for b in range(1, Bmax + 1)}
    assert max(pieces.values()) > pieces[Bmax]  # the case at hand: a smaller call that needs more
    for B, nl, heads, cap in [(b, nlmax, Hkv, 20) for b in range(Bmax, 0, -1)] + [(Bmax, 9, Hkv, 20), (Bmax, 1, Hkv, 20), (7, 11, 5, 20), (1, 1, 1, 20), (9, nlmax, Hkv, 17)]:
        paged = o4.Paged(rng, B, cap * 16, 16)
        cache = Cache(rng, paged, nl, heads, D) if kind == "4" else Dense(rng, paged, nl, heads, D, dtype)
        q = torch.randn((nl, B, T, heads, D), generator=torch.Generator("cuda").manual_seed(B), device="cuda").to(DT[dtype])
        path, alen = np.tile(np.arange(H + 1, dtype=np.int32), (B, 1)), rng.integers(0, H + 1, B).astype(np.int32)
        kv_len = rng.integers(H + 1, cap * 16 + 1, B).astype(np.int32)
        mass, want = (torch.zeros((nl, B, heads, paged.positions), device="cuda") for _ in range(2))
        qs, rest = q[0].numel() * q.element_size(), (dev(path), dev(alen), dev(kv_len), 0.0, mass)
        if kind == "4":
            ctx.cast_attention_mass_q4(q, cache.kc, cache.kr, B, nl, qs, *cache.strides, heads, heads, D, *cache.where(), *rest)
        else:
            ctx.cast_attention_mass(q, cache.k, B, nl, qs, cache.stride, heads, heads, D, *cache.where(), *rest)
        assert ctx.cast_poll_status()[0] == 0
        own = context(binding, B, T, H)
        run_mass(own, cache, q, path, alen, kv_len, want)
        assert own.cast_poll_status()[0] == 0
        assert torch.equal(mass, want) and bool((mass.sum((0, 2, 3)) > 0).all())


def test_mass_refuses(binding):
    rng = np.random.default_rng(9)
    B, T, Hq, Hkv, D, H = 5, 16, 4, 2, 128, 4
    paged = o4.Paged(rng, B, 96, 16)
    paged.table[4, 1] = -3
    cache = Dense(rng, paged, 1, Hkv, D, "bf16")
    q = torch.randn((1, B, T, Hq, D), device="cuda").to(torch.bfloat16)
    ok = np.tile(np.arange(H + 1, dtype=np.int32), (B, 1))
    good = dict(path=ok, alen=np.array([2] * B, np.int32), kv_len=np.array([50] * 4 + [15], np.int32))

    def run(expect, b, **kw):
        a = {k: v.copy() for k, v in good.items()}
        for k, v in kw.items():
            a[k][b] = v
        ctx = context(binding, B, T, H)
        mass = torch.zeros((1, B, Hkv, paged.positions), device="cuda")
        run_mass(ctx, cache, q, a["path"], a["alen"], a["kv_len"], mass)
        assert ctx.cast_poll_status()[0] == expect
        rest = [i for i in range(B) if i != b]
        check_mass(mass[:, rest], torch.zeros_like(mass[:, rest]), Sub(cache, rest), q[:, rest], a["path"][rest], a["alen"][rest], a["kv_len"][rest])
        return mass[:, b]

    class Sub:
        def __init__(self, c, rest):
            self.c, self.rest, self.Hkv = c, rest, c.Hkv

        def rows(self, which, l, b, h, n):
            return self.c.rows(which, l, self.rest[b], h, n)

    assert not run(0, 0, alen=-1).any()
    assert not run(6, 1, alen=H + 1).any()          # more rows than a path holds
    assert not run(6, 1, path=[0, T, 2, 3, 4]).any()
    assert not run(6, 2, path=[0, 1, -1, 3, 4]).any()
    assert not run(6, 0, kv_len=2).any()            # fewer positions than rows
    assert not run(7, 3, kv_len=97).any()           # past the capacity
    m = run(7, 4, kv_len=50)                        # a bad page: its positions count as masked
    assert not m[0, :, 16:32].any() and bool((m[0, :, :16] > 0).all())
    ctx = context(binding, B, T, H)
    with pytest.raises(binding.CastError) as e:
        run_mass(ctx, cache, q, ok, good["alen"], good["kv_len"], torch.zeros((1, B, Hkv, 96), device="cuda"), rows=1)
    assert e.value.code == 3
    with pytest.raises(TypeError):
        run_mass(ctx, cache, q, ok, good["alen"], good["kv_len"], torch.zeros((1, B, Hkv, 96), device="cuda", dtype=torch.float64))


# ------------------------------------------------------------------------------------------------ eviction
EVICT = [  # cache, dtype, Hkv, D, page, budget, recent, lengths
    ("16", "bf16", 8, 128, 16, 40, 8, [100, 40, 41, 0]),
    ("16", "bf16", 2, 64, 0, 300, 0, [1000, 299, 301]),
    ("16", "f32", 2, 128, 7, 33, 33, [200, 34]),
    ("16", "f32", 1, 64, 24, 1, 0, [2500, 1, 2]),
    ("4", "bf16", 8, 128, 16, 40, 8, [100, 40, 41, 0]),
    ("4", "bf16", 3, 64, 0, 700, 123, [4001, 2048, 700]),
    ("4", "bf16", 1, 128, 5, 64, 1, [640, 65]),
    ("16", "bf16", 1, 128, 64, 1999, 500, [9000, 2000]),
]


@pytest.mark.parametrize("weights", ["spread", "ties", "odd"])
@pytest.mark.parametrize("kind,dtype,Hkv,D,page,budget,recent,lens", EVICT)
def test_eviction(binding, kind, dtype, Hkv, D, page, budget, recent, lens, weights):
    rng = np.random.default_rng(D + page + budget)
    B, nl = len(lens), 2
    paged = o4.Paged(rng, B, max(lens) + 3, page)
    cache = Cache(rng, paged, nl, Hkv, D) if kind == "4" else Dense(rng, paged, nl, Hkv, D, dtype)
    P = paged.positions
    m = np.exp(rng.normal(0, 3, (nl, B, Hkv, P))).astype(np.float32)
    if weights == "ties":
        m = rng.integers(0, 3, m.shape).astype(np.float32)
    if weights == "odd":
        m[rng.random(m.shape) < 0.2] = np.nan
        m[rng.random(m.shape) < 0.2] = np.inf
        m[rng.random(m.shape) < 0.2] = -np.inf
        m[rng.random(m.shape) < 0.2] = -0.0
        m[rng.random(m.shape) < 0.2] = 0.0
        m[rng.random(m.shape) < 0.1] = np.float32(1e-42)
    mass, lengths = dev(m), np.array(lens, np.int32)
    kept, kv_len = torch.full((nl, B, Hkv, budget), -9, dtype=torch.int32, device="cuda"), dev(lengths)
    ctx = context(binding, B)
    args = (*cache.where(), budget, recent, mass, kept, kv_len)
    if kind == "4":
        bufs = [t.clone().cpu().numpy() if t.dtype == torch.uint8 else t.view(torch.int16).clone().cpu().numpy() for t in (cache.kc, cache.kr, cache.vc, cache.vr)]
        ctx.cast_evict_kv_q4(cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides, B, nl, Hkv, D, *args)
        got = cache.bits()
    else:
        as_int = torch.int16 if dtype == "bf16" else torch.int32
        bufs = [t.view(as_int).cpu().numpy().copy() for t in (cache.k, cache.v)]
        ctx.cast_evict_kv(cache.k, cache.v, B, nl, cache.stride, Hkv, D, *args)
        got = [t.view(as_int).cpu().numpy() for t in (cache.k, cache.v)]
    assert ctx.cast_poll_status()[0] == 0
    want_m, want_k = m.copy(), np.full((nl, B, Hkv, budget), -1, np.int32)
    for l in range(nl):
        for b in range(B):
            for h in range(Hkv):
                pos = o4.keep(m[l, b, h], lens[b], budget, recent)
                want_k[l, b, h, :len(pos)] = pos
                if lens[b] <= budget:
                    continue
                want_m[l, b, h, :len(pos)] = m[l, b, h, pos]
                want_m[l, b, h, len(pos):lens[b]] = 0
                src, to = paged.at(b, pos), paged.at(b, np.arange(len(pos)))
                for buf in bufs:
                    a = buf[l][:, h] if kind == "4" else buf[l][:, :, h]
                    a[to] = a[src]
    np.testing.assert_array_equal(kept.cpu().numpy(), want_k)
    np.testing.assert_array_equal(mass.cpu().numpy().view(np.int32), want_m.view(np.int32))
    np.testing.assert_array_equal(kv_len.cpu().numpy(), np.minimum(lengths, budget))
    for a, w in zip(got, bufs):
        np.testing.assert_array_equal(a, w)


def test_eviction_refuses(binding):
    rng = np.random.default_rng(5)
    B = 4
    paged = o4.Paged(rng, B, 64, 8)
    paged.table[0, 7], paged.table[1, 3] = paged.pages, -1   # the first lies behind the sequence's length
    cache = Dense(rng, paged, 1, 2, 64, "bf16")
    k, v = cache.k.clone(), cache.v.clone()
    mass = torch.rand((1, B, 2, 64), device="cuda")
    m = mass.clone()
    kept, kv_len = torch.zeros((1, B, 2, 10), dtype=torch.int32, device="cuda"), dev(np.array([50, 50, 65, -1], np.int32))
    ctx = context(binding, B)

    def call(budget=10, recent=2, D=64, B=B, n_layers=1):
        ctx.cast_evict_kv(cache.k, cache.v, B, n_layers, cache.stride, 2, D, *cache.where(), budget, recent, mass, kept, kv_len)

    for kw, code in ((dict(budget=0, recent=0), 1), (dict(recent=11), 1), (dict(recent=-1), 1), (dict(D=32), 2), (dict(B=5), 3), (dict(n_layers=0), 1)):
        with pytest.raises(binding.CastError) as e:
            call(**kw)
        assert e.value.code == code, kw
    call()
    assert ctx.cast_poll_status()[0] == 7
    np.testing.assert_array_equal(kv_len.cpu().numpy(), [10, 50, 65, -1])
    assert bool((kept[:, 1:] == -1).all()) and bool((kept[0, 0] >= 0).all())
    assert torch.equal(mass[:, 1:], m[:, 1:])
    other = np.unique(np.concatenate([paged.table[b][(paged.table[b] >= 0) & (paged.table[b] < paged.pages)] for b in (1, 2, 3)]))
    assert torch.equal(cache.k[0, other], k[0, other]) and torch.equal(cache.v[0, other], v[0, other])


@pytest.mark.parametrize("kind", ["16", "4"])
@pytest.mark.parametrize("captured", [False, True])
def test_mass_then_eviction_then_attention(binding, kind, captured):
    """As a program uses them: the accepted rows' weights of all layers, then the cut, then the next step's attention over what is
    left - captured and replayed, and from another stream."""
    rng = np.random.default_rng(31)
    B, nl, T, Hq, Hkv, D, H, budget, recent = 2, 2, 9, 8, 2, 128, 5, 120, 20
    paged = o4.Paged(rng, B, 330, 16)
    cache = Cache(rng, paged, nl, Hkv, D) if kind == "4" else Dense(rng, paged, nl, Hkv, D, "bf16")
    ctx = context(binding, B, T, H)
    (ctx.cast_reserve_attention_q4 if kind == "4" else ctx.cast_reserve_attention)(torch.bfloat16, B, Hq, Hkv, D, paged.page, paged.cap)
    ctx.cast_reserve_attention_mass(torch.bfloat16, B, nl, H + 1, Hq, Hkv, D, paged.page, paged.cap)
    path, alen = np.tile(np.arange(H + 1, dtype=np.int32), (B, 1)), np.array([4, 0], np.int32)
    lens = np.array([300, 101], np.int32)
    q = torch.randn((nl, B, T, Hq, D), generator=torch.Generator("cuda").manual_seed(6), device="cuda").to(torch.bfloat16)
    mass, kept = torch.zeros((nl, B, Hkv, paged.positions), device="cuda"), torch.zeros((nl, B, Hkv, budget), dtype=torch.int32, device="cuda")
    rows = {w: [[[cache.rows(w, l, b, h, lens[b])[0] for h in range(Hkv)] for b in range(B)] for l in range(nl)] for w in "kv"}
    start = [t.clone() for t in ((cache.kc, cache.kr, cache.vc, cache.vr) if kind == "4" else (cache.k, cache.v))]
    kv_len, out = dev(lens), torch.zeros_like(q[0])
    none = torch.zeros((B, T, 1), dtype=torch.int32, device="cuda")  # masks that leave the prefix alone
    n_tree, path_d, alen_d, where, qs = dev(np.array([T, T], np.int32)), dev(path), dev(alen), cache.where(), q[0].numel() * 2

    def step():
        if kind == "4":
            ctx.cast_attention_mass_q4(q, cache.kc, cache.kr, B, nl, qs, *cache.strides, Hq, Hkv, D, *where, path_d, alen_d, kv_len, 0.0, mass)
            ctx.cast_evict_kv_q4(cache.kc, cache.kr, cache.vc, cache.vr, *cache.strides, B, nl, Hkv, D, *where, budget, recent, mass, kept, kv_len)
            ctx.cast_tree_attention_q4(q[1], cache.kc[1], cache.kr[1], cache.vc[1], cache.vr[1], B, Hq, Hkv, D, *where, kv_len, none, n_tree, None, 0.0, out)
        else:
            ctx.cast_attention_mass(q, cache.k, B, nl, qs, cache.stride, Hq, Hkv, D, *where, path_d, alen_d, kv_len, 0.0, mass)
            ctx.cast_evict_kv(cache.k, cache.v, B, nl, cache.stride, Hkv, D, *where, budget, recent, mass, kept, kv_len)
            ctx.cast_tree_attention(q[1], cache.k[1], cache.v[1], B, Hq, Hkv, D, *where, kv_len, none, n_tree, 0.0, out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        for _ in range(2):  # the second pass from the same start
            for t, s in zip((cache.kc, cache.kr, cache.vc, cache.vr) if kind == "4" else (cache.k, cache.v), start):
                t.copy_(s)
            kv_len.copy_(torch.from_numpy(lens))
            mass.zero_()
            graph.replay() if captured else step()
    side.synchronize()
    assert ctx.cast_poll_status()[0] == 0
    np.testing.assert_array_equal(kv_len.cpu().numpy(), [budget, 101])
    x, got = q.double().cpu().numpy(), out.double().cpu().numpy()
    for l in range(nl):
        for b in range(B):
            n = int(alen[b]) + 1
            for h in range(Hkv):
                add = o4.mass_of(x[l, b, :n, h * 4:h * 4 + 4], rows["k"][l][b][h], lens[b] - n + np.arange(n) + 1, D ** -0.5)
                mine = kept[l, b, h].cpu().numpy()
                mine = mine[mine >= 0]
                left = np.setdiff1d(np.arange(lens[b]), mine)
                assert len(mine) == min(budget, lens[b]) and (np.diff(mine) > 0).all()
                if len(left):  # nothing that left outweighs what stayed of the older ones, but for the weights' error
                    old = mine[mine < lens[b] - recent]
                    assert add[left].max() <= add[old].min() * (1 + 1e-4) and left.max() < lens[b] - recent
                if l == 1:
                    k, v = rows["k"][l][b][h][mine], rows["v"][l][b][h][mine]
                    want, _ = o4.attend(x[1, b, :, h * 4:h * 4 + 4], k, v, v, len(mine), np.zeros((T, 0), bool), D ** -0.5)
                    assert np.abs(got[b, :, h * 4:h * 4 + 4] - want).max() < 2e-2


def test_early_reads_beside_the_new_calls(binding):
    """With early reads promised: attention over the 16-bit cache right behind rows that came out of a 4-bit cache, behind the
    weights of the accepted rows, and behind an eviction - with the bits of a context without the promise that waits for
    every call."""
    rng = np.random.default_rng(40)
    B, cap, T, Hq, Hkv, D, H, budget = 4, 2048, 12, 32, 8, 128, 4, 700
    paged = o4.Paged(rng, B, cap, 0)
    stores = [Cache(rng, paged, 1, Hkv, D) for _ in range(2)]
    q = torch.randn((1, B, T, Hq, D), generator=torch.Generator("cuda").manual_seed(9), device="cuda").to(torch.bfloat16)
    lens = np.array([2030, 1500, 701, 12], np.int32)
    anc = torch.ones((B, T, 1), dtype=torch.int32, device="cuda")
    n_tree, all_rows, path, alen = dev(np.full(B, T, np.int32)), dev(np.full(B, cap, np.int32)), dev(np.tile(np.arange(H + 1, dtype=np.int32), (B, 1))), dev(np.array([4, 2, 0, 1], np.int32))

    def run(promise):
        ctx = context(binding, B, T, H)
        ctx.cast_reserve_attention(torch.bfloat16, B, Hq, Hkv, D, 0, cap)
        ctx.cast_reserve_attention_mass(torch.bfloat16, B, 1, H + 1, Hq, Hkv, D, 0, cap)
        ctx.cast_set_attention_early_reads(promise)
        k, v = (torch.zeros((1, B, cap, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        where, kv_len = (0, None, cap, 0), dev(lens)
        mass, kept = torch.zeros((1, B, Hkv, cap), device="cuda"), torch.zeros((1, B, Hkv, budget), dtype=torch.int32, device="cuda")
        outs = torch.zeros((12, *q.shape), dtype=torch.bfloat16, device="cuda")
        at = iter(outs)
        torch.cuda.synchronize()

        def between():
            if not promise:
                torch.cuda.synchronize()

        def attend():
            between()
            ctx.cast_tree_attention(q[0], k[0], v[0], B, Hq, Hkv, D, *where, kv_len, anc, n_tree, 0.0, next(at)[0])
            between()

        for c in stores + stores:
            ctx.cast_load_kv_q4(c.kc, c.kr, c.vc, c.vr, *c.strides, B, 1, cap, Hkv, D, *where, None, all_rows, k, v)
            attend()
            ctx.cast_attention_mass(q, k, B, 1, q.numel() * 2, k.numel() * 2, Hq, Hkv, D, *where, path, alen, kv_len, 0.0, mass)
            attend()
            ctx.cast_evict_kv(k, v, B, 1, k.numel() * 2, Hkv, D, *where, budget, 100, mass, kept, kv_len)
            attend()
        assert ctx.cast_poll_status()[0] == 0
        np.testing.assert_array_equal(kv_len.cpu().numpy(), np.minimum(lens, budget))
        return outs, mass, kept

    for a, b in zip(run(True), run(False)):
        assert torch.equal(a, b) and bool(a.any())
