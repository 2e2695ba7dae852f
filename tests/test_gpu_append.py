"""cast_append_kv against 64 bits: norm per head, rotation, and where the rows go."""
import numpy as np
import pytest
import torch

import chunk_oracle as co
import q4_oracle as o4

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step, relative to the value
EPS = 1e-6


@pytest.fixture(scope="module")
def binding():
    from paper_2510_26577_b200 import build
    build.build()
    from paper_2510_26577_b200 import binding as b
    b.load_library()
    return b


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def context(binding, B):
    return binding.CastContext(max_batch=B, vocab=1000, top_k=4, max_depth=6, total_token=8, max_tree=8)


def split(x, Hq, Hkv, D):
    """Views of a fused projection's output [.., (Hq + 2 Hkv) D]."""
    q, k, v = x.split([Hq * D, Hkv * D, Hkv * D], -1)
    return q.unflatten(-1, (Hq, D)), k.unflatten(-1, (Hkv, D)), v.unflatten(-1, (Hkv, D))


def close(got, x, want, dtype, magnitude):
    """Half a step of the output, and of 32 bits: the sum of squares is off by D / 2 + 4 half steps at most and the root, the weight and
    the product by 8 more, (D / 2 + 12) 2^-24 < 2^-17.7 of the value; the turns' fraction, doubled, by half a step of a number up to 1,
    an angle of pi 2^-24, sine and cosine by 2^-23 and the products by 3 2^-24, below 2^-21 of the pair's size. `want`: the values,
    and the pair's size."""
    value, pair = want
    np.testing.assert_allclose(got, value, rtol=0, atol=0) if pair is None else None
    if pair is not None:
        err = np.abs(got - value)
        tol = HALF[dtype] * np.abs(value) + (2.0 ** -17.7 + 2.0 ** -21) * pair * magnitude
        assert not (err > tol * 1.001 + 1e-30).any(), (np.nanmax(err - tol), np.nanmax(err))


def turned(x, weight, pos, inv, interleaved, magnitude):
    """What queries or keys become, and the size of the pairs (|a| + |b|) that their errors count in."""
    y = co.normalised(x, weight, EPS)
    r = 2 * len(inv)
    size = np.abs(y)
    if r:
        lo = np.arange(0, r, 2) if interleaved else np.arange(r // 2)
        hi = lo + (1 if interleaved else r // 2)
        both = size[..., lo] + size[..., hi]
        size[..., lo], size[..., hi] = both, both
    return co.rotated(y, pos, inv, interleaved, magnitude), size


CASES = [  # dtype, Hq, Hkv, D, page, rows, rot, interleaved, norm, packed, tree, offset
    ("bf16", 32, 8, 128, 16, 60, 128, False, True, False, True, 0),
    ("bf16", 32, 8, 128, 16, 1, 64, True, False, False, False, 100000),
    ("bf16", 28, 4, 128, 24, 333, 128, False, True, True, False, 0),
    ("bf16", 8, 8, 64, 0, 65, 64, True, True, True, False, 2000000000),
    ("bf16", 7, 1, 64, 1, 19, 24, False, False, False, False, 7),      # half of the pairs' distance is no piece of 16 bytes
    ("bf16", 5, 5, 128, 7, 33, 2, False, True, True, False, 0),
    ("bf16", 130, 1, 64, 16, 9, 0, False, True, False, False, 0),       # the norm alone
    ("bf16", 4, 2, 128, 64, 40, 0, False, False, False, False, 0),      # a plain store
    ("bf16", 4, 4, 128, 8, 700, 40, True, False, True, False, 0),
    ("f32", 8, 8, 64, 24, 33, 64, False, True, False, True, 0),
    ("f32", 6, 2, 128, 0, 50, 100, False, True, True, False, 123456),
    ("f32", 3, 3, 128, 16, 12, 128, True, False, False, False, 0),
]


@pytest.mark.parametrize("dtype,Hq,Hkv,D,page,rows,rot,inter,norm,packed,tree,offset", CASES)
def test_append(binding, dtype, Hq, Hkv, D, page, rows, rot, inter, norm, packed, tree, offset):
    rng = np.random.default_rng(Hq * 100 + rows)
    B = 5
    n = np.array([rows, 0, max(1, rows // 3), rows, rows // 2], np.int32)
    first = np.array([0, 0, 0, rows // 2, 3], np.int32)
    start = np.array([37, 5, 0, 64, 9], np.int32)
    order = [3, 0, 4, 1, 2]  # packed: not in the order of the sequences, with rows between them that belong to nobody
    row0 = np.arange(B) * rows
    total = B * rows
    if packed:
        at = 2
        for b in order:
            row0[b] = at
            at += n[b] + 1
        total = at + 3
    paged = o4.Paged(rng, B, rows + 70, page)
    gen = torch.Generator("cuda").manual_seed(rows)
    x = torch.randn((total, (Hq + 2 * Hkv) * D), generator=gen, device="cuda").mul_(2).to(DT[dtype])
    x[row0[2]:row0[2] + 1, (Hq + Hkv) * D] = float("inf")  # values are moved as they are
    q, k, v = split(x if packed else x.view(B, rows, -1), Hq, Hkv, D)
    depth = rng.integers(0, 9, (B, rows)).astype(np.int32) if tree else None
    inv = 10000.0 ** (-np.arange(0, rot, 2) / max(rot, 1))
    w = [dev((1 + 0.3 * rng.normal(size=D)).astype(np.float32)) if norm else None for _ in range(2)]
    position = (start + offset).astype(np.int32) if offset else None
    magnitude = 1.25 if inter else 0.0
    shape = (paged.pages, page, Hkv, D) if page else (B, paged.cap, Hkv, D)
    kc, vc = (torch.full(shape, -77.0, device="cuda").to(DT[dtype]) for _ in range(2))
    q_out = torch.full((total, Hq, D), -77.0, device="cuda").to(DT[dtype])
    ctx = context(binding, B)
    stride = x.stride(0) * x.element_size()
    ctx.cast_append_kv(q, stride, k, stride, v, stride, B, total if packed else rows, Hq, Hkv, D, dev(row0.astype(np.int32)) if packed else None,
                       dev(first), dev(n), dev(depth), dev(position), dev(inv) if rot else None, rot, int(inter), magnitude, w[0], w[1], EPS,
                       page, dev(paged.table), paged.cap, paged.pages, dev(start), q_out, kc, vc)
    assert ctx.cast_poll_status()[0] == 0
    want_k, want_v = (torch.full(shape, -77.0).to(DT[dtype]) for _ in range(2))
    touched = np.zeros(total, bool)
    host = [t.reshape(total, -1, D).double().cpu().numpy() for t in (q, k)]
    got_q, got_k = q_out.double().cpu().numpy(), kc.double().cpu().numpy()
    seen_k = np.zeros(shape[:2], bool)
    for b in range(B):
        t = np.arange(min(first[b], n[b]), n[b])
        r = row0[b] + t
        touched[r] = True
        pos = start[b].astype(np.int64) + offset + (depth[b, t] if tree else t)
        m = magnitude or 1.0
        pg, sl = paged.at(b, start[b] + t)
        seen_k[pg, sl] = True
        want_v[pg, sl] = v.reshape(total, Hkv, D)[r].cpu()
        for rows_in, got, weight in ((host[0][r], got_q[r], w[0]), (host[1][r], got_k[pg, sl], w[1])):
            value, pair = turned(rows_in, None if weight is None else weight.cpu().numpy(), pos, inv, inter, m)
            close(got, rows_in, (value, pair if norm or rot else None), dtype, max(m, 1.0))
    assert (got_q[~touched] == -77.0).all() and (got_k[~seen_k] == -77.0).all()
    assert torch.equal(vc.cpu().view(torch.uint8), want_v.view(torch.uint8))


@pytest.mark.parametrize("seed", range(12))
def test_append_mixes(binding, seed):
    """Any rotation, heads that fill no whole piece, few rows and more than the device has warps."""
    rng = np.random.default_rng(500 + seed)
    dtype, D = ["bf16", "bf16", "f32"][seed % 3], [64, 128][seed % 2]
    Hq, Hkv = int(rng.integers(1, 20)), int(rng.integers(1, 9))
    rows = [1, 3, 40, 900][int(rng.integers(0, 4))] if seed else 1500
    rot = int(rng.choice([0, 2, 8, 12, 16, 20, 40, D // 2, D - 4, D]))
    test_append(binding, dtype, Hq, Hkv, D, int(rng.choice([0, 3, 16, 64])), rows, rot, bool(rng.integers(0, 2)), bool(rng.integers(0, 2)), seed % 2 == 1, False,
                int(rng.choice([0, 5000])))


def simple(ctx, q, k, v, B, rows, Hq, Hkv, D, n, cap, start, q_out, kc, vc, inv, **kw):
    e = k.element_size() if k is not None else q.element_size()
    a = dict(row_start=None, first=None, depth=None, position=None, page=0, table=None, pages=0)
    a.update(kw)
    ctx.cast_append_kv(q, Hq * D * e, k, Hkv * D * e, v, Hkv * D * e, B, rows, Hq, Hkv, D, a["row_start"], a["first"], n, a["depth"], a["position"],
                       inv, 0 if inv is None else 2 * inv.numel(), 0, 1.0, None, None, EPS, a["page"], a["table"], cap, a["pages"], start, q_out, kc, vc)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parts_and_in_place(binding, dtype):
    """Queries alone, in place; keys and values alone, into a dense buffer: the bits of the whole call."""
    B, rows, Hq, Hkv, D = 2, 50, 6, 2, 128
    q, k, v = (torch.randn((B, rows, h, D), device="cuda").to(DT[dtype]) for h in (Hq, Hkv, Hkv))
    n, inv = dev(np.array([50, 31], np.int32)), dev(10000.0 ** (-np.arange(64) / 64))
    pos = dev(np.array([1000, 0], np.int32))
    ctx = context(binding, B)
    q_out, kc, vc = q.clone(), torch.zeros_like(k), torch.zeros_like(v)
    simple(ctx, q, k, v, B, rows, Hq, Hkv, D, n, rows, None, q_out, kc, vc, inv, position=pos)
    k2, v2, mine = torch.zeros_like(k), torch.zeros_like(v), q.clone()
    simple(ctx, None, k, v, B, rows, Hq, Hkv, D, n, rows, None, None, k2, v2, inv, position=pos)
    simple(ctx, mine, None, None, B, rows, Hq, Hkv, D, n, rows, None, mine, None, None, inv, position=pos)
    assert ctx.cast_poll_status()[0] == 0
    for a, b in ((q_out, mine), (kc, k2), (vc, v2)):
        assert torch.equal(a, b)
    assert torch.equal(q_out[1, 31:], q[1, 31:]) and not torch.equal(q_out, q)
    assert torch.equal(vc[0], v[0]) and bool((vc[1, 31:] == 0).all())


def test_places_outside_are_refused(binding):
    B, rows, Hq, Hkv, D = 5, 8, 2, 1, 64
    q, k, v = (torch.randn((B, rows, h, D), device="cuda") for h in (Hq, Hkv, Hkv))
    table = np.arange(B * 4).reshape(B, 4).astype(np.int32)
    table[1, 2], table[2, 0] = B * 4, -1
    start = dev(np.array([28, 12, 2, -3, 0], np.int32))  # 0 runs past its 32 positions; 1, 2 into bad pages; 3 begins below 0
    n = dev(np.full(B, rows, np.int32))
    ctx = context(binding, B)
    for b in range(B):
        only = dev(np.where(np.arange(B) == b, rows, 0).astype(np.int32))
        q_out, kc, vc = torch.zeros_like(q), torch.zeros(B * 4, 8, Hkv, D, device="cuda"), torch.zeros(B * 4, 8, Hkv, D, device="cuda")
        simple(ctx, q, k, v, B, rows, Hq, Hkv, D, only, 4, start, q_out, kc, vc, None, page=8, table=dev(table), pages=B * 4)
        status, detail = ctx.cast_poll_status()
        assert (status, detail) == ((7, b) if b < 4 else (0, 0))
        assert torch.equal(q_out[b], q[b])  # queries do not depend on it
        stored = [t for t in range(rows) if (p := int(start[b]) + t) >= 0 and p < 32 and 0 <= table[b, p // 8] < B * 4]
        assert len(stored) == (4, 4, 2, 5, 8)[b]
        assert int((vc != 0).any(-1).sum()) == len(stored)
        for t in stored:
            p = int(start[b]) + t
            assert torch.equal(vc[table[b, p // 8], p % 8], v[b, t]) and torch.equal(kc[table[b, p // 8], p % 8], k[b, t])
    # packed rows outside the buffer: the sequence is left out
    for row_start, bad in ((np.array([0, 8, 33, 16, 24]), 2), (np.array([0, 8, -1, 16, 24]), 2)):
        vc = torch.zeros(B, 32, Hkv, D, device="cuda")
        simple(ctx, q, k, v, B, B * rows, Hq, Hkv, D, n, 32, None, q_out, torch.zeros_like(vc), vc, None, row_start=dev(row_start.astype(np.int32)))
        assert ctx.cast_poll_status() == (6, bad)
        assert bool((vc[bad] == 0).all()) and bool((vc[[0, 1, 3, 4], :8] != 0).all())


def test_refusals(binding):
    ctx = context(binding, 2)
    B, rows, Hq, Hkv, D = 2, 4, 2, 1, 64
    q, k, v = (torch.randn((B, rows, h, D), device="cuda") for h in (Hq, Hkv, Hkv))
    n, inv, kc = dev(np.full(B, rows, np.int32)), dev(np.ones(16)), torch.zeros(B, rows, Hkv, D, device="cuda")
    base = dict(q=q, qs=Hq * D * 4, k=k, ks=Hkv * D * 4, v=v, vs=Hkv * D * 4, B=B, rows=rows, Hq=Hq, Hkv=Hkv, D=D, n=n, inv=inv, rot=32, eps=EPS,
                page=0, table=None, cap=rows, pages=0, q_out=q.clone(), kc=kc, vc=kc.clone(), qw=None)

    def call(**kw):
        a = {**base, **kw}
        ctx.cast_append_kv(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["B"], a["rows"], a["Hq"], a["Hkv"], a["D"], None, None, a["n"], None, None,
                           a["inv"], a["rot"], 0, 1.0, a["qw"], None, a["eps"], a["page"], a["table"], a["cap"], a["pages"], None, a["q_out"], a["kc"], a["vc"])

    call()
    for code, kw in ((1, dict(n=None)), (1, dict(q=None, k=None, v=None)), (1, dict(v=None)), (1, dict(q_out=None)), (1, dict(kc=None)), (1, dict(inv=None)),
                     (1, dict(rot=-2)), (1, dict(eps=-1.0)), (1, dict(eps=float("nan"))), (1, dict(B=0)), (1, dict(rows=0)), (1, dict(cap=0)),
                     (1, dict(page=8)), (1, dict(page=-1)), (2, dict(D=32)), (2, dict(rot=33)), (2, dict(rot=66)), (3, dict(B=3)), (3, dict(rows=1 << 30)),
                     (4, dict(k=k.bfloat16(), ks=Hkv * D * 2)), (4, dict(q=q.half(), qs=Hq * D * 2)), (3, dict(cap=2 ** 31 - 1))):
        with pytest.raises(binding.CastError) as e:
            call(**kw)
        assert e.value.code == code, (kw, e.value)
    flat = torch.zeros(B * rows * Hq * D + 1, device="cuda")
    with pytest.raises(binding.CastError) as e:  # not aligned to 16 bytes
        call(q_out=flat[1:])
    assert e.value.code == 2
    for kw in (dict(qs=Hq * D * 4 + 16), dict(q=q.transpose(1, 2)), dict(q=q.cpu()), dict(q=q[..., ::2])):
        with pytest.raises(AssertionError):
            call(**kw)
    with pytest.raises(TypeError):
        call(inv=inv.float())
    assert ctx.cast_poll_status()[0] == 0


def test_rows_past_32_bits(binding):
    """A cache of more than 2^32 bytes, its last pages, and a projection's output of the same size."""
    B, rows, Hq, Hkv, D, page = 1, 3, 1, 8, 128, 16
    pages = (1 << 32) // (page * Hkv * D * 2) + 40
    kc, vc = (torch.zeros((pages, page, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    wide = torch.zeros(((1 << 32) // (8 * D * 2) // 1000 + 1, 1000, 8, D), dtype=torch.bfloat16, device="cuda").view(-1, 8, D)
    total = wide.shape[0]
    wide[total - rows:] = torch.randn((rows, 8, D), device="cuda").bfloat16()
    table = dev(np.array([[pages - 1, pages - 2]], np.int32))
    ctx = context(binding, B)
    ctx.cast_append_kv(None, 0, wide, 8 * D * 2, wide, 8 * D * 2, B, total, Hq, Hkv, D, dev(np.array([total - rows], np.int32)), None,
                       dev(np.array([rows], np.int32)), None, None, None, 0, 0, 1.0, None, None, EPS, page, table, 2, pages,
                       dev(np.array([14], np.int32)), None, kc, vc)
    assert ctx.cast_poll_status()[0] == 0
    for c in (kc, vc):
        assert torch.equal(c[pages - 1, 14:], wide[total - 3:total - 1]) and torch.equal(c[pages - 2, :1], wide[total - 1:])
        assert bool((c[:pages - 2] == 0).all())
