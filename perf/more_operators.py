"""New rows on their way into the cache, attention of chunks of new tokens over it, and attention under a sliding window, as
timed cases.

Every case is one pass through calls of `paper_2510_26577_b200.binding.CastContext`, as a serving loop makes them, or the same
operators in plain torch operations:

  append  queries, keys and values of new tokens as a projection leaves them: queries and keys normalised per head and rotated
          by their positions, keys and values stored in the cache
  chunk   causal attention of a chunk of new tokens per sequence over the paged cache, one token (decoding) to thousands (a
          prompt), where a window is given only over the last `window` positions and the first `sinks`
  tree    verification attention of a draft tree under such a window
  layers  both together, layer after layer: append, then the chunk's or the tree's attention

Rows of new tokens lie as [batch, rows, ...], or packed, sequence b's from row_start[b] on.
"""
import numpy as np
import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-6


def _case(kind, name=None, **kw):
    c = {} if name is None else {"name": name}
    c.update(kind=kind, **kw)
    return c


def _heads(q_heads, kv_heads, head_dim):
    return {"q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim}


def _where(page, lo, hi):
    return {"page": page, "prefix_lo": lo, "prefix_hi": hi}


def _rows(lo, hi, packed):
    return {"rows_lo": lo, "rows_hi": hi, "packed": packed}


def _rope(rot_dim, interleaved, norm, factor=1.0, offset=0):
    """factor: the context is stretched by so much; offset: positions that left the cache before what it holds."""
    return {"rot_dim": rot_dim, "interleaved": interleaved, "norm": norm, "factor": factor, "offset": offset}


def _mask(window, sinks):
    return {"window": window, "sinks": sinks}


LLAMA, NONE = _heads(32, 8, 128), _mask(0, 0)


def listed():
    return [
        # the 60 tree tokens of one user of an 8B model, one layer: a call in front of every layer's attention, latency alone
        _case("append", "append_tree_b1", dtype="bf16", layers=1, batch=1, tree=True, **_rows(60, 60, False), **LLAMA, **_where(16, 2048, 2048), **_rope(128, False, True)),
        # a decoding step of a loaded server, one token per sequence, pairs of neighbours, half of the head rotated, positions far out
        _case("append", "append_decode_b64", dtype="bf16", layers=4, batch=64, tree=False, **_rows(1, 1, False), **LLAMA, **_where(16, 512, 4096),
              **_rope(64, True, False, 8.0, 100000)),
        # chunks of prompts, ragged, packed, out of one fused projection
        _case("append", "append_prefill", dtype="bf16", layers=2, batch=4, tree=False, **_rows(1500, 4097, True), **LLAMA, **_where(16, 0, 4096), **_rope(128, False, True)),
        # a decoding step's attention, one token per sequence of a loaded server: bound by the cache
        _case("chunk", "chunk_decode_b64", dtype="bf16", layers=2, batch=64, **_rows(1, 1, False), **LLAMA, **_where(16, 512, 4096), **NONE),
        # a whole prompt of an 8B model
        _case("chunk", "chunk_prefill", dtype="bf16", layers=2, batch=1, **_rows(4096, 4096, False), **LLAMA, **_where(0, 0, 0), **NONE),
        # the next thousand tokens of two long prompts, a GQA group of seven: bound by the tensor cores
        _case("chunk", "chunk_long", dtype="bf16", layers=1, batch=2, **_rows(1000, 1000, False), **_heads(28, 4, 128), **_where(16, 32768, 32768), **NONE),
        # a mixed batch of a model with a window: prompts and decoding side by side, packed
        _case("chunk", "chunk_mixed_window", dtype="bf16", layers=2, batch=24, **_rows(1, 700, True), **_heads(64, 8, 128), **_where(32, 100, 8192), **_mask(1024, 4)),
        # a small model in 32 bits, heads of 64 dimensions, pages of an odd size
        _case("chunk", "chunk_f32_d64", dtype="f32", layers=2, batch=3, **_rows(20, 131, False), **_heads(8, 8, 64), **_where(24, 200, 900), **_mask(256, 1)),
        # one user's fixed tree of 60 tokens behind a long prefix
        _case("tree", "tree_window_b1", dtype="bf16", layers=4, batch=1, **_rows(60, 60, False), **LLAMA, **_where(16, 8192, 8192), **_mask(1024, 4)),
        # a loaded server, ragged: some sequences shorter than the window, some far longer
        _case("tree", "tree_window_b64", dtype="bf16", layers=2, batch=64, **_rows(6, 12, False), **LLAMA, **_where(16, 512, 8192), **_mask(2048, 64)),
        # four layers of a verification step under a window, from the projection's output on
        _case("layers", "layers_tree", dtype="bf16", layers=4, batch=8, tree=True, **_rows(30, 60, False), **LLAMA, **_where(16, 1024, 4096), **_mask(1024, 4),
              **_rope(128, False, True)),
        # two layers of a prompt's chunk
        _case("layers", "layers_prefill", dtype="bf16", layers=2, batch=3, tree=False, **_rows(500, 2000, True), **LLAMA, **_where(16, 0, 2048), **NONE,
              **_rope(128, False, False, 4.0)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def _draw_once(rng):
    kind = rng.choice(["append", "append", "chunk", "chunk", "chunk", "tree", "tree", "layers"])
    dtype = "f32" if rng.random() < 0.15 else "bf16"
    group, kv_heads = rng.choice([1, 2, 4, 4, 7, 8]), rng.choice([1, 2, 4, 8, 8])
    head_dim = 64 if rng.random() < 0.3 else 128
    tree = kind == "tree" or (kind in ("append", "layers") and rng.random() < 0.4)
    hi = _log_int(rng, 16, 32768)
    lo = hi if rng.random() < 0.3 else max(0 if not tree else 1, hi // rng.randint(2, 8))
    rows_hi = _log_int(rng, 1, 128) if tree else 1 if rng.random() < 0.3 else _log_int(rng, 2, 4097)
    rows_lo = rows_hi if rng.random() < 0.3 else max(1, rows_hi // rng.randint(2, 20))
    c = dict(dtype=dtype, layers=_log_int(rng, 1, 32), batch=_log_int(rng, 1, 64), **_rows(rows_lo, rows_hi, not tree and rng.random() < 0.5),
             **_heads(group * kv_heads, kv_heads, head_dim), **_where(rng.choice([0, 8, 16, 16, 24, 32, 64, 128]), lo, hi))
    if kind in ("append", "layers"):
        c.update(tree=tree, **_rope(rng.choice([head_dim, head_dim, head_dim // 2, 32, 24]), rng.random() < 0.4, rng.random() < 0.5,
                                    rng.choice([1.0, 1.0, 4.0, 32.0]), rng.choice([0, 0, 1000, 120000])))
    if kind != "append":
        c.update(_mask(0, 0) if kind != "tree" and rng.random() < 0.5 else _mask(_log_int(rng, 16, 4096), rng.choice([0, 1, 4, 64, 200])))
    return _case(kind, **c)


def _room(case):
    """Bytes that a plain pass and its inputs hold, roughly."""
    wide = case["q_heads"] + 2 * case["kv_heads"]
    cache = 2 * case["layers"] * case["batch"] * _capacity(case) * case["kv_heads"] * case["head_dim"] * SIZE[case["dtype"]]
    return cache + case["layers"] * case["batch"] * case["rows_hi"] * wide * case["head_dim"] * 24 + 4e9


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / (15 if case["dtype"] == "f32" else 200))


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _cost(c))
    while True:
        c = _draw_once(rng)
        if _cost(c) <= most[c["kind"]] and _room(c) <= 2e10:
            return c


# ---------------------------------------------------------------------------------------------------- inputs
def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=DTYPE[dtype])


def _capacity(case):
    """Positions reserved per sequence, in whole pages."""
    unit = case["page"] or 1
    return -(-(case["prefix_hi"] + case["rows_hi"]) // unit) * unit


def _trees(B, cap, depth, n_tree, rng):
    """Random rooted trees in creation order: depths [B, cap] and ancestor masks (host arrays)."""
    parent, level = np.full((B, cap), -1, np.int32), np.full((B, cap), -1, np.int32)
    anc = np.zeros((B, cap, (cap + 31) // 32), np.uint32)
    for b in range(B):
        for t in range(int(n_tree[b])):
            p = -1 if t == 0 else int(min(rng.integers(0, t), rng.integers(0, t)))  # early nodes have more children
            while p >= 0 and level[b, p] >= depth:
                p = parent[b, p]
            parent[b, t], level[b, t] = p, 0 if p < 0 else level[b, p] + 1
            if p >= 0:
                anc[b, t] = anc[b, p]
            anc[b, t, t >> 5] |= np.uint32(1 << (t & 31))
    return level, anc


def _frequencies(rot_dim, factor):
    """Angle per position of every pair, in 64 bits, and the factor on what is rotated: pairs that turn less than once in the
    original 8192 positions are slowed down by `factor`, those that turn 32 times or more are left alone, between them a ramp."""
    inv = 500000.0 ** (-np.arange(0, rot_dim, 2) / rot_dim)
    if factor == 1.0:
        return inv, 1.0
    turns = 8192 * inv / (2 * np.pi)
    keep = np.clip((turns - 1) / (32 - 1), 0, 1)
    return inv * (keep + (1 - keep) / factor), 0.1 * np.log(factor) + 1.0


def _decoding(case):
    """A mixed batch: every other sequence has one new token."""
    return case["packed"] and case["rows_lo"] == 1


class State:
    pass


def prepare(case, seed):
    gen, rng = torch.Generator(device="cuda"), np.random.Generator(np.random.Philox(seed))
    gen.manual_seed(seed)
    kind, dtype, B, nl, unit, Hq, Hkv, D = (case[k] for k in ("kind", "dtype", "batch", "layers", "page", "q_heads", "kv_heads", "head_dim"))
    s = State()
    s.case = case
    # the cache of all layers, its page table, the sequences' lengths
    positions = _capacity(case)
    s.seq_cap, s.pages, s.table = positions // (unit or 1), 0, None
    if unit:
        s.pages = B * s.seq_cap
        s.table = _dev(rng.permutation(s.pages).astype(np.int32).reshape(B, s.seq_cap))
    s.L = rng.integers(case["prefix_lo"], case["prefix_hi"] + 1, B)
    s.kv_len = _dev(s.L.astype(np.int32))
    shape = (nl, s.pages, unit, Hkv, D) if unit else (nl, B, positions, Hkv, D)
    s.k, s.v = _randn(shape, dtype, gen), _randn(shape, dtype, gen)
    # the new rows of every sequence
    s.n = rng.integers(case["rows_lo"], case["rows_hi"] + 1, B)
    if _decoding(case):
        s.n[::2] = 1
    s.n_rows = _dev(s.n.astype(np.int32))
    s.first = np.arange(B) * case["rows_hi"]
    s.total, s.rows, s.row_start = B * case["rows_hi"], case["rows_hi"], None
    if case["packed"]:
        s.first = np.concatenate([[0], np.cumsum(s.n)[:-1]])
        # a buffer for the most rows that come; what lies behind the last sequence belongs to nobody
        s.total = s.rows = B * case["rows_hi"] if not _decoding(case) else (B - B // 2) + (B // 2) * case["rows_hi"]
        s.row_start = _dev(s.first.astype(np.int32))
    s.depth = s.anc = None
    if kind == "tree" or case.get("tree"):
        level, anc = _trees(B, case["rows_hi"], 8, s.n, rng)
        s.level, s.depth, s.anc = level, _dev(level), _dev(anc.view(np.int32))
    if kind in ("append", "layers"):
        # one projection's output: queries, keys and values side by side in a row
        s.qkv = _randn((nl, s.total, (Hq + 2 * Hkv) * D), dtype, gen)
        inv, s.magnitude = _frequencies(case["rot_dim"], case["factor"])
        s.inv_freq = _dev(inv)
        s.q_weight = s.k_weight = None
        if case["norm"]:
            s.q_weight, s.k_weight = (1 + 0.3 * torch.randn(D, generator=gen, device="cuda") for _ in range(2))
        s.position = s.kv_len + case["offset"] if case["offset"] else None
        s.q = torch.zeros((nl if kind == "append" else 1, s.total, Hq, D), dtype=DTYPE[dtype], device="cuda")
    else:
        s.q = _randn((nl, s.total, Hq, D), dtype, gen)
    if kind != "append":
        s.out = torch.zeros((nl, s.total, Hq, D), dtype=DTYPE[dtype], device="cuda")
    if own:
        _context(s)
    else:
        _indices(s)
    return s


def _context(s):
    from paper_2510_26577_b200 import binding
    c = s.case
    tokens = c["rows_hi"] if s.anc is not None else 8
    s.ctx = binding.CastContext(max_batch=c["batch"], vocab=32000, top_k=8, max_depth=8, total_token=tokens, max_tree=tokens)
    if c["kind"] != "append":
        s.ctx.cast_reserve_chunk_attention(DTYPE[c["dtype"]], c["head_dim"])


def _indices(s):
    """What the plain forms index with: the live rows, their sequences, and the page and slot of every position."""
    c = s.case
    unit, B = c["page"], c["batch"]
    at = torch.arange(_capacity(c), device="cuda")
    s.page_of = s.table.long()[:, at // unit] if unit else torch.arange(B, device="cuda")[:, None].expand(B, len(at))
    s.slot_of = (at % unit if unit else at).expand(B, len(at))
    s.seq = _dev(np.repeat(np.arange(B), s.n))
    s.t = _dev(np.concatenate([np.arange(n) for n in s.n]))
    s.row = _dev(np.concatenate([f + np.arange(n) for f, n in zip(s.first, s.n)]))


def _split(s, layer):
    """The layer's queries, keys and values [rows, heads, D], views of the projection's output."""
    c, x = s.case, s.qkv[layer]
    Hq, Hkv, D = c["q_heads"], c["kv_heads"], c["head_dim"]
    return (x[:, :Hq * D].unflatten(1, (Hq, D)), x[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D)), x[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D)))


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _run_own(s):
    c = s.case
    B, nl, Hq, Hkv, D, page = (c[k] for k in ("batch", "layers", "q_heads", "kv_heads", "head_dim", "page"))
    cache = (page, s.table, s.seq_cap, s.pages)

    def append(layer, q_out):
        q, k, v = _split(s, layer)
        stride = s.qkv.stride(1) * s.qkv.element_size()
        s.ctx.cast_append_kv(q, stride, k, stride, v, stride, B, s.rows, Hq, Hkv, D, s.row_start, None, s.n_rows, s.depth, s.position,
                             s.inv_freq, c["rot_dim"], int(c["interleaved"]), s.magnitude, s.q_weight, s.k_weight, EPS, *cache, s.kv_len,
                             q_out, s.k[layer], s.v[layer])

    def attend(layer, q):
        if s.anc is not None:
            s.ctx.cast_tree_attention_window(q, s.k[layer], s.v[layer], B, Hq, Hkv, D, *cache, s.kv_len, s.anc, s.depth, s.n_rows, None,
                                             c["window"], c["sinks"], 0.0, s.out[layer])
        else:
            s.ctx.cast_chunk_attention(q, s.k[layer], s.v[layer], B, s.rows, s.row_start, Hq, Hkv, D, *cache, s.kv_len, s.n_rows,
                                       c["window"], c["sinks"], 0.0, s.out[layer])

    for layer in range(nl):
        if c["kind"] == "append":
            append(layer, s.q[layer])
        elif c["kind"] == "layers":
            append(layer, s.q[0])
            attend(layer, s.q[0])
        else:
            attend(layer, s.q[layer])
    if c["kind"] == "append":
        return {"q": s.q, "k": s.k, "v": s.v}
    return {"attention": s.out, "k": s.k, "v": s.v} if c["kind"] == "layers" else {"attention": s.out}


# ---------------------------------------------------------------------------------------------------- the plain forms
def _turned(s, x, weight):
    """Live rows [rows, heads, D] in 32 bits, normalised and rotated; the angles in 64."""
    c = s.case
    rot = c["rot_dim"]
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight
    base = s.position if s.position is not None else s.kv_len
    step = s.depth.flatten()[s.row] if s.depth is not None else s.t
    angle = (base[s.seq] + step).double()[:, None] * s.inv_freq
    cos, sin = ((f(angle) * s.magnitude).float()[:, None] for f in (torch.cos, torch.sin))
    head, rest = x[..., :rot], x[..., rot:]
    a, b = (head[..., 0::2], head[..., 1::2]) if c["interleaved"] else (head[..., :rot // 2], head[..., rot // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    head = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([head, rest], -1)


def _plain_append(s, layer, q_out):
    q, k, v = (x[s.row].float() for x in _split(s, layer))
    at = s.kv_len[s.seq].long() + s.t
    page, slot = s.page_of[s.seq, at], s.slot_of[s.seq, at]
    q_out[s.row] = _turned(s, q, s.q_weight).to(q_out.dtype)
    s.k[layer][page, slot] = _turned(s, k, s.k_weight).to(s.k.dtype)
    s.v[layer][page, slot] = v.to(s.v.dtype)


def _plain_seen(s, b, t, T):
    """Whether the rows t of sequence b see its positions [rows, T]."""
    c = s.case
    L, p = int(s.L[b]), torch.arange(T, device="cuda")
    if s.anc is None:
        pos, key = L + t[:, None], p
        seen = key <= pos
    else:
        node = (p - L).clamp_min(0)
        bit = (s.anc[b][t][:, node // 32] >> (node % 32)) & 1 != 0
        seen = (p < L) | bit
        pos, key = L + s.depth[b][t].long()[:, None], torch.where(p < L, p, L + s.depth[b][node].long())
    if c["window"]:
        seen = seen & ((key > pos - c["window"]) | (key < c["sinks"]))
    return seen


def _plain_attend(s, layer, q):
    c = s.case
    Hq, Hkv, D = c["q_heads"], c["kv_heads"], c["head_dim"]
    G = Hq // Hkv
    for b in range(c["batch"]):
        n, first = int(s.n[b]), int(s.first[b])
        T = int(s.L[b]) + n
        page, slot = s.page_of[b, :T], s.slot_of[b, :T]
        k, v = (x[layer][page, slot].float().transpose(0, 1) for x in (s.k, s.v))  # [Hkv, T, D]
        step = max(1, min(n, int(3e8 / (Hq * T))))
        for t0 in range(0, n, step):
            t = torch.arange(t0, min(t0 + step, n), device="cuda")
            x = q[first + t0:first + t0 + len(t)].float().unflatten(1, (Hkv, G)).permute(1, 2, 0, 3).flatten(1, 2)  # [Hkv, G rows, D]
            x = (x @ k.transpose(1, 2)).mul_(D ** -0.5).unflatten(1, (G, len(t)))
            x.masked_fill_(~_plain_seen(s, b, t, T), -torch.inf)
            w = x.sub_(x.amax(-1, keepdim=True)).exp_()
            l = w.sum(-1, keepdim=True)
            o = (w.flatten(1, 2) @ v).unflatten(1, (G, len(t))) / l
            s.out[layer, first + t0:first + t0 + len(t)] = o.permute(2, 0, 1, 3).flatten(1, 2).to(s.out.dtype)


def run(s):
    if own:
        return _run_own(s)
    kind = s.case["kind"]
    for layer in range(s.case["layers"]):
        if kind in ("append", "layers"):
            _plain_append(s, layer, s.q[layer if kind == "append" else 0])
        if kind != "append":
            _plain_attend(s, layer, s.q[layer if kind != "layers" else 0])
    if kind == "append":
        return {"q": s.q, "k": s.k, "v": s.v}
    return {"attention": s.out, "k": s.k, "v": s.v} if kind == "layers" else {"attention": s.out}


# ---------------------------------------------------------------------------------------------------- bounds
def work(case):
    """Each input read once, each output written once; prefixes and new rows at their mean lengths. Attention: the positions
    that some row of a sequence sees, and two multiply-adds per dimension and pair of a query and a position that it sees."""
    kind, B, nl, Hq, Hkv, D = (case[k] for k in ("kind", "batch", "layers", "q_heads", "kv_heads", "head_dim"))
    size = SIZE[case["dtype"]]
    L, tree = (case["prefix_lo"] + case["prefix_hi"]) / 2, kind == "tree" or case.get("tree")
    mean = (case["rows_lo"] + case["rows_hi"]) / 2
    groups = [(B - B // 2, 1.0), (B // 2, mean)] if _decoding(case) else [(B, mean)]
    bytes_ = flops = 0.0
    for count, n in groups:  # sequences with n new rows each
        if kind in ("append", "layers"):  # read: the projection's output; written: keys and values, and the queries where they are asked for
            bytes_ += nl * count * n * ((Hq + 2 * Hkv) + 2 * Hkv + (Hq if kind == "append" else 0)) * D * size
        if kind == "append":
            continue
        own_, new = (min(5, n), n) if tree else ((n + 1) / 2, n)  # new positions that a row sees, that the sequence has
        seen, all_ = L + own_, L + new
        if case["window"]:
            most = case["window"] + case["sinks"]
            if tree:
                seen, all_ = min(seen, most), min(all_, most + new)
            else:
                short = max(0.0, min(n, most - L))  # rows that see everything before them
                seen = (short * (L + (short + 1) / 2) + (n - short) * most) / n
                all_ = min(all_, most + n)
        cached, queries = (all_ - new, n) if kind == "layers" else (all_, 2 * n)
        bytes_ += nl * count * (2 * Hkv * cached + queries * Hq) * D * size
        flops += nl * count * 4 * Hq * D * n * seen
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """Sequence by sequence, head by head, from the definitions."""
    nl, Hq, Hkv, D = (case[k] for k in ("layers", "q_heads", "kv_heads", "head_dim"))
    G, kind = Hq // Hkv, case["kind"]
    if work(case)["flops"] > 4e12 or nl * case["batch"] * Hq > 20000 or work(case)["bytes"] > 1e10:
        return None
    s = prepare(case, seed)
    if kind in ("append", "layers"):
        s.k, s.v = s.k.double(), s.v.double()
        s.q = torch.zeros_like(s.q, dtype=torch.float64)
    if kind != "append":
        out = torch.zeros_like(s.out, dtype=torch.float64)

    def place(b, p):
        unit = case["page"]
        return (s.table[b].long()[p // unit], p % unit) if unit else (torch.full_like(p, b), p)

    def step_of(b, n):
        return torch.from_numpy(s.level[b, :n].astype(np.int64)).cuda() if s.depth is not None else torch.arange(n, device="cuda")

    def turn(x, pos, weight):  # x [rows, heads, D]: every pair as a complex number times e^(i angle)
        if weight is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS) * weight.double()
        r = case["rot_dim"]
        lo = torch.arange(0, r, 2) if case["interleaved"] else torch.arange(r // 2)
        hi = lo + (1 if case["interleaved"] else r // 2)
        z = torch.complex(x[..., lo], x[..., hi]) * torch.polar(torch.full((len(x), 1, r // 2), s.magnitude, dtype=torch.float64, device="cuda"),
                                                               (pos.double()[:, None] * s.inv_freq)[:, None])
        y = x.clone()
        y[..., lo], y[..., hi] = z.real, z.imag
        return y

    for layer in range(nl):
        q_all = s.q[layer if kind != "layers" else 0]
        for b in range(case["batch"]):
            n, L, r0 = int(s.n[b]), int(s.L[b]), int(s.first[b])
            if kind in ("append", "layers"):
                q, k, v = (x[r0:r0 + n].double() for x in _split(s, layer))
                pos = L + case["offset"] + step_of(b, n)
                where = place(b, L + torch.arange(n, device="cuda"))
                q_all[r0:r0 + n] = turn(q, pos, s.q_weight)
                s.k[layer][where], s.v[layer][where] = turn(k, pos, s.k_weight), v
            if kind == "append":
                continue
            p = torch.arange(L + n, device="cuda")
            where = place(b, p)
            stands = torch.cat([p[:L], L + step_of(b, n)])  # the position that a cache row stands for
            age = (L + step_of(b, n))[:, None] - stands
            hidden = age < 0
            if s.anc is not None:
                words = s.anc[b, :n].cpu().numpy().view(np.uint32)
                bits = torch.from_numpy(np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:, :n].astype(bool)).cuda()
                hidden[:, L:] |= ~bits
            if case["window"]:
                hidden |= (age >= case["window"]) & (stands >= case["sinks"])
            for h in range(Hq):
                kh, vh = (x[layer][where[0], where[1], h // G].double() for x in (s.k, s.v))
                for t0 in range(0, n, 1024):
                    x = torch.einsum("td,pd->tp", q_all[r0 + t0:min(r0 + t0 + 1024, r0 + n), h].double(), kh) / D ** 0.5
                    x.masked_fill_(hidden[t0:t0 + 1024], -torch.inf)
                    out[layer, r0 + t0:r0 + t0 + len(x), h] = torch.softmax(x, -1) @ vh
    if kind == "append":
        return {"q": s.q, "k": s.k, "v": s.v}
    return {"attention": out, "k": s.k, "v": s.v} if kind == "layers" else {"attention": out}
