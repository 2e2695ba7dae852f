"""The key/value cache held in 4 bits, and eviction from a cache by accumulated attention weight, as timed cases.

Every case is one pass through calls of `paper_2510_26577_b200.binding.CastContext`, as a decoding loop makes them, or the
same operators in plain torch operations:

  store    keys and values of new rows quantised into the cache, and read back as the next chunk of a prefill reads them
  attend   tree-masked verification attention over the 4-bit cache, layer after layer
  compact  the end of a greedy step on the 4-bit cache: accepted rows to the front of the tree region, and read back
  mass     the attention weight of the accepted rows, accumulated per position and kv-head of all layers
  evict    the rows with the least weight leave the cache of all layers

A 4-bit row is D codes and a pair (step, low) per position and kv-head; it stands for low + step * code. Codes lie as
[num_pages, Hkv, page, D/2] (dims 2i and 2i + 1 in the low and high half of byte i), pairs as [num_pages, Hkv, page, 2] bf16;
page 0 is one run of seq_capacity positions per sequence.
"""
import numpy as np
import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def _case(kind, name=None, **kw):
    c = {} if name is None else {"name": name}
    c.update(kind=kind, **kw)
    return c


def _heads(q_heads, kv_heads, head_dim):
    return {"q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim}


def _where(page, lo, hi):
    return {"page": page, "prefix_lo": lo, "prefix_hi": hi}


def listed():
    return [
        # the 60 tree tokens of one user of an 8B model, one layer: a call in front of every layer's attention, latency alone
        _case("store", "store_tree_b1", dtype="bf16", layers=1, batch=1, rows=60, **_heads(32, 8, 128), **_where(16, 2048, 2048)),
        # chunks of prompts, ragged, behind what is cached already
        _case("store", "store_prefill", dtype="bf16", layers=2, batch=4, rows=4097, **_heads(32, 8, 128), **_where(16, 0, 4096)),
        # one interactive user of an 8B model: a fixed tree of 60 tokens, four of the layers
        _case("attend", "attend_b1", dtype="bf16", layers=4, batch=1, tokens=60, ragged=False, **_heads(32, 8, 128), **_where(0, 2048, 2048)),
        # a loaded server: ragged paged sequences with small trees
        _case("attend", "attend_b64", dtype="bf16", layers=2, batch=64, tokens=12, ragged=True, **_heads(32, 8, 128), **_where(16, 512, 4096)),
        # long context, a GQA group of seven
        _case("attend", "attend_long", dtype="bf16", layers=2, batch=4, tokens=96, ragged=False, **_heads(28, 4, 128), **_where(16, 32768, 32768)),
        # a small model in 32 bits, heads of 64 dimensions, pages of an odd size
        _case("attend", "attend_f32_d64", dtype="f32", layers=2, batch=4, tokens=33, ragged=True, **_heads(8, 8, 64), **_where(24, 300, 1111)),
        # the end of a step: one user, and a loaded server, all 32 layers
        _case("compact", "compact_b1", dtype="bf16", layers=32, batch=1, depth=6, tokens=60, **_heads(32, 8, 128), **_where(16, 2048, 2048)),
        _case("compact", "compact_b64", dtype="bf16", layers=32, batch=64, depth=6, tokens=12, **_heads(32, 8, 128), **_where(16, 128, 1024)),
        # the weights of what eight sequences accepted, over a cache in 16 bits, eight of the layers
        _case("mass", "mass_bf16", cache="16", dtype="bf16", layers=8, batch=8, depth=6, tokens=60, **_heads(32, 8, 128), **_where(16, 1024, 4096)),
        # the same over long sequences in 4 bits
        _case("mass", "mass_q4_long", cache="4", dtype="bf16", layers=2, batch=4, depth=6, tokens=96, **_heads(28, 4, 128), **_where(16, 32768, 32768)),
        # a server halves what four sequences hold, all layers
        _case("evict", "evict_bf16", cache="16", dtype="bf16", layers=32, batch=4, budget=4096, recent=512, **_heads(32, 8, 128), **_where(16, 6000, 8192)),
        # one user's 4-bit cache is cut to a quarter
        _case("evict", "evict_q4_b1", cache="4", dtype="bf16", layers=8, batch=1, budget=1000, recent=100, **_heads(32, 8, 128), **_where(0, 4001, 4001)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def _draw_once(rng):
    kind = rng.choice(["store", "attend", "attend", "attend", "compact", "mass", "mass", "evict", "evict"])
    dtype = "f32" if rng.random() < 0.15 else "bf16"
    group, kv_heads = rng.choice([1, 2, 4, 4, 7, 8]), rng.choice([1, 2, 4, 8, 8])
    head_dim = 64 if rng.random() < 0.3 else 128
    hi = _log_int(rng, 16, 32768)
    lo = hi if rng.random() < 0.3 else max(1, hi // rng.randint(2, 8))
    c = dict(dtype=dtype, layers=_log_int(rng, 1, 32), batch=_log_int(rng, 1, 64), **_heads(group * kv_heads, kv_heads, head_dim),
             **_where(rng.choice([0, 8, 16, 16, 24, 32, 64, 128]), lo, hi))
    if kind == "store":
        return _case(kind, rows=_log_int(rng, 1, 4097), **c)
    if kind == "attend":
        return _case(kind, tokens=_log_int(rng, 1, 128), ragged=rng.random() < 0.5, **c)
    if kind == "compact":
        return _case(kind, depth=rng.randint(3, 13), tokens=rng.randint(14, 128), **c)
    if kind == "mass":
        return _case(kind, cache=rng.choice(["16", "4"]), depth=rng.randint(3, 13), tokens=rng.randint(14, 128), **c)
    budget = max(1, round(hi * rng.uniform(0.1, 1.1)))
    return _case(kind, cache=rng.choice(["16", "4"]), budget=budget, recent=rng.randint(0, budget), **c)


def _room(case):
    """Bytes that a plain pass and its inputs hold, roughly."""
    positions = case["batch"] * _capacity(case) * case["kv_heads"] * case["head_dim"]
    rows = case.get("rows", 0) * case["batch"] * case["kv_heads"] * case["head_dim"] * case["layers"] * 24
    heads = case["batch"] * _capacity(case) * case["q_heads"] * 16 * (case["tokens"] if case["kind"] == "attend" else case.get("depth", 0) + 1)
    layers = case["layers"] if case["kind"] in ("mass", "evict") else 1  # what these take in one piece
    return positions * (4 * case["layers"] + 24 * layers) + rows + heads * layers


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
def _generators(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g, np.random.Generator(np.random.Philox(seed))


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=DTYPE[dtype])


def _capacity(case):
    """Positions reserved per sequence, in whole pages."""
    unit = case["page"] or 1
    return -(-(case["prefix_hi"] + max(case.get("tokens", 0), case.get("rows", 0))) // unit) * unit


def _trees(B, cap, depth, n_tree, rng):
    """Random rooted trees in creation order: parents, depths [B, cap] and ancestor masks (host arrays)."""
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
    return parent, level, anc


def _quantise(x):
    """Codes [..., D/2] and (step, low) [..., 2] of rows [..., D]."""
    x = x.float()
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    low = lo.to(torch.bfloat16).float()
    step = ((hi - lo) / torch.full_like(hi, 15)).to(torch.bfloat16).float()  # (a division: by a plain 15 it would be a product)
    codes = torch.where(step > 0, torch.round((x - low) / step).clamp(0, 15), torch.zeros_like(x)).to(torch.uint8)
    return codes[..., 0::2] | (codes[..., 1::2] << 4), torch.cat([step, low], -1).to(torch.bfloat16)


def _values(codes, pair):
    """What a 4-bit row stands for, fp32."""
    nibbles = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()
    return pair[..., 1:].float() + pair[..., :1].float() * nibbles


class State:
    pass


def _prepare_cache(case, s, gen, rng, four_bits):
    """The caches of all layers, their page table and the sequences' lengths."""
    B, nl, unit, Hkv, D = (case[k] for k in ("batch", "layers", "page", "kv_heads", "head_dim"))
    positions = s.positions = _capacity(case)
    s.seq_cap, s.pages, s.table = positions // (unit or 1), 0, None
    if unit:
        s.pages = B * s.seq_cap
        s.table = _dev(rng.permutation(s.pages).astype(np.int32).reshape(B, s.seq_cap))
    s.kv0 = _dev(rng.integers(case["prefix_lo"], case["prefix_hi"] + 1, B).astype(np.int32))
    s.kv_len = s.kv0.clone()
    pages, slots = (s.pages, unit) if unit else (B, positions)
    # the position -> (page, slot) map of the plain forms
    at = torch.arange(positions, device="cuda")
    s.page_of = (s.table.long()[:, at // unit] if unit else torch.arange(B, device="cuda")[:, None].expand(B, positions))
    s.slot_of = (at % unit if unit else at).expand(B, positions)
    if not four_bits:
        s.k, s.v = (_randn((nl, pages, slots, Hkv, D), case["dtype"], gen) for _ in range(2))
        s.stride = s.k[0].numel() * s.k.element_size()
        return
    s.kc, s.vc = (torch.empty((nl, pages, Hkv, slots, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    s.kr, s.vr = (torch.empty((nl, pages, Hkv, slots, 2), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for layer in range(nl):
        for codes, pair in ((s.kc, s.kr), (s.vc, s.vr)):
            codes[layer], pair[layer] = _quantise(_randn((pages, Hkv, slots, D), "bf16", gen))
    s.code_stride, s.pair_stride = s.kc[0].numel(), s.kr[0].numel() * 2


def _accepted(case, s, rng):
    """A greedy step's outcome: a random root-to-node path of each tree, as the linear indices of its nodes."""
    B, H = case["batch"], case["depth"]
    parent, _, _ = _trees(B, case["tokens"], H, np.full(B, case["tokens"]), rng)
    path, n = np.full((B, H + 1), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        t, nodes = int(rng.integers(0, case["tokens"])), []
        while t >= 0:
            nodes.append(t)
            t = parent[b, t]
        path[b, :len(nodes)], n[b] = nodes[::-1], len(nodes) - 1
    s.path, s.accept_len = _dev(path), _dev(n)


def prepare(case, seed):
    gen, rng = _generators(seed)
    kind, B, nl, Hkv, D = (case[k] for k in ("kind", "batch", "layers", "kv_heads", "head_dim"))
    s = State()
    s.case = case
    _prepare_cache(case, s, gen, rng, four_bits=case.get("cache", "4") == "4")
    s.total = case.get("tokens", 8)
    if kind == "store":
        s.new_k, s.new_v = (_randn((nl, B, case["rows"], Hkv, D), case["dtype"], gen) for _ in range(2))
        s.n_rows = _dev(rng.integers(max(1, case["rows"] // 2), case["rows"] + 1, B).astype(np.int32))
        s.back_k, s.back_v = torch.zeros_like(s.new_k), torch.zeros_like(s.new_v)
    if kind == "attend":
        n = rng.integers(max(1, s.total // 2), s.total + 1, B) if case["ragged"] else np.full(B, s.total)
        _, _, anc = _trees(B, s.total, 8, n, rng)
        s.anc, s.n_tree = _dev(anc.view(np.int32)), _dev(n.astype(np.int32))
    if kind in ("attend", "mass"):
        s.q = _randn((nl, B, s.total, case["q_heads"], D), case["dtype"], gen)
        s.out = torch.zeros_like(s.q)
    if kind in ("compact", "mass"):
        _accepted(case, s, rng)
    if kind == "compact":
        s.back_k, s.back_v = (torch.zeros((nl, B, case["depth"] + 1, Hkv, D), dtype=DTYPE[case["dtype"]], device="cuda") for _ in range(2))
        s.n_rows = s.accept_len + 1
    if kind == "mass":
        s.kv_len += s.accept_len + 1  # the accepted rows stand behind the prefix
    if kind in ("mass", "evict"):  # a heavy-tailed sum per position, zero where there is none yet
        s.mass0 = torch.randn((nl, B, Hkv, s.positions), generator=gen, device="cuda").mul_(1.5).exp_()
        s.mass0 *= torch.arange(s.positions, device="cuda") < s.kv0[:, None, None]
        if kind == "mass":
            s.mass0 /= s.positions  # a few rows' weights so far
        s.mass = s.mass0.clone()
    if kind == "evict":
        s.kept = torch.zeros((nl, B, Hkv, case["budget"]), dtype=torch.int32, device="cuda")
        s.n_rows = s.kv0.clamp(max=case["budget"])
        s.none = torch.zeros_like(s.kv0)
        if case["cache"] == "4":
            s.back_k, s.back_v = (torch.zeros((nl, B, case["budget"], Hkv, D), dtype=DTYPE[case["dtype"]], device="cuda") for _ in range(2))
    s.ctx = _context(case, s) if own else None
    return s


def _context(case, s):
    from paper_2510_26577_b200 import binding
    ctx = binding.CastContext(max_batch=case["batch"], vocab=32000, top_k=8, max_depth=case.get("depth", 8),
                              total_token=s.total, max_tree=s.total)
    heads = (case["q_heads"], case["kv_heads"], case["head_dim"], case["page"], s.seq_cap)
    if case["kind"] == "attend":
        ctx.cast_reserve_attention_q4(s.q.dtype, case["batch"], *heads)
    if case["kind"] == "mass":
        ctx.cast_reserve_attention_mass(s.q.dtype, case["batch"], case["layers"], case["depth"] + 1, *heads)
    return ctx


# ---------------------------------------------------------------------------------------------------- the framework's calls
def _run_own(s):
    c = s.case
    B, nl, Hq, Hkv, D, page = (c[k] for k in ("batch", "layers", "q_heads", "kv_heads", "head_dim", "page"))
    cache = (page, s.table, s.seq_cap, s.pages)
    if c["kind"] == "store":
        s.ctx.cast_store_kv_q4(s.new_k, s.new_v, B, nl, c["rows"], Hkv, D, *cache, s.kv_len, s.n_rows, s.kc, s.kr, s.vc, s.vr,
                               s.code_stride, s.pair_stride)
        s.ctx.cast_load_kv_q4(s.kc, s.kr, s.vc, s.vr, s.code_stride, s.pair_stride, B, nl, c["rows"], Hkv, D, *cache, s.kv_len,
                              s.n_rows, s.back_k, s.back_v)
        return {"k": s.back_k, "v": s.back_v}
    if c["kind"] == "attend":
        for layer in range(nl):
            s.ctx.cast_tree_attention_q4(s.q[layer], s.kc[layer], s.kr[layer], s.vc[layer], s.vr[layer], B, Hq, Hkv, D, *cache,
                                         s.kv_len, s.anc, s.n_tree, None, 0.0, s.out[layer])
        return {"attention": s.out}
    if c["kind"] == "compact":
        s.kv_len.copy_(s.kv0)  # the call advances the lengths in place: a pass starts from the same prefix as the one before
        s.ctx.cast_compact_kv_q4(s.kc, s.kr, s.vc, s.vr, s.code_stride, s.pair_stride, B, nl, Hkv, D, *cache, s.path, s.accept_len,
                                 s.kv_len)
        s.ctx.cast_load_kv_q4(s.kc, s.kr, s.vc, s.vr, s.code_stride, s.pair_stride, B, nl, c["depth"] + 1, Hkv, D, *cache, s.kv0,
                              s.n_rows, s.back_k, s.back_v)
        return {"k": s.back_k, "v": s.back_v, "kv_len": s.kv_len}
    if c["kind"] == "mass":
        q_stride = s.q[0].numel() * s.q.element_size()
        if c["cache"] == "16":
            s.ctx.cast_attention_mass(s.q, s.k, B, nl, q_stride, s.stride, Hq, Hkv, D, *cache, s.path, s.accept_len, s.kv_len, 0.0,
                                      s.mass)
        else:
            s.ctx.cast_attention_mass_q4(s.q, s.kc, s.kr, B, nl, q_stride, s.code_stride, s.pair_stride, Hq, Hkv, D, *cache, s.path,
                                         s.accept_len, s.kv_len, 0.0, s.mass)
        return {"mass": s.mass}
    s.kv_len.copy_(s.kv0)  # as above: eviction shortens what it is given
    s.mass.copy_(s.mass0)
    out = {"mass": s.mass, "kept": s.kept, "kv_len": s.kv_len}
    if c["cache"] == "16":
        s.ctx.cast_evict_kv(s.k, s.v, B, nl, s.stride, Hkv, D, *cache, c["budget"], c["recent"], s.mass, s.kept, s.kv_len)
        return {**out, "k": s.k, "v": s.v}
    s.ctx.cast_evict_kv_q4(s.kc, s.kr, s.vc, s.vr, s.code_stride, s.pair_stride, B, nl, Hkv, D, *cache, c["budget"], c["recent"],
                           s.mass, s.kept, s.kv_len)
    s.ctx.cast_load_kv_q4(s.kc, s.kr, s.vc, s.vr, s.code_stride, s.pair_stride, B, nl, c["budget"], Hkv, D, *cache, s.none, s.n_rows,
                          s.back_k, s.back_v)
    return {**out, "k": s.back_k, "v": s.back_v}


# ---------------------------------------------------------------------------------------------------- the plain forms
def _places(s, start, n_rows, rows):
    """Page and slot [B, rows] of the positions start + t; a mask of the rows t < n_rows. The others' place is that of position 0."""
    t = torch.arange(rows, device="cuda")
    live = t < n_rows[:, None]
    at = torch.where(live, start[:, None].long() + t, torch.zeros_like(t))
    return s.page_of.gather(1, at), s.slot_of.gather(1, at), live


def _read_back(s, start, rows):
    """The rows start + t, t < n_rows, of all layers into back_k, back_v."""
    pages, slots, live = _places(s, start, s.n_rows, rows)
    for codes, pair, back in ((s.kc, s.kr, s.back_k), (s.vc, s.vr, s.back_v)):
        x = _values(codes[:, pages, :, slots], pair[:, pages, :, slots])  # [B, rows, layers, Hkv, D]
        back.copy_(torch.where(live[None, :, :, None, None], x.movedim(2, 0).to(back.dtype), back))


def _plain_store(s):
    pages, slots, live = _places(s, s.kv_len, s.n_rows, s.case["rows"])
    p, t = pages[live], slots[live]
    for x, codes, pair in ((s.new_k, s.kc, s.kr), (s.new_v, s.vc, s.vr)):
        c, r = _quantise(x[:, live])  # [layers, live rows, Hkv, ...]
        codes[:, p, :, t], pair[:, p, :, t] = c.movedim(1, 0), r.movedim(1, 0)
    _read_back(s, s.kv_len, s.case["rows"])
    return {"k": s.back_k, "v": s.back_v}


def _weights(x):
    """Softmax over the last axis; a row without any finite entry gives zeros."""
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(top > -torch.inf, top, torch.zeros_like(top)))
    return e / e.sum(-1, keepdim=True).clamp_min(torch.finfo(x.dtype).tiny)


def _grouped(q, Hkv):
    """[..., T, Hq, D] -> [..., Hkv, T * G, D], the group's heads of a token side by side."""
    *lead, T, Hq, D = q.shape
    return q.reshape(*lead, T, Hkv, Hq // Hkv, D).movedim(-3, -4).reshape(*lead, Hkv, T * (Hq // Hkv), D)


def _plain_attend(s):
    c = s.case
    B, Hkv, D, T = c["batch"], c["kv_heads"], c["head_dim"], s.total
    G = c["q_heads"] // Hkv
    word = torch.arange(T, device="cuda")
    bits = (s.anc[:, :, word // 32] >> (word % 32)) & 1 != 0  # [B, T, T]
    node = torch.arange(s.positions, device="cuda") - s.kv_len[:, None]  # the tree token at a position
    seen = bits.gather(2, node.clamp(0, T - 1)[:, None, :].expand(B, T, s.positions)) & (node >= 0)[:, None] & (node < s.n_tree[:, None])[:, None]
    seen |= (node < 0)[:, None]
    live = (word < s.n_tree[:, None])[..., None, None]
    hide = torch.where(seen, 0.0, -torch.inf).repeat_interleave(G, 1)[:, None]  # [B, 1, T * G, positions]
    for layer in range(c["layers"]):
        k = _values(s.kc[layer][s.page_of, :, s.slot_of], s.kr[layer][s.page_of, :, s.slot_of]).transpose(1, 2)  # [B, Hkv, positions, D]
        x = _grouped(s.q[layer].float(), Hkv) @ k.transpose(2, 3)
        w = _weights(x.mul_(D ** -0.5).add_(hide))
        v = _values(s.vc[layer][s.page_of, :, s.slot_of], s.vr[layer][s.page_of, :, s.slot_of]).transpose(1, 2)
        o = (w @ v).reshape(B, Hkv, T, G, D).transpose(1, 2).reshape(B, T, Hkv * G, D)
        s.out[layer].copy_(torch.where(live, o.to(s.out.dtype), s.out[layer]))
    return {"attention": s.out}


def _plain_compact(s):
    s.kv_len.copy_(s.kv0)
    rows = s.case["depth"] + 1
    pages, slots, live = _places(s, s.kv_len, s.n_rows, rows)
    src = s.kv_len[:, None].long() + s.path.clamp_min(0)
    from_page, from_slot = s.page_of.gather(1, src)[live], s.slot_of.gather(1, src)[live]
    for x in (s.kc, s.kr, s.vc, s.vr):
        x[:, pages[live], :, slots[live]] = x[:, from_page, :, from_slot]
    s.kv_len += s.accept_len + 1
    _read_back(s, s.kv0, rows)
    return {"k": s.back_k, "v": s.back_v, "kv_len": s.kv_len}


def _accepted_queries(s):
    """Queries of the accepted rows [layers, B, H + 1, Hq, D] and what they see [B, H + 1, positions]: row i of n the positions
    below kv_len - n + i + 1, a row past n none."""
    i = torch.arange(s.path.shape[1], device="cuda")
    at = s.path.clamp_min(0).long()[None, :, :, None, None].expand(s.q.shape[0], -1, -1, *s.q.shape[3:])
    first = (s.kv_len - s.accept_len)[:, None, None] + i[:, None]
    seen = (torch.arange(s.positions, device="cuda") < first) & (i <= s.accept_len[:, None])[..., None]
    return s.q.gather(2, at), seen


def _plain_mass(s):
    c = s.case
    Hkv, D = c["kv_heads"], c["head_dim"]
    if c["cache"] == "16":
        k = s.k[:, s.page_of, s.slot_of].float().transpose(2, 3)  # [layers, B, Hkv, positions, D]
    else:
        k = _values(s.kc[:, s.page_of, :, s.slot_of], s.kr[:, s.page_of, :, s.slot_of]).permute(2, 0, 3, 1, 4)
    q, seen = _accepted_queries(s)
    x = _grouped(q.float(), Hkv) @ k.transpose(3, 4)
    hide = torch.where(seen, 0.0, -torch.inf).repeat_interleave(c["q_heads"] // Hkv, 1)[:, None]
    s.mass += _weights(x.mul_(D ** -0.5).add_(hide)).sum(3)
    return {"mass": s.mass}


def _plain_evict(s):
    c = s.case
    budget, recent, nl, B, Hkv = c["budget"], c["recent"], c["layers"], c["batch"], c["kv_heads"]
    s.kv_len.copy_(s.kv0)
    s.mass.copy_(s.mass0)
    n = s.kv_len.long()[:, None, None]
    at = torch.arange(s.positions, device="cuda")
    # sorted by weight, the last `recent` first, what lies behind the sequence last; ties to the lower position
    weight = torch.where(at >= n - recent, torch.inf, s.mass).masked_fill(at >= n, -torch.inf)
    best = weight.sort(dim=-1, descending=True, stable=True).indices
    best = torch.where(n > budget, best, at)[..., :budget]
    live = torch.arange(best.shape[-1], device="cuda") < n.clamp(max=budget)
    kept = torch.where(live, best, s.positions).sort(-1).values  # [layers, B, Hkv, up to budget]
    s.kept.fill_(-1)[..., :kept.shape[-1]] = torch.where(live, kept, -1)
    src = torch.where(live, kept, 0)
    live = live.expand(nl, B, Hkv, -1)
    mass = torch.where(live, s.mass.gather(3, src), 0.0)
    s.mass.masked_fill_(at < n, 0.0)  # what lies behind the sequence stays as it is
    l, b, h, j = live.nonzero(as_tuple=True)
    s.mass[l, b, h, j] = mass[l, b, h, j]
    old = src[l, b, h, j]
    to, frm = (s.page_of[b, j], s.slot_of[b, j]), (s.page_of[b, old], s.slot_of[b, old])
    s.kv_len.clamp_(max=budget)
    out = {"mass": s.mass, "kept": s.kept, "kv_len": s.kv_len}
    if c["cache"] == "16":
        s.k[l, to[0], to[1], h] = s.k[l, frm[0], frm[1], h]
        s.v[l, to[0], to[1], h] = s.v[l, frm[0], frm[1], h]
        return {**out, "k": s.k, "v": s.v}
    for x in (s.kc, s.kr, s.vc, s.vr):
        x[l, to[0], h, to[1]] = x[l, frm[0], h, frm[1]]
    _read_back(s, s.none, budget)
    return {**out, "k": s.back_k, "v": s.back_v}


def run(s):
    if own:
        return _run_own(s)
    return {"store": _plain_store, "attend": _plain_attend, "compact": _plain_compact, "mass": _plain_mass, "evict": _plain_evict}[s.case["kind"]](s)


# ---------------------------------------------------------------------------------------------------- bounds
def work(case):
    """Each input read once, each output written once; prefixes and accepted paths at their mean lengths."""
    kind, B, nl, Hq, Hkv, D = (case[k] for k in ("kind", "batch", "layers", "q_heads", "kv_heads", "head_dim"))
    size, row4 = SIZE[case["dtype"]], D // 2 + 4
    prefix = (case["prefix_lo"] + case["prefix_hi"]) / 2
    if kind == "store":
        rows = nl * B * Hkv * 2 * 0.75 * case["rows"]
        return {"bytes": rows * (2 * D * size + 2 * row4), "flops": 0}
    if kind == "attend":
        t = case["tokens"] * (0.75 if case["ragged"] else 1.0)
        return {"bytes": nl * B * (2 * Hkv * (prefix + t) * row4 + 2 * t * Hq * D * size), "flops": nl * B * 4 * t * Hq * D * (prefix + 4)}
    accepted = min(4, case.get("depth", 0) + 1)
    if kind == "compact":
        return {"bytes": nl * B * Hkv * 2 * accepted * (3 * row4 + D * size), "flops": 0}
    row = row4 if case["cache"] == "4" else D * size
    if kind == "mass":
        return {"bytes": nl * B * (Hkv * (prefix + accepted) * (row + 8) + accepted * Hq * D * size),
                "flops": nl * B * 2 * accepted * Hq * D * prefix}
    keep = min(prefix, case["budget"])
    moved = keep if prefix > keep else 0  # all behind the first row that leaves
    back = keep * 2 * (row + D * size) if case["cache"] == "4" else 0
    return {"bytes": nl * B * Hkv * (4 * prefix + moved * 4 * row + 8 * keep + 4 * (prefix - keep) + back), "flops": 0}


# ---------------------------------------------------------------------------------------------------- 64 bits
def _exact_row_values(x):
    """fp32 rows through the quantiser, one numpy step after the other (its codes are defined in 32-bit arithmetic; the bf16
    pair by rounding to nearest even), as the 64-bit values that they stand for."""
    x = x.astype(np.float32)

    def bf16(a):
        u = a.astype(np.float32).view(np.uint32).astype(np.uint64)
        return ((u + 0x7fff + ((u >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)

    lo, hi = x.min(-1, keepdims=True), x.max(-1, keepdims=True)
    low, step = bf16(lo), bf16((hi - lo) / np.float32(15))
    with np.errstate(divide="ignore", invalid="ignore"):
        code = np.where(step > 0, np.clip(np.rint((x - low) / step), 0, 15), 0)
    return low.astype(np.float64) + step.astype(np.float64) * code


def _decoded(codes, pair):
    """Values [..., D] in 64 bits, from bytes and pairs on the device."""
    pair = pair.double()
    out = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.float64, device=codes.device)
    out[..., 0::2], out[..., 1::2] = (codes % 16).double(), (codes // 16).double()
    return out * pair[..., 0:1] + pair[..., 1:2]


def _sequence(s, b, n):
    """Flat cache rows of the first n positions of sequence b."""
    unit = s.case["page"] or s.positions
    p = torch.arange(n, device="cuda")
    page = s.table[b].long()[p // unit] if s.table is not None else torch.full_like(p, b)
    return page, p % unit


def exact(case, seed):
    """Sequence by sequence, head by head, from the definitions."""
    rows = case.get("tokens", 1) if case["kind"] == "attend" else case.get("depth", 0) + 1
    if case["kind"] in ("attend", "mass") and case["layers"] * case["batch"] * _capacity(case) * case["q_heads"] * rows * case["head_dim"] > 2e13:
        return None
    if case["kind"] == "store" and case["layers"] * case["batch"] * case["rows"] * case["kv_heads"] * case["head_dim"] > 1e8:
        return None
    s = prepare(case, seed)
    B, nl, Hq, Hkv, D = (case[k] for k in ("batch", "layers", "q_heads", "kv_heads", "head_dim"))
    G, kind, scale = Hq // Hkv, case["kind"], case["head_dim"] ** -0.5
    if kind == "store":
        out = {}
        for name, x in (("k", s.new_k), ("v", s.new_v)):
            y = _exact_row_values(x.float().cpu().numpy())
            for b in range(B):
                y[:, b, int(s.n_rows[b]):] = 0.0
            out[name] = torch.from_numpy(y)
        return out
    if kind == "attend":
        out = torch.zeros(nl, B, s.total, Hq, D, dtype=torch.float64, device="cuda")
        for layer in range(nl):
            for b in range(B):
                n, L = int(s.n_tree[b]), int(s.kv_len[b])
                page, slot = _sequence(s, b, L + n)
                words = s.anc[b, :n].cpu().numpy().view(np.uint32)
                bits = torch.from_numpy(np.unpackbits(words.view(np.uint8), axis=1, bitorder="little")[:, :n].astype(bool)).cuda()
                for h in range(Hkv):
                    k, v = _decoded(s.kc[layer][page, h, slot], s.kr[layer][page, h, slot]), _decoded(s.vc[layer][page, h, slot], s.vr[layer][page, h, slot])
                    x = torch.einsum("tgd,pd->tgp", s.q[layer, b, :n, h * G:(h + 1) * G].double(), k) * scale
                    x[:, :, L:].masked_fill_(~bits[:, None], -torch.inf)
                    out[layer, b, :n, h * G:(h + 1) * G] = torch.einsum("tgp,pd->tgd", torch.softmax(x, -1), v)
        return {"attention": out}
    if kind == "compact":
        back = {name: torch.zeros(nl, B, case["depth"] + 1, Hkv, D, dtype=torch.float64, device="cuda") for name in "kv"}
        for b in range(B):
            n, L = int(s.accept_len[b]) + 1, int(s.kv0[b])
            page, slot = _sequence(s, b, s.positions)
            src = L + s.path[b, :n].long()
            for name, codes, pair in (("k", s.kc, s.kr), ("v", s.vc, s.vr)):
                x = _decoded(codes[:, page[src], :, slot[src]], pair[:, page[src], :, slot[src]])
                back[name][:, b, :n] = x.transpose(0, 1)
        return {**back, "kv_len": None}
    if kind == "mass":
        mass = s.mass0.double()
        for layer in range(nl):
            for b in range(B):
                n, L = int(s.accept_len[b]) + 1, int(s.kv_len[b])
                page, slot = _sequence(s, b, L)
                hidden = torch.arange(L, device="cuda")[None] > (L - n + torch.arange(n, device="cuda"))[:, None]
                for h in range(Hkv):
                    k = s.k[layer][page, slot, h].double() if case["cache"] == "16" else _decoded(s.kc[layer][page, h, slot], s.kr[layer][page, h, slot])
                    x = torch.einsum("tgd,pd->tgp", s.q[layer, b, s.path[b, :n].long(), h * G:(h + 1) * G].double(), k) * scale
                    mass[layer, b, h, :L] += torch.softmax(x.masked_fill(hidden[:, None], -torch.inf), -1).sum((0, 1))
        return {"mass": mass}
    return None  # eviction copies what it keeps: its outputs are its inputs' values
