"""cast_append_kv right in front of an attention that reads early: the append releases its dependents before it writes, so what it
writes (the queries, the cache rows of the tree) must be what the attention waits for."""
import numpy as np
import pytest
import torch

import q4_oracle as o4
from test_gpu_chunk_attention import binding, dev  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hq,Hkv,page,kv,n", [(32, 8, 16, [2048], [60]), (32, 8, 16, [512, 4000, 1, 0, 130, 77, 1500, 900], [12, 7, 60, 1, 33, 60, 2, 24]),
                                              (8, 1, 0, [700, 40], [16, 16])])
@pytest.mark.parametrize("captured", [False, True])
def test_append_then_attention_with_early_reads(binding, Hq, Hkv, page, kv, n, captured):  # noqa: F811
    """Six layers one behind the other, and a chunk's attention over the appended rows between two of them; what is to be written holds NaN
    before every pass. The same bits as without the promise."""
    rng = np.random.default_rng(len(kv))
    B, D, layers, tokens = len(kv), 128, 6, 64
    L, N = np.array(kv, np.int32), np.array(n, np.int32)
    paged = o4.Paged(rng, B, int((L + N).max()) + 1, page)
    where = (page, dev(paged.table), paged.cap, paged.pages)
    anc, depth = np.zeros((B, tokens, 2), np.uint32), np.full((B, tokens), -1, np.int32)
    for b in range(B):
        vis = np.eye(tokens, dtype=bool)
        for t in range(N[b]):
            at = int(rng.integers(0, t)) if t else -1
            depth[b, t] = depth[b, at] + 1 if t else 0
            if t:
                vis[t] |= vis[at]
            for j in np.flatnonzero(vis[t]):
                anc[b, t, j >> 5] |= np.uint32(1 << (j & 31))
    gen = torch.Generator("cuda").manual_seed(5)
    x = torch.randn((layers, B, tokens, (Hq + 2 * Hkv) * D), generator=gen, device="cuda").bfloat16()
    shape = (layers, *paged.shape, Hkv, D)
    kc, vc = (torch.randn(shape, generator=gen, device="cuda").bfloat16() for _ in range(2))
    rows = [tuple(dev(a).long() for a in paged.at(b, L[b] + np.arange(N[b]))) for b in range(B)]
    inv, weight = dev(10000.0 ** (-np.arange(64) / 64)), torch.rand(D, generator=gen, device="cuda") + 0.5
    args = dict(kv_len=dev(L), n=dev(N), anc=dev(anc.view(np.int32)), depth=dev(depth))
    q_out, out, other = (torch.empty((layers, B, tokens, Hq, D), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    ctx = binding.CastContext(max_batch=B, vocab=1000, top_k=4, max_depth=6, total_token=tokens, max_tree=tokens)
    ctx.cast_reserve_attention(torch.bfloat16, B, Hq, Hkv, D, page, paged.cap)
    ctx.cast_reserve_chunk_attention(torch.bfloat16, D)
    stride = x.stride(2) * 2

    def step(stream=None):
        for l in range(layers):
            q, k, v = (a.unflatten(-1, (-1, D)) for a in x[l].split([Hq * D, Hkv * D, Hkv * D], -1))
            ctx.cast_append_kv(q, stride, k, stride, v, stride, B, tokens, Hq, Hkv, D, None, None, args["n"], args["depth"], None, inv, 128, 0, 0.0, weight,
                               weight, 1e-6, *where, args["kv_len"], q_out[l], kc[l], vc[l])
            if l == 3:
                ctx.cast_chunk_attention(q_out[l], kc[l], vc[l], B, tokens, None, Hq, Hkv, D, *where, args["kv_len"], args["n"], 0, 0, 0.0, other[l])
            ctx.cast_tree_attention(q_out[l], kc[l], vc[l], B, Hq, Hkv, D, *where, args["kv_len"], args["anc"], args["n"], 0.0, out[l])

    def clear():
        for t in (q_out, out, other):
            t.fill_(float("nan"))
        for b in range(B):
            for c in (kc, vc):
                c[(slice(None), *rows[b])] = float("nan")

    def results():
        torch.cuda.synchronize()
        assert ctx.cast_poll_status()[0] == 0
        return [t.clone().view(torch.int16) for t in (out, q_out, other[3])]

    clear()
    step()
    want = results()
    for b in range(B):
        assert not bool(torch.isnan(out[:, b, :N[b]]).any()) and bool(torch.isnan(out[:, b, N[b]:]).all())
    ctx.cast_set_attention_early_reads(True)
    graph = None
    if captured:
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            step()
    for _ in range(20):
        clear()
        graph.replay() if captured else step()
        for got, ref in zip(results(), want):
            assert torch.equal(got, ref)
