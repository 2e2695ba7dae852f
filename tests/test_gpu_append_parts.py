"""cast_append_kv of queries alone, or of keys and values alone: the other side's number of heads is nobody's business."""
import numpy as np
import pytest
import torch

from test_gpu_append import binding, context, dev, simple  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("other", [0, -1, 40000, 2 ** 31 - 1])
def test_heads_of_what_is_not_given(binding, other):  # noqa: F811
    B, rows, D = 2, 9, 64
    q, k, v = (torch.randn((B, rows, h, D), device="cuda") for h in (6, 2, 2))
    n, inv = dev(np.array([9, 4], np.int32)), dev(10000.0 ** (-np.arange(32) / 32))
    ctx = context(binding, B)
    q_out, kc, vc = (torch.zeros_like(x) for x in (q, k, v))
    simple(ctx, q, k, v, B, rows, 6, 2, D, n, rows, None, q_out, kc, vc, inv)
    outs = [torch.zeros_like(x) for x in (q, k, v)]
    e = 4 * D
    ctx.cast_append_kv(q, 6 * e, None, 0, None, 0, B, rows, 6, other, D, None, None, n, None, None, inv, 64, 0, 1.0, None, None, 1e-6, 0, None, rows, 0,
                       None, outs[0], None, None)
    ctx.cast_append_kv(None, 0, k, 2 * e, v, 2 * e, B, rows, other, 2, D, None, None, n, None, None, inv, 64, 0, 1.0, None, None, 1e-6, 0, None, rows, 0,
                       None, None, outs[1], outs[2])
    assert ctx.cast_poll_status()[0] == 0
    for got, want in zip(outs, (q_out, kc, vc)):
        assert torch.equal(got, want)
    with pytest.raises(binding.CastError) as err:  # more heads than a call takes
        ctx.cast_append_kv(q[0, 0], 70000 * e, None, 0, None, 0, B, rows, 70000, 2, D, None, None, n, None, None, inv, 64, 0, 1.0, None, None, 1e-6, 0, None, rows,
                           0, None, outs[0], None, None)
    assert err.value.code == 3
