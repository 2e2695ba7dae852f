"""Frequencies of rotary positions against their formulas, and refusals that need no device."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

from paper_2510_26577_b200.rotary import inverse_frequencies

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def plain(d, base):
    return base ** (-np.arange(0, d, 2) / d)


@pytest.mark.parametrize("d,base", [(2, 10000.0), (24, 500000.0), (128, 10000.0)])
def test_plain_linear_and_ntk(d, base):
    inv, m = inverse_frequencies(d, base, device="cpu")
    np.testing.assert_allclose(inv.numpy(), plain(d, base), rtol=1e-14)
    assert m == 1.0 and str(inv.dtype) == "torch.float64"
    inv, m = inverse_frequencies(d, base, scaling="linear", factor=4.0, device="cpu")
    np.testing.assert_allclose(inv.numpy(), plain(d, base) / 4, rtol=1e-14)
    if d > 2:
        inv, m = inverse_frequencies(d, base, scaling="ntk", factor=4.0, device="cpu")
        assert m == 1.0 and inv[0] == 1.0
        assert abs(inv[-1].item() * 4 / plain(d, base)[-1] - 1) < 1e-12  # the slowest pair turns a quarter as fast


def test_yarn():
    d, base, f, ctx = 128, 10000.0, 16.0, 4096
    inv, m = inverse_frequencies(d, base, scaling="yarn", factor=f, context=ctx, device="cpu")
    theta = plain(d, base)
    turns = ctx * theta / (2 * math.pi)
    np.testing.assert_allclose(inv.numpy()[turns > 32 * 1.2], theta[turns > 32 * 1.2], rtol=1e-14)
    np.testing.assert_allclose(inv.numpy()[turns < 1 / 1.2], theta[turns < 1 / 1.2] / f, rtol=1e-14)
    ratio = inv.numpy() / theta
    assert (np.diff(ratio) <= 1e-15).all() and m == 0.1 * math.log(f) + 1
    mid = (turns < 32 / 1.2) & (turns > 1.2)  # a straight line in the pair's index
    assert np.abs(np.diff(ratio[mid], 2)).max() < 1e-12 and mid.sum() > 10


def test_llama3():
    d, base, f, ctx = 128, 500000.0, 8.0, 8192
    inv, m = inverse_frequencies(d, base, scaling="llama3", factor=f, context=ctx, device="cpu")
    for got, theta in zip(inv.tolist(), plain(d, base)):
        wave = 2 * math.pi / theta
        if wave < ctx / 4:
            want = theta
        elif wave > ctx / 1:
            want = theta / f
        else:
            s = (ctx / wave - 1) / (4 - 1)
            want = (1 - s) * theta / f + s * theta
        assert abs(got / want - 1) < 1e-12
    assert m == 1.0


@pytest.mark.parametrize("kw", [dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=8, base=0.0), dict(rot_dim=8, factor=0.0), dict(rot_dim=8, scaling="other"),
                                dict(rot_dim=8, scaling="yarn", factor=2.0), dict(rot_dim=2, scaling="ntk"),
                                dict(rot_dim=8, scaling="llama3", context=10, low_freq_factor=4.0)])
def test_refused(kw):
    with pytest.raises(ValueError):
        inverse_frequencies(device="cpu", **kw)


def test_calls_refuse_a_missing_context():
    """INVALID_ARG, before anything is asked of a device."""
    from paper_2510_26577_b200 import build
    lib = ctypes.CDLL(build.build())
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "cast.h")).read(), flags=re.S)
    some = ctypes.create_string_buffer(64)
    for name in ("cast_append_kv", "cast_reserve_chunk_attention", "cast_chunk_attention", "cast_tree_attention_window"):
        kinds = [ctypes.c_void_p if "*" in a else ctypes.c_float if "float" in a else ctypes.c_size_t if "size_t" in a else ctypes.c_int
                 for a in re.search(r"\b%s\(([^)]*)\)" % name, text).group(1).split(",")]
        f = getattr(lib, name)
        f.argtypes, f.restype = kinds, ctypes.c_int
        assert f(*[0 if t is not ctypes.c_void_p else None for t in kinds]) == 1, name
        assert f(None, *[ctypes.cast(some, t) if t is ctypes.c_void_p else t(1) for t in kinds[1:]]) == 1, name
