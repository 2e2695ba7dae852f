"""The C-ABI library builds for sm_100a, loads without a GPU, and exports every
symbol that include/cast.h declares (no compute call is made here)."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib_path():
    from paper_2510_26577_b200 import build
    return build.build()


def _declared():
    text = open(os.path.join(ROOT, "include", "cast.h")).read()
    return sorted(set(re.findall(r"CAST_API[^;(]*?\b(cast_\w+)\s*\(", text)))


def test_header_declares_the_five_calls():
    names = _declared()
    for n in ("cast_tree_expand", "cast_select_nodes", "cast_tree_attention", "cast_accept", "cast_compact_kv"):
        assert n in names


def test_library_exports_every_declared_symbol(lib_path):
    lib = ctypes.CDLL(lib_path)
    for name in _declared():
        assert hasattr(lib, name), name


def test_binding_lists_every_declared_symbol(lib_path):
    from paper_2510_26577_b200 import binding
    assert sorted(binding.EXPORTS) == _declared()
    lib = binding.load_library()
    assert lib.cast_status_string(3) == b"capacity exceeded"


def test_config_struct_matches_header_layout():
    from paper_2510_26577_b200.binding import CastConfig
    # 3 doubles + 14 int32 = 80 bytes, no padding (doubles first)
    assert ctypes.sizeof(CastConfig) == 80
    assert CastConfig.max_batch.offset == 24 and CastConfig.rerank_per_row.offset == 76


def test_calls_of_the_4_bit_cache_and_of_eviction_refuse_a_missing_context():
    """INVALID_ARG from every entry point, before anything is asked of a device."""
    from paper_2510_26577_b200 import binding
    lib = binding.load_library()
    names = [n for n in _declared() if n.endswith("_q4") or "mass" in n or "evict" in n]
    assert len(names) == 10
    some = ctypes.create_string_buffer(64)
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "cast.h")).read(), flags=re.S)
    for n in names:
        kinds = [ctypes.c_void_p if "*" in a else ctypes.c_float if "float" in a else ctypes.c_size_t if "size_t" in a else ctypes.c_int
                 for a in re.search(r"\b%s\(([^)]*)\)" % n, text).group(1).split(",")]
        f = ctypes.CDLL(lib._name)[n]
        f.argtypes, f.restype = kinds, ctypes.c_int
        assert f(*[0 if t is not ctypes.c_void_p else None for t in kinds]) == 1, n
        assert f(None, *[ctypes.cast(some, t) if t is ctypes.c_void_p else t(1) for t in kinds[1:]]) == 1, n
