"""Calls of the 4-bit cache that are too large for a launch, or whose outputs lie over their inputs: refused on the host."""
import ctypes

import pytest

ONE = ctypes.c_void_p(256)  # never dereferenced


def cache_of(gsi, heads, dim):
    return gsi.KvCacheDesc(256, 256, 256, 256, 4, heads, dim, 16, 0)


@pytest.mark.parametrize("heads,dim,T", [(4096, 256, 1 << 16), (1, 32, 1 << 29), (8, 128, 1 << 26)])
def test_more_rows_than_a_launch_takes(heads, dim, T):
    """A launch has fewer than 2^24 workgroups of 16 tokens x 128 elements."""
    from paper_2605_03109_amd import gsi

    c = cache_of(gsi, heads, dim)
    row = heads * dim
    assert gsi.lib.gsi_kv_append(ctypes.byref(c), ONE, ONE, T, row, row, 0, ONE, None) == gsi.GSI_ERR_SHAPE
    assert gsi.lib.gsi_kv_expand(ctypes.byref(c), ONE, T, ONE, ONE, 1, None) == gsi.GSI_ERR_SHAPE


def test_more_tiles_than_a_launch_takes():
    from paper_2605_03109_amd import gsi

    c = cache_of(gsi, 4096, 64)
    B = 1 << 14
    assert gsi.lib.gsi_kv_attention(ctypes.byref(c), ONE, B, 4096, 4096 * 64, 0, ONE, ONE, B, ONE, 3, 1, 48, ctypes.c_float(0.1), ONE, None, ONE, 1 << 50,
                                    None) == gsi.GSI_ERR_SHAPE
    assert gsi.lib.gsi_kv_attention_workspace_bytes(ctypes.byref(c), B, 4096, 0, B, 1, 48) == 0


NAMES = ("kv_len", "n_new", "free", "n_free", "table", "out", "start", "slots", "positions", "status")


@pytest.mark.parametrize("moved,to,code", [
    ("out", ("kv_len", 4), "SHAPE"), ("out", ("kv_len", -4), "SHAPE"), ("out", ("n_new", 0), "SHAPE"), ("start", ("n_new", 4), "SHAPE"),
    ("slots", ("free", 12), "SHAPE"), ("status", ("n_free", -4), "SHAPE"), ("table", ("free", -28), "SHAPE"), ("positions", ("kv_len", 0), "SHAPE"),
    ("positions", ("kv_len", 2), "ALIGN"), ("status", ("n_free", 1), "ALIGN")])
def test_outputs_over_inputs(moved, to, code):
    """Two requests, four free pages, a table of two by four entries, five tokens; every tensor in a page of its own but one."""
    from paper_2605_03109_amd import gsi

    at = {n: 4096 * (i + 1) for i, n in enumerate(NAMES)}
    at[moved] = at[to[0]] + to[1]
    p = {n: ctypes.c_void_p(v) for n, v in at.items()}
    assert gsi.lib.gsi_kv_tables(p["kv_len"], p["n_new"], 2, p["free"], p["n_free"], 4, p["table"], 4, 16, 5, p["out"], p["start"], p["slots"],
                                 p["positions"], p["status"], None) == getattr(gsi, "GSI_ERR_" + code)


@pytest.mark.parametrize("T", [-1, (1 << 29) + 1])
def test_steps_of_too_many_tokens(T):
    from paper_2605_03109_amd import gsi

    p = [ctypes.c_void_p(4096 * (i + 1)) for i in range(10)]
    assert gsi.lib.gsi_kv_tables(p[0], p[1], 2, p[2], p[3], 4, p[4], 4, 16, T, *p[5:], None) == gsi.GSI_ERR_SHAPE
