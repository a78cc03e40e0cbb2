"""Calls of the 4-bit cache whose outputs lie over their inputs or over each other: refused on the host."""
import ctypes

import pytest

F32, BF16 = 0, 1
# a cache of 4 pages, 2 heads of 64, 16 tokens: 4096 bytes of codes and 256 of scales, twice; three tokens
CACHE = dict(K=0x10000, K_scale=0x20000, V=0x30000, V_scale=0x40000)
AT = dict(rows_k=0x50000, rows_v=0x60000, slots=0x70000, Q=0x80000, O=0x90000, lse=0xa0000, start=0xb0000, lens=0xc0000, table=0xd0000, ws=0x100000)


def cache_of(gsi):
    return gsi.KvCacheDesc(CACHE["K"], CACHE["K_scale"], CACHE["V"], CACHE["V_scale"], 4, 2, 64, 16, 0)


def ptr(at, name):
    return ctypes.c_void_p(at[name])


def refused(gsi, code):
    return code == gsi.GSI_ERR_SHAPE and "lies over" in gsi.last_error()


@pytest.mark.parametrize("over", [("rows_k", "K", 4080), ("rows_k", "V_scale", 0), ("rows_v", "K_scale", 240), ("rows_v", "V", -3 * 256 - 2 * 128 + 16),
                                  ("slots", "V", 4092), ("slots", "K", -4)])
@pytest.mark.parametrize("x", [F32, BF16])
def test_rows_that_lie_in_the_cache(over, x):
    """bf16: three rows of 256 bytes, 128 apart; fp32 twice as long."""
    from paper_2605_03109_amd import gsi

    at = dict(AT, **{over[0]: CACHE[over[1]] + over[2]})
    c = cache_of(gsi)
    assert refused(gsi, gsi.lib.gsi_kv_append(ctypes.byref(c), ptr(at, "rows_k"), ptr(at, "rows_v"), 3, 192, 192, x, ptr(at, "slots"), None))


@pytest.mark.parametrize("over", [("rows_k", CACHE["K"] + 4080), ("rows_v", CACHE["V_scale"] - 752), ("rows_k", AT["slots"]), ("rows_v", AT["rows_k"]),
                                  ("rows_v", AT["rows_k"] - 752), ("slots", AT["rows_v"] + 764)])
def test_values_over_what_they_are_read_from(over):
    from paper_2605_03109_amd import gsi

    at = dict(AT, **{over[0]: over[1]})
    c = cache_of(gsi)
    assert refused(gsi, gsi.lib.gsi_kv_expand(ctypes.byref(c), ptr(at, "slots"), 3, ptr(at, "rows_k"), ptr(at, "rows_v"), BF16, None))


# O: three rows of 4 x 64 bf16, 1536 bytes; lse 48 bytes; three starts, two lengths, a table of two by three entries
@pytest.mark.parametrize("over", [("O", AT["Q"] + 16), ("O", AT["Q"] - 1520), ("O", CACHE["K"]), ("O", CACHE["K_scale"] + 240), ("O", CACHE["V"] - 1520),
                                  ("O", CACHE["V_scale"]), ("O", AT["table"]), ("O", AT["lens"]), ("O", AT["start"]), ("lse", AT["Q"] + 1532),
                                  ("lse", AT["O"] - 44), ("lse", AT["table"] + 20), ("lse", CACHE["V"]), ("lse", AT["start"] + 8), ("lse", AT["lens"] - 44)])
def test_attention_over_its_inputs(over):
    from paper_2605_03109_amd import gsi

    at = dict(AT, **{over[0]: over[1]})
    c = cache_of(gsi)
    assert refused(gsi, gsi.lib.gsi_kv_attention(ctypes.byref(c), ptr(at, "Q"), 3, 4, 256, BF16, ptr(at, "start"), ptr(at, "lens"), 2, ptr(at, "table"), 3, 2,
                                                 48, ctypes.c_float(0.1), ptr(at, "O"), ptr(at, "lse"), ptr(at, "ws"), 1 << 20, None))


def test_attention_in_the_place_of_fused_queries():
    """Only where a row of Q is a row of O."""
    from paper_2605_03109_amd import gsi

    c = cache_of(gsi)
    at = dict(AT, O=AT["Q"])
    assert refused(gsi, gsi.lib.gsi_kv_attention(ctypes.byref(c), ptr(at, "Q"), 3, 4, 512, BF16, ptr(at, "start"), ptr(at, "lens"), 2, ptr(at, "table"), 3, 2,
                                                 48, ctypes.c_float(0.1), ptr(at, "O"), None, ptr(at, "ws"), 1 << 20, None))


@pytest.mark.parametrize("over", ["O", "Q", "table"])
def test_a_workspace_over_the_rest(over):
    from paper_2605_03109_amd import gsi

    c = cache_of(gsi)
    T, B = 2, 2
    need = gsi.lib.gsi_kv_attention_workspace_bytes(ctypes.byref(c), T, 4, BF16, B, 1, 100000)
    assert need > 0
    at = dict(AT, ws=AT[over] & ~0xff)
    assert refused(gsi, gsi.lib.gsi_kv_attention(ctypes.byref(c), ptr(at, "Q"), T, 4, 256, BF16, ptr(at, "start"), ptr(at, "lens"), B, ptr(at, "table"), 3, 1,
                                                 100000, ctypes.c_float(0.1), ptr(at, "O"), None, ptr(at, "ws"), need, None))


NAMES = ("kv_len", "n_new", "free", "n_free", "table", "out", "start", "slots", "positions", "status")


@pytest.mark.parametrize("moved,to", [("out", ("start", 8)), ("slots", ("positions", 16)), ("positions", ("table", 28)), ("status", ("slots", -4)), ("start", ("status", 4))])
def test_tables_over_each_other(moved, to):
    """Two requests, a table of two by four entries, five tokens; every tensor in a page of its own but one."""
    from paper_2605_03109_amd import gsi

    at = {n: 4096 * (i + 1) for i, n in enumerate(NAMES)}
    at[moved] = at[to[0]] + to[1]
    p = {n: ctypes.c_void_p(v) for n, v in at.items()}
    assert refused(gsi, gsi.lib.gsi_kv_tables(p["kv_len"], p["n_new"], 2, p["free"], p["n_free"], 4, p["table"], 4, 16, 5, p["out"], p["start"], p["slots"],
                                              p["positions"], p["status"], None))
