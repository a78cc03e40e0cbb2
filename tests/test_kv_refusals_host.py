"""What the calls of the 4-bit cache refuse, on the host before anything is enqueued, and the binding's own checks."""
import ctypes

import pytest
import torch


def cache_of(gsi, **kw):
    f = dict(K=256, K_scale=256, V=256, V_scale=256, n_pages=4, heads=2, dim=64, page=16, reserved=0)
    f.update(kw)
    return gsi.KvCacheDesc(*[f[n] for n, _ in gsi.KvCacheDesc._fields_])


ONE = ctypes.c_void_p(256)  # never dereferenced
F32 = ctypes.c_float(0.1)


def append(gsi, c, K=ONE, V=ONE, T=3, ks=128, vs=128, dt=0, slots=ONE):
    return gsi.lib.gsi_kv_append(ctypes.byref(c) if c is not None else None, K, V, T, ks, vs, dt, slots, None)


def attend(gsi, c, Q=ONE, T=3, heads=4, qs=256, dt=0, start=ONE, lens=ONE, B=2, table=ONE, width=3, max_q=1, max_len=48, scale=F32, O=ONE, lse=None,
           ws=ONE, wsn=1 << 40):
    return gsi.lib.gsi_kv_attention(ctypes.byref(c), Q, T, heads, qs, dt, start, lens, B, table, width, max_q, max_len, scale, O, lse, ws, wsn, None)


@pytest.mark.parametrize("field,value,code", [("K", None, "NULL"), ("V_scale", None, "NULL"), ("heads", 0, "SHAPE"), ("dim", 48, "SHAPE"), ("dim", 288, "SHAPE"),
                                              ("dim", 0, "SHAPE"), ("page", 24, "SHAPE"), ("page", 8, "SHAPE"), ("page", 8192, "SHAPE"), ("n_pages", 0, "SHAPE"),
                                              ("n_pages", 1 << 30, "SHAPE"), ("reserved", 1, "SHAPE"), ("K", 264, "ALIGN"), ("V_scale", 257, "ALIGN")])
def test_a_cache_that_no_call_takes(field, value, code):
    from paper_2605_03109_amd import gsi

    c = cache_of(gsi, **{field: value})
    want = getattr(gsi, "GSI_ERR_" + code)
    assert append(gsi, c) == want and attend(gsi, c) == want
    assert gsi.lib.gsi_kv_expand(ctypes.byref(c), ONE, 3, ONE, ONE, 0, None) == want
    assert gsi.lib.gsi_kv_attention_workspace_bytes(ctypes.byref(c), 3, 4, 0, 2, 1, 48) == 0


def test_rows():
    from paper_2605_03109_amd import gsi

    c = cache_of(gsi)
    assert append(gsi, None) == gsi.GSI_ERR_NULL
    assert append(gsi, c, T=0, K=None) == gsi.GSI_OK
    assert append(gsi, c, T=-1) == gsi.GSI_ERR_SHAPE
    assert append(gsi, c, K=None) == gsi.GSI_ERR_NULL and append(gsi, c, slots=None) == gsi.GSI_ERR_NULL
    assert append(gsi, c, dt=2) == gsi.GSI_ERR_DTYPE
    assert append(gsi, c, ks=127) == gsi.GSI_ERR_SHAPE and append(gsi, c, vs=1) == gsi.GSI_ERR_SHAPE
    assert append(gsi, c, K=ctypes.c_void_p(258)) == gsi.GSI_ERR_ALIGN
    expand = lambda **k: gsi.lib.gsi_kv_expand(ctypes.byref(c), k.get("slots", ONE), k.get("T", 3), k.get("K", ONE), ONE, k.get("dt", 1), None)  # noqa: E731
    assert expand(K=None) == gsi.GSI_ERR_NULL and expand(slots=None) == gsi.GSI_ERR_NULL
    assert expand(K=ctypes.c_void_p(264)) == gsi.GSI_ERR_ALIGN and expand(dt=5) == gsi.GSI_ERR_DTYPE
    assert expand(T=0, K=None) == gsi.GSI_OK and expand(T=-2) == gsi.GSI_ERR_SHAPE


def test_tables():
    from paper_2605_03109_amd import gsi

    def tables(**k):
        two = ctypes.c_void_p(512)
        return gsi.lib.gsi_kv_tables(k.get("len", ONE), k.get("new", ONE), k.get("B", 2), k.get("free", ONE), k.get("n_free", ONE), k.get("cap", 4),
                                     k.get("table", ONE), k.get("width", 4), k.get("page", 16), k.get("T", 5), k.get("out", two), two, k.get("slots", two),
                                     two, k.get("status", two), None)

    assert tables(B=0, len=None) == gsi.GSI_OK
    for bad in ({"B": -1}, {"B": 16385}, {"T": -1}, {"page": 17}, {"page": 8}, {"width": 0}, {"cap": -1}, {"out": ONE}):
        assert tables(**bad) == gsi.GSI_ERR_SHAPE, bad
    for bad in ({"len": None}, {"new": None}, {"free": None}, {"n_free": None}, {"table": None}, {"out": None}, {"slots": None}, {"status": None}):
        assert tables(**bad) == gsi.GSI_ERR_NULL, bad
    assert tables(table=ctypes.c_void_p(258)) == gsi.GSI_ERR_ALIGN


def test_attention():
    from paper_2605_03109_amd import gsi

    c = cache_of(gsi)
    assert attend(gsi, c, T=0, Q=None, start=None, B=0) == gsi.GSI_OK
    for bad in ({"heads": 3}, {"heads": 0}, {"T": -1}, {"B": -1}, {"qs": 255}, {"width": 0}, {"max_q": 0}, {"max_len": 0}, {"start": None},
                {"scale": ctypes.c_float(float("nan"))}, {"scale": ctypes.c_float(float("inf"))}, {"width": 1 << 27}):
        assert attend(gsi, c, **bad) == gsi.GSI_ERR_SHAPE, bad
    for bad in ({"Q": None}, {"O": None}, {"lens": None}, {"table": None}):
        assert attend(gsi, c, **bad) == gsi.GSI_ERR_NULL, bad
    assert attend(gsi, c, dt=2) == gsi.GSI_ERR_DTYPE
    for bad in ({"Q": ctypes.c_void_p(258)}, {"O": ctypes.c_void_p(260)}, {"lse": ctypes.c_void_p(258)}, {"table": ctypes.c_void_p(257)}):
        assert attend(gsi, c, **bad) == gsi.GSI_ERR_ALIGN, bad


def test_the_binding_checks_tensors():
    from paper_2605_03109_amd import gsi

    u8 = dict(dtype=torch.uint8)
    with pytest.raises(ValueError):  # host tensors
        gsi.KvCache(torch.zeros(2, 1, 16, 16, **u8), torch.zeros(2, 1, 1, 16, **u8), torch.zeros(2, 1, 16, 16, **u8), torch.zeros(2, 1, 1, 16, **u8))
    with pytest.raises(ValueError):
        gsi.KvCache(torch.zeros(2, 1, 16, 16, **u8), torch.zeros(2, 1, 16, 1, **u8), torch.zeros(2, 1, 16, 16, **u8), torch.zeros(2, 1, 16, 1, **u8))
    with pytest.raises(ValueError):
        gsi._i32("slots", torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError):
        gsi._i32("slots", torch.zeros(3, dtype=torch.int32), 4)
