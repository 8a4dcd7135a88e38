"""Host-side checks of the key/value cache's entry points (no GPU needed): sizes, and
requests that are refused before anything is enqueued (the device addresses are fakes)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def logq():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_01127_gb300 as m
    return m


def fake(n=1):
    return 0x10000 * n


def cache_struct(logq, cb=None, v_cb=None, **kw):
    a = dict(k_codes=fake(1), k_range=fake(2), v_codes=fake(3), v_range=fake(4), pages=10, page_size=64, heads=8,
             head_dim=128, dtype=logq.LOGQ_BF16)
    a.update(kw)
    k = cb if cb is not None else logq.logq_build_codebook(4, 1.5, 1.0)
    v = v_cb if v_cb is not None else logq.logq_build_codebook(4, 1.6, 1.0)
    s = logq.KVCacheStruct(a["k_codes"], a["k_range"], a["v_codes"], a["v_range"], ctypes.pointer(k), ctypes.pointer(v),
                           a["pages"], a["page_size"], a["heads"], a["head_dim"], a["dtype"])
    s.keep = (k, v)
    return s


def test_sizes(logq):
    L = logq.lib
    assert ctypes.sizeof(logq.KVCacheStruct) == 6 * 8 + 8 + 4 * 4
    assert L.logq_kv_code_bytes(10, 64, 8, 128) == 10 * 64 * 8 * 64
    assert L.logq_kv_code_bytes(2 ** 31 - 1, 1024, 1024, 128) == (2 ** 31 - 1) * 1024 * 1024 * 64
    for bad in ((0, 64, 8, 128), (2 ** 31, 64, 8, 128), (1, 48, 8, 128), (1, 8, 8, 128), (1, 2048, 8, 128), (1, 64, 0, 128),
                (1, 64, 8, 96), (1, 64, 8, 0), (-1, 64, 8, 64)):
        assert L.logq_kv_code_bytes(*bad) == 0, bad
    assert L.logq_kv_attention_workspace_bytes(32, 8, 128) > 256
    for bad in ((0, 8, 128), (30, 8, 128), (4, 8, 128), (32, 0, 128), (32, 8, 80), (131072, 8, 128)):
        assert L.logq_kv_attention_workspace_bytes(*bad) == 0, bad


CACHE_REFUSALS = [
    (dict(k_codes=None), "INVALID_ARG"), (dict(v_range=None), "INVALID_ARG"), (dict(k_range=fake(2) + 8), "INVALID_ARG"),
    (dict(pages=0), "INVALID_ARG"), (dict(pages=2 ** 31), "INVALID_ARG"), (dict(page_size=8), "INVALID_ARG"),
    (dict(page_size=96), "INVALID_ARG"), (dict(heads=0), "INVALID_ARG"), (dict(heads=1025), "INVALID_ARG"),
    (dict(head_dim=0), "INVALID_ARG"), (dict(head_dim=96), "UNSUPPORTED"), (dict(dtype=0), "UNSUPPORTED"),
    (dict(bits=3), "UNSUPPORTED"), (dict(bits=8), "UNSUPPORTED"), (dict(range_=2.0), "INVALID_ARG"),
    (dict(qmax=3), "INVALID_ARG"),
]


@pytest.mark.parametrize("change,status", CACHE_REFUSALS, ids=lambda x: str(x))
def test_cache_refusals(logq, change, status):
    change = dict(change)
    cb = logq.logq_build_codebook(change.pop("bits", 4), 1.5, change.pop("range_", 1.0))
    cb.qmax = change.pop("qmax", cb.qmax)
    s = cache_struct(logq, v_cb=cb, **change)
    L, want = logq.lib, getattr(logq, "LOGQ_ERR_" + status)
    assert L.logq_kv_append(ctypes.byref(s), fake(5), 1024, fake(6), 1024, fake(7), 4, None, None, None) == want
    assert L.logq_kv_attention(ctypes.byref(s), fake(5), 4096, 32, 4, fake(6), fake(7), 2, fake(8), 16, 0.1, 0, 1, fake(9),
                               fake(10), 1 << 40, None) == want


def test_null_cache(logq):
    L = logq.lib
    assert L.logq_kv_append(None, fake(5), 1024, fake(6), 1024, fake(7), 4, None, None, None) == logq.LOGQ_ERR_INVALID_ARG


def test_append_refusals(logq):
    s = cache_struct(logq)

    def call(k=fake(5), ks=1024, v=fake(6), vs=1024, slots=fake(7), n=4, kv=None, vv=None):
        return logq.lib.logq_kv_append(ctypes.byref(s), k, ks, v, vs, slots, n, kv, vv, None)

    bad = logq.LOGQ_ERR_INVALID_ARG
    assert call(k=None) == bad and call(v=fake(6) + 2) == bad and call(slots=fake(7) + 4) == bad and call(slots=None) == bad
    assert call(ks=1016) == bad and call(vs=1028) == bad and call(vs=2 ** 31 + 8) == bad
    assert call(n=-1) == bad and call(n=2 ** 31) == bad
    assert call(kv=fake(8)) == bad and call(vv=fake(8)) == bad and call(kv=fake(8), vv=fake(9) + 8) == bad
    assert call(n=0, k=None, v=None, slots=None) == logq.LOGQ_OK


def test_attention_refusals(logq):
    s = cache_struct(logq)
    need = logq.logq_kv_attention_workspace_bytes(32, 8, 128)

    def call(q=fake(5), qs=4096, hq=32, n=4, q_start=fake(6), kv=fake(7), r=2, table=fake(8), width=16, scale=0.1, window=0,
             max_q=1, out=fake(9), ws=fake(10), wsb=None):
        return logq.lib.logq_kv_attention(ctypes.byref(s), q, qs, hq, n, q_start, kv, r, table, width, scale, window, max_q,
                                          out, ws, need if wsb is None else wsb, None)

    bad = logq.LOGQ_ERR_INVALID_ARG
    assert call(q=None) == bad and call(q=fake(5) + 8) == bad and call(out=None) == bad and call(out=fake(9) + 4) == bad
    assert call(q_start=None) == bad and call(kv=fake(7) + 2) == bad and call(table=None) == bad
    assert call(hq=0) == bad and call(hq=30) == bad and call(hq=65544) == bad
    assert call(qs=4088) == bad and call(qs=4100) == bad
    assert call(n=-1) == bad and call(n=2 ** 27) == bad and call(r=-1) == bad
    assert call(width=0) == bad and call(width=2 ** 30 // 64 + 1) == bad
    assert call(scale=float("nan")) == bad and call(scale=float("inf")) == bad
    assert call(window=-1) == bad and call(max_q=-1) == bad
    assert call(ws=None) == logq.LOGQ_ERR_WORKSPACE and call(ws=fake(10) + 128) == logq.LOGQ_ERR_WORKSPACE
    assert call(wsb=need - 1) == logq.LOGQ_ERR_WORKSPACE
    assert call(n=0, q=None, out=None) == logq.LOGQ_OK and call(r=0, q_start=None) == logq.LOGQ_OK


def test_plan_refusals(logq):
    names = ["ctx", "new", "r", "table", "width", "page", "ring", "ring_n", "state", "state_out", "tokens", "q_start", "kv",
             "pos", "slots", "ws", "wsb"]
    ok = dict(zip(names, [fake(1), fake(2), 3, fake(3), 8, 16, fake(4), 10, fake(5), fake(6), 7, fake(7), fake(8), fake(9),
                          fake(10), None, 0]))

    def call(**kw):
        a = {**ok, **kw}
        return logq.lib.logq_kv_plan(*[a[n] for n in names], None)

    bad = logq.LOGQ_ERR_INVALID_ARG
    for kw in (dict(ctx=None), dict(new=fake(2) + 2), dict(table=None), dict(kv=None), dict(ring=None), dict(state=None),
               dict(state_out=None), dict(q_start=None), dict(pos=None), dict(slots=fake(10) + 4), dict(r=-1), dict(tokens=-1),
               dict(tokens=2 ** 31), dict(width=0), dict(page=24), dict(page=8), dict(ring_n=0), dict(ring_n=2 ** 31)):
        assert call(**kw) == bad, kw
    # in place: the arrival count needs a workspace
    assert call(state_out=fake(5)) == logq.LOGQ_ERR_WORKSPACE
    assert call(state_out=fake(5), ws=fake(11), wsb=255) == logq.LOGQ_ERR_WORKSPACE
    assert call(state_out=fake(5), ws=fake(11) + 8, wsb=256) == logq.LOGQ_ERR_WORKSPACE


def test_binding_refuses_sizes(logq):
    with pytest.raises(logq.LogqError):
        logq.new_kv_cache(4, 48, 8, 128)
    with pytest.raises(logq.LogqError):
        logq.new_kv_workspace(30, 8, 128)
