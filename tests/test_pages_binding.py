"""Refusals of the page calls, on the host: nothing is launched."""
import ctypes

import pytest

from pages_util import Model, filled, n_pages_of
from paper_2607_07740_amd import api

P = ctypes.c_void_p
A, MIS = P(0x1000), P(0x1002)
BAD, UNS = api.JL_ERR_INVALID_ARG, api.JL_ERR_UNSUPPORTED


def _table(**kw):
    d = dict(table=0x1000, lens=0x2000, refs=0x3000, B=4, max_pages=8, n_pages=32, page_size=64)
    d.update(kw)
    return api._PagesStruct(*[d[n] for n, _ in api._PagesStruct._fields_])


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), BAD), (dict(max_pages=0), BAD), (dict(n_pages=0), BAD), (dict(page_size=0), BAD),
    (dict(table=None), BAD), (dict(lens=None), BAD), (dict(refs=None), BAD),
    (dict(table=0x1002), BAD), (dict(lens=0x1001), BAD), (dict(refs=0x1004), BAD),
    (dict(max_pages=1 << 20, page_size=1 << 11), BAD), (dict(B=2049), UNS),
    (dict(n_pages=(1 << 30) + 1), UNS)])
def test_tables_are_checked(kw, code):
    L, t = api.lib(), _table(**kw)
    r = ctypes.byref(t)
    assert L.jl_pages_fork(r, A, None) == code
    assert L.jl_pages_reserve(r, A, A, A, A, A, None) == code
    assert L.jl_pages_compact(r, A, A, A, None) == code
    assert L.jl_last_error().decode() != ""


def test_arguments_beside_the_table_are_checked():
    L, t = api.lib(), _table()
    r = ctypes.byref(t)
    for x in (None, MIS):
        assert L.jl_pages_fork(r, x, None) == BAD
        for i in range(5):
            args = [A] * 5
            args[i] = x
            assert L.jl_pages_reserve(r, *args, None) == BAD
        for i in range(3):
            args = [A] * 3
            args[i] = x
            assert L.jl_pages_compact(r, *args, None) == BAD
    assert L.jl_pages_fork(None, A, None) == BAD
    assert L.jl_pages_reserve(None, A, A, A, A, A, None) == BAD
    assert L.jl_pages_compact(None, A, A, A, None) == BAD


def test_pools_are_checked():
    L = api.lib()

    def call(ptr=0x1000, size=64, n=1, n_pages=4, moves=A, count=A, most=2):
        pool = (api._PoolStruct * 2)((0x1000, 64), (ptr, size))
        return L.jl_copy_pages(pool, n + 1 if n else 0, n_pages, moves, count, most, None)

    assert call(ptr=None) == BAD and call(ptr=0x1002) == BAD
    assert call(size=0) == BAD and call(size=2) == BAD and call(size=66) == BAD
    assert call(n=0) == BAD and call(n_pages=0) == BAD and call(most=-1) == BAD
    assert call(moves=None) == BAD and call(count=MIS) == BAD
    assert call(size=1 << 50, n_pages=1 << 20) == BAD  # past 62 bits in all
    assert call(size=1 << 46) == BAD  # units of a move past 32 bits
    assert L.jl_copy_pages(None, 1, 4, A, A, 2, None) == BAD
    assert call(most=0) == api.JL_OK  # nothing to do, nothing launched


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), BAD), (dict(n=0), BAD), (dict(Hkv=0), BAD), (dict(n_pages=0), BAD),
    (dict(page=0), BAD), (dict(d=127), BAD), (dict(d=64), UNS), (dict(k=None), BAD),
    (dict(v=MIS), BAD), (dict(kc=P(0x1008)), BAD), (dict(vc=None), BAD), (dict(starts=None), BAD),
    (dict(n_new=MIS), BAD), (dict(cu=MIS), BAD), (dict(table=MIS), BAD), (dict(max_pages=0), BAD),
    (dict(max_pages=1 << 20, page=1 << 11), BAD), (dict(table=None, B=33), BAD),
    (dict(B=1 << 16, n=1 << 16), BAD), (dict(Hkv=1 << 28), BAD)])
def test_append_arguments_are_checked(kw, code):
    d = dict(kc=A, vc=A, n_pages=32, page=64, table=A, max_pages=8, k=A, v=A, starts=A, n_new=None,
             cu=None, B=4, n=2, Hkv=2, d=128)
    d.update(kw)
    assert api.lib().jl_cache_append(
        d["kc"], d["vc"], d["n_pages"], d["page"], d["table"], d["max_pages"], d["k"], d["v"],
        d["starts"], d["n_new"], d["cu"], d["B"], d["n"], d["Hkv"], d["d"], None) == code


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    with pytest.raises(TypeError):
        api.pages_alloc(2, 3, 4, 64, device="cpu")
    with pytest.raises(TypeError):
        api.pages_fork(None, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        api.pages_reserve("pages", torch.zeros(2, dtype=torch.int32))
    x = torch.zeros((2, 4, 2, 128), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        api.cache_append(x, x, x, x, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        api.copy_pages([x], torch.zeros((1, 2), dtype=torch.int32), torch.ones(1, dtype=torch.int32))


def test_the_model_keeps_its_counts():
    import numpy as np
    rng = np.random.default_rng(0)
    m = filled(rng, 20, 10, 150, 8)
    for _ in range(30):
        m.fork([int(x) for x in rng.integers(-1, 20, 20)])
        m.reserve([int(x) for x in rng.integers(0, 5, 20)])
        m.compact()
        refs = list(m.refs)
        m.count()
        assert refs == m.refs
        assert all(sum(p >= 0 for p in r) == n_pages_of(n, 8) for r, n in zip(m.table, m.lens))


def _plan(fn="jl_bifocal_shared_plan", **kw):
    d = dict(lens=A, members=None, starts=A, shared=A, B=4, n=2, Hq=8, Hkv=2, d=128, max_pages=8,
             page=64, w=32, w0=4, plan=A, bytes=1 << 20)
    d.update(kw)
    views = (d["w"], d["w0"]) if "bifocal" in fn else ()
    return getattr(api.lib(), fn)(d["lens"], d["members"], d["starts"], d["shared"], d["B"], d["n"],
                                  d["Hq"], d["Hkv"], d["d"], d["max_pages"], d["page"], *views,
                                  d["plan"], d["bytes"], None)


SIZES = [(dict(B=0), BAD), (dict(n=0), BAD), (dict(Hq=7), BAD), (dict(Hkv=0), BAD), (dict(d=64), UNS),
         (dict(d=3), BAD), (dict(Hq=18), UNS), (dict(B=2049), UNS), (dict(n=2049), UNS),
         (dict(page=8), BAD), (dict(page=48), BAD), (dict(max_pages=0), BAD),
         (dict(max_pages=1 << 18), UNS), (dict(Hq=1 << 17, Hkv=1 << 17), BAD)]


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(lens=None), BAD), (dict(starts=MIS), BAD), (dict(shared=None), BAD), (dict(members=MIS), BAD),
    (dict(plan=None), api.JL_ERR_WORKSPACE), (dict(bytes=64), api.JL_ERR_WORKSPACE),
    (dict(plan=P(0x1008)), BAD)])
def test_plan_arguments_are_checked(kw, code):
    assert _plan(**kw) == code
    assert _plan("jl_rope_shared_plan", **kw) == code


def test_plan_windows_are_checked():
    assert _plan(w=0) == BAD and _plan(w0=-1) == BAD


@pytest.mark.parametrize("kw,code", SIZES + [
    (dict(q=None), BAD), (dict(k=MIS), BAD), (dict(v=None), BAD), (dict(o=P(0x1004)), BAD),
    (dict(table=None), BAD), (dict(plan=None), api.JL_ERR_WORKSPACE), (dict(theta=0.0), BAD),
    (dict(plan_bytes=8), api.JL_ERR_WORKSPACE), (dict(ws=None), api.JL_ERR_WORKSPACE),
    (dict(ws_bytes=100), api.JL_ERR_WORKSPACE), (dict(ws=P(0x1004)), BAD), (dict(n_pages=0), BAD),
    (dict(n_pages=1 << 26), UNS), (dict(theta=float("inf")), BAD)])
def test_shared_decode_arguments_are_checked(kw, code):
    d = dict(q=A, k=A, v=A, table=A, max_pages=8, page=64, n_pages=32, plan=A, plan_bytes=1 << 24, o=A,
             B=4, n=2, Hq=8, Hkv=2, d=128, theta=1e6, ws=A, ws_bytes=1 << 40)
    d.update(kw)
    head = (d["q"], d["k"], d["v"], d["table"], d["max_pages"], d["page"], d["n_pages"], d["plan"],
            d["plan_bytes"], d["o"], d["B"], d["n"], d["Hq"], d["Hkv"], d["d"], d["theta"])
    L = api.lib()
    assert L.jl_bifocal_decode_shared(*head, 32, 4, d["ws"], d["ws_bytes"], None) == code
    assert L.jl_rope_attention_decode_shared(*head, d["ws"], d["ws_bytes"], None) == code


def test_sizes_of_plans_and_workspaces():
    assert api.shared_plan_bytes(4, 2, 8, 2) > 0
    assert api.decode_shared_workspace_bytes(4, 8, 2) % 16 == 0
    for bad in ((0, 1, 8, 2), (4, 0, 8, 2), (4, 1, 7, 2), (4, 1, 18, 2), (4096, 1, 8, 2)):
        assert api.shared_plan_bytes(*bad) == 0
    assert api.decode_shared_workspace_bytes(4, 8, 2, 64) == 0
    assert api.decode_shared_workspace_bytes(4096, 8, 2) == 0
    one, two = (api.varlen_paged_workspace_bytes(4, t, 8, 2, 64, 64) for t in (40, 4000))
    assert 0 < one < two
    for bad in ((0, 40, 8, 2, 64, 64), (4, 0, 8, 2, 64, 64), (4, 40, 7, 2, 64, 64),
                (4, 40, 8, 2, 0, 64), (4, 40, 8, 2, 64, 48), (2049, 40, 8, 2, 64, 64),
                (4, 40, 8, 2, 64, 64, 96), (4, 1 << 21, 8, 2, 64, 64)):
        assert api.varlen_paged_workspace_bytes(*bad) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), BAD), (dict(T=0), BAD), (dict(Hq=7), BAD), (dict(Hkv=0), BAD), (dict(d=64), UNS),
    (dict(d=5), BAD), (dict(Hq=514), UNS), (dict(B=2049), UNS), (dict(T=1 << 21), UNS),
    (dict(T=1 << 30, Hq=512, Hkv=256), UNS), (dict(page=8), BAD), (dict(page=80), BAD),
    (dict(max_pages=0), BAD), (dict(max_pages=1 << 18), UNS), (dict(n_pages=0), BAD),
    (dict(n_pages=1 << 26), UNS), (dict(theta=-1.0), BAD), (dict(q=None), BAD), (dict(k=MIS), BAD),
    (dict(v=None), BAD), (dict(o=P(0x1008)), BAD), (dict(lse=MIS), BAD), (dict(table=None), BAD),
    (dict(cu=MIS), BAD), (dict(lens=None), BAD), (dict(ws=None), api.JL_ERR_WORKSPACE),
    (dict(ws_bytes=4096), api.JL_ERR_WORKSPACE),
    (dict(ws=P(0x1008)), BAD)])
def test_chunk_arguments_are_checked(kw, code):
    d = dict(q=A, k=A, v=A, table=A, max_pages=8, page=64, n_pages=32, cu=A, lens=A, o=A, lse=None,
             B=4, T=20, Hq=8, Hkv=2, d=128, theta=1e6, ws=A, ws_bytes=1 << 40)
    d.update(kw)
    ws = (d["ws"], d["ws_bytes"], None)
    head = (d["q"], d["k"], d["v"], d["table"], d["max_pages"], d["page"], d["n_pages"], d["cu"],
            d["lens"], d["o"], d["lse"], d["B"], d["T"], d["Hq"], d["Hkv"], d["d"], d["theta"])
    L = api.lib()
    assert L.jl_bifocal_prefill_varlen_paged(*head, 32, 4, *ws) == code
    assert L.jl_rope_attention_varlen_paged(*head, *ws) == code
    for w in ((0, 4), (32, -1)):
        assert L.jl_bifocal_prefill_varlen_paged(*head, *w, *ws) in (BAD, code)


def test_packed_chunks_take_as_many_sequences_as_they_say():
    """2048 of them, of a token each or with as many rows as a few sequences may have."""
    for g, T in ((1, 1300000), (4, 327000), (8, 163000), (100, 10000), (256, 5000)):
        few, many = (api.varlen_paged_workspace_bytes(B, T, g, 1, 64, 64) for B in (1, 2048))
        assert 0 < few < many
        assert api.varlen_paged_workspace_bytes(2048, 2048, g, 1, 64, 64) > 0
        assert api.varlen_paged_workspace_bytes(1, 2 * T, g, 1, 64, 64) == 0
