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
