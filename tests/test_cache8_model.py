"""The fp64 model of the 8-bit cache that the GPU tests compare with, and the refusals of the
8-bit entry points, on the CPU."""
import ctypes
import math

import numpy as np
import pytest

import cache8_util as C
from paper_2607_07740_amd import api

P = ctypes.c_void_p
A, A2, MIS = P(0x1000), P(0x2000), P(0x1002)


# ------------------------------------------------------------------ the model
def test_e4m3_rounds_to_the_nearest_number_ties_to_even():
    finite = np.array(sorted({x for x in C.E4M3 if not math.isnan(x)}))
    assert finite[-1] == 448.0 and len(finite) == 253
    assert (C.E4M3[C.e4m3(finite)] == finite).all()
    mid = (finite[1:] + finite[:-1]) / 2  # a tie goes to the even mantissa
    got = C.e4m3(mid) & 127
    assert (got % 2 == 0).all()
    assert (np.abs(C.E4M3[C.e4m3(mid)] - mid) == (finite[1:] - finite[:-1]) / 2).all()
    x = np.random.default_rng(0).standard_normal(20000) * 100
    near = finite[np.abs(x[:, None] - finite[None]).argmin(1)]
    assert (C.E4M3[C.e4m3(x)] == near).all()
    assert C.E4M3[C.e4m3(1e9)] == 448.0 and C.E4M3[C.e4m3(-math.inf)] == -448.0
    assert math.isnan(C.E4M3[C.e4m3(math.nan)])


def test_scale_is_the_smallest_power_of_two_that_holds_the_block():
    for top in (1e-30, 0.1, 1.0, 447.9, 448.0, 448.1, 896.0, 3e30):
        s = float(C.scale_of(top))
        assert top <= 448 * s and top > 448 * s / 2
    assert C.scale_of(0.0) == 2.0 ** -117 and C.scale_of(C.BF16_MAX) == 2.0 ** 119
    # every value of the cache is a bf16
    for e in (-117, 0, 119):
        x = C.E4M3[~np.isnan(C.E4M3)] * 2.0 ** e
        assert (C.to_bf16(x) == x).all()


def test_images_are_permutations():
    y = np.arange(C.BLOCK * C.D).reshape(C.BLOCK, C.D)
    for pack in (C.pack_k, C.pack_v):
        assert (np.sort(pack(y)) == np.arange(C.BLOCK * C.D)).all()
    k = C.pack_k(y).reshape(2, 2, 2, 4, 16, 8, 2)
    assert k[1, 0, 1, 3, 7, 5, 1] == y[32 + 7, 64 + 32 + 24 + 5]
    v = C.pack_v(y).reshape(2, 4, 4, 16, 2, 2, 4)
    assert v[1, 3, 2, 9, 1, 0, 3] == y[32 + 8 + 3, 96 + 16 + 9]


def test_model_attention_is_the_dense_definition():
    from oracle import oracle as O
    from paper_2607_07740_amd import synth
    q, kc, vc, lens = synth.decode_inputs(2, 4, 2, 192, [190, 70], seed=3)
    m = C.Model(2, 3, 2)
    f = lambda x: synth.bf16_to_f32(x).astype(np.float64)  # noqa: E731
    m.append(f(kc), f(vc), [0, 0])
    kd, vd = (synth.bf16_bits(m.rows(x).astype(np.float32)) for x in "kv")
    want, _, _ = O.decode(q, kd, vd, lens, theta=1e6, w_pretrained=64, w_local=20)
    got, _ = C.decode(f(q), m, lens, 64, 20)
    assert np.abs(got - want).max() < 1e-12


def test_appending_in_pieces_gives_the_same_rows_where_no_scale_moves():
    rng = np.random.default_rng(1)
    x = C.to_bf16(rng.standard_normal((1, 150, 2, C.D)))
    x[:, :, :, 0] = 4.0  # fixes every block's scale from its first row on
    x = np.clip(x, -4, 4)
    one, many = C.Model(1, 3, 2), C.Model(1, 3, 2)
    one.append(x, x, [0])
    at = 0
    for n in (1, 62, 1, 1, 40, 45):
        many.append(x[:, at:at + n], x[:, at:at + n], [at])
        at += n
    for a, b in ((one.k, many.k), (one.v, many.v), (one.ks, many.ks), (one.mean, many.mean)):
        assert (a == b).all()


# ------------------------------------------------------------------ refusals
class Cache(ctypes.Structure):
    _fields_ = api._Cache8Struct._fields_


def _cache(**kw):
    a = dict(k=0x1000, v=0x2000, k_scale=0x3000, v_scale=0x4000, k_mean=0x5000, n_pages=4,
             page_size=128, Hkv=2, head_dim=128)
    a.update(kw)
    return Cache(**a)


def _entries(cache, table=A, max_pages=2, B=2, Hq=8, q=A, lens=A2, o=A, theta=1e6, w=64, w0=8,
             ws=A, ws_bytes=1 << 30, blocks=A2, n_select=4, scores=A):
    """Every entry point that takes a cache, by name."""
    L = api.lib()
    ref = None if cache is None else ctypes.byref(cache)
    head = (ref, table, max_pages)
    return {
        "append": lambda: L.jl_cache8_append(*head, A, A, A2, None, B, 5, None),
        "read": lambda: L.jl_cache8_read(*head, A, A, B, 0, 64, None),
        "decode": lambda: L.jl_bifocal_decode8(*head, q, lens, o, B, Hq, theta, w, w0, ws,
                                               ws_bytes, None),
        "rope": lambda: L.jl_rope_attention_decode8(*head, q, lens, o, B, Hq, theta, ws, ws_bytes,
                                                    None),
        "blocks": lambda: L.jl_bifocal_decode8_blocks(*head, q, lens, blocks, n_select, o, B, Hq,
                                                      theta, w, w0, ws, ws_bytes, None),
        "rope_blocks": lambda: L.jl_rope_attention_decode8_blocks(
            *head, q, lens, blocks, n_select, o, B, Hq, theta, ws, ws_bytes, None),
        "scores": lambda: L.jl_bifocal_block_scores8(*head, q, lens, scores, B, Hq, theta, w,
                                                     None),
        "rope_scores": lambda: L.jl_rope_block_scores8(*head, q, lens, scores, B, Hq, theta, None),
    }


def _refused(entries, names, code):
    for name in names:
        assert entries[name]() == code, (name, api.lib().jl_last_error())
        assert api.lib().jl_last_error().decode() != "", name


ALL = ("append", "read", "decode", "rope", "blocks", "rope_blocks", "scores", "rope_scores")
QUERY = ("decode", "rope", "blocks", "rope_blocks", "scores", "rope_scores")
DECODE = ("decode", "rope", "blocks", "rope_blocks")
BIFOCAL = ("decode", "blocks")


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), api.JL_ERR_INVALID_ARG), (dict(v=0x1008), api.JL_ERR_INVALID_ARG),
    (dict(k_mean=None), api.JL_ERR_INVALID_ARG), (dict(k_scale=None), api.JL_ERR_INVALID_ARG),
    (dict(v_scale=0x1002), api.JL_ERR_INVALID_ARG), (dict(n_pages=0), api.JL_ERR_INVALID_ARG),
    (dict(Hkv=0), api.JL_ERR_INVALID_ARG), (dict(page_size=0), api.JL_ERR_INVALID_ARG),
    (dict(page_size=96), api.JL_ERR_INVALID_ARG), (dict(page_size=32), api.JL_ERR_INVALID_ARG),
    (dict(head_dim=64), api.JL_ERR_UNSUPPORTED), (dict(head_dim=127), api.JL_ERR_INVALID_ARG),
    (dict(n_pages=1 << 30), api.JL_ERR_UNSUPPORTED),
    (dict(page_size=1 << 23), api.JL_ERR_UNSUPPORTED),  # two pages: past 2^23 positions
])
def test_every_entry_refuses_a_bad_cache(kw, code):
    _refused(_entries(_cache(**kw)), ALL, code)


def test_every_entry_refuses_bad_pages_and_batches():
    _refused(_entries(None), ALL, api.JL_ERR_INVALID_ARG)
    _refused(_entries(_cache(), table=MIS), ALL, api.JL_ERR_INVALID_ARG)
    _refused(_entries(_cache(), max_pages=0), ALL, api.JL_ERR_INVALID_ARG)
    _refused(_entries(_cache(), B=0), ALL, api.JL_ERR_INVALID_ARG)
    _refused(_entries(_cache(), table=None, B=5), ALL, api.JL_ERR_INVALID_ARG)  # 4 sequences
    _refused(_entries(_cache(Hkv=16384, n_pages=100), B=1 << 16, Hq=16384, n_select=1 << 10),
             QUERY, api.JL_ERR_INVALID_ARG)


def test_queries_and_outputs_are_checked():
    c = _cache()
    _refused(_entries(c, Hq=7), QUERY, api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, Hq=0), QUERY, api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, Hq=18), QUERY, api.JL_ERR_UNSUPPORTED)  # a group of 9
    for theta in (0.0, -1.0, math.nan, math.inf):
        _refused(_entries(c, theta=theta), QUERY, api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, q=None), QUERY, api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, q=P(0x1004)), QUERY, api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, lens=None), QUERY, api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, lens=MIS), QUERY, api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, o=None), DECODE, api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, w=0), BIFOCAL + ("scores",), api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, w0=-1), BIFOCAL, api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, ws=None), DECODE, api.JL_ERR_WORKSPACE)
    need = api.decode8_workspace_bytes(8, 2)
    _refused(_entries(c, ws_bytes=need - 1), DECODE, api.JL_ERR_WORKSPACE)
    _refused(_entries(c, ws=P(0x1008)), DECODE, api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, blocks=None), ("blocks", "rope_blocks"), api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, n_select=0), ("blocks", "rope_blocks"), api.JL_ERR_INVALID_ARG)
    _refused(_entries(c, scores=None), ("scores", "rope_scores"), api.JL_ERR_INVALID_ARG)
    assert need > 4096 and api.decode8_workspace_bytes(8, 3) == 0
    assert api.decode8_workspace_bytes(18, 2) == 0 and api.decode8_workspace_bytes(8, 2, 64) == 0


def test_append_and_read_are_checked():
    L, c = api.lib(), _cache()
    ref = ctypes.byref(c)

    def append(k=A, v=A, starts=A2, n_new=None, B=2, n=5):
        return L.jl_cache8_append(ref, A, 2, k, v, starts, n_new, B, n, None)
    for kw in (dict(k=None), dict(v=P(0x1008)), dict(starts=None), dict(starts=MIS), dict(n=0),
               dict(n_new=MIS), dict(n=2 ** 31 - 1, B=100)):
        assert append(**kw) == api.JL_ERR_INVALID_ARG, kw
    for start, n in ((-1, 4), (0, 0), (0, 257), (256, 1), (2 ** 31 - 1, 2 ** 31 - 1)):
        assert L.jl_cache8_read(ref, A, 2, A, A, 2, start, n, None) == api.JL_ERR_INVALID_ARG
    assert L.jl_cache8_read(ref, A, 2, None, A, 2, 0, 4, None) == api.JL_ERR_INVALID_ARG
    assert L.jl_cache8_read(ref, A, 2, A, P(0x1004), 2, 0, 4, None) == api.JL_ERR_INVALID_ARG


def _select(scores=A, lens=A2, blocks=A, B=1, Hkv=2, n_blocks=100, n_select=20, w_local=64,
            n_first=1):
    return api.lib().jl_select_blocks(scores, lens, blocks, B, Hkv, n_blocks, n_select, w_local,
                                      n_first, None)


@pytest.mark.parametrize("kw,code", [
    (dict(scores=None), api.JL_ERR_INVALID_ARG), (dict(lens=MIS), api.JL_ERR_INVALID_ARG),
    (dict(blocks=None), api.JL_ERR_INVALID_ARG), (dict(B=0), api.JL_ERR_INVALID_ARG),
    (dict(Hkv=0), api.JL_ERR_INVALID_ARG), (dict(n_blocks=0), api.JL_ERR_INVALID_ARG),
    (dict(n_select=0), api.JL_ERR_INVALID_ARG), (dict(w_local=-1), api.JL_ERR_INVALID_ARG),
    (dict(n_first=-1), api.JL_ERR_INVALID_ARG), (dict(n_blocks=131073), api.JL_ERR_UNSUPPORTED),
    (dict(n_select=2, w_local=64), api.JL_ERR_INVALID_ARG),  # the band may lie in 2 blocks, + 1
    (dict(n_select=3, w_local=65), api.JL_ERR_INVALID_ARG),  # 66 keys in 3 blocks
    (dict(n_select=99, w_local=2 ** 31 - 1), api.JL_ERR_INVALID_ARG),  # the whole sequence
    (dict(B=65536, Hkv=1024), api.JL_ERR_INVALID_ARG),
])
def test_select_refuses(kw, code):
    assert _select(**kw) == code
    assert api.lib().jl_last_error().decode() != ""


def test_a_band_never_lies_in_more_blocks_than_the_check_counts():
    for w0 in range(0, 300):
        most = max(len({k // 64 for k in range(max(0, q - w0), q + 1)}) for q in range(0, 600))
        assert most <= (w0 + 127) // 64
        if w0 < 250:
            assert most == (w0 + 127) // 64
