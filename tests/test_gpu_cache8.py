"""The 8-bit cache on the GPU: appended rows against the fp64 model byte for byte, rows read
back, decode over all keys and over listed blocks, block scores and their choice."""
import math

import numpy as np
import pytest

import cache8_util as C
from paper_2607_07740_amd import api
from parity_util import say

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def dev(x, dtype=BF):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(dtype).cuda()


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def normals(rng, *shape, size=1.0):
    return C.to_bf16(rng.standard_normal(shape) * size)


def upload(p):
    k, v, ks, vs, mean = p
    return api.Cache8(torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(),
                      dev(ks, torch.float32), dev(vs, torch.float32), dev(mean))


def paged(B, max_pages, spare, seed):
    rng = np.random.default_rng(seed)
    n = B * max_pages + spare
    return rng.permutation(n)[:B * max_pages].reshape(B, max_pages).astype(np.int32), n


def filled(rng, B, nb, Hkv, lens, size=1.0):
    """A model whose sequences hold lens[b] normals, K and V of different sizes per head."""
    m = C.Model(B, nb, Hkv)
    heads = 2.0 ** rng.uniform(-2, 2, (1, 1, Hkv, 1))
    n = max(max(lens), 1)
    m.append(normals(rng, B, n, Hkv, C.D), C.to_bf16(normals(rng, B, n, Hkv, C.D) * heads * size),
             [0] * B, lens)
    return m


def check(got, want, bound, what, norm=True):
    """Every value within its own bound, and, where the values are many, the error's norm within
    half a bf16 step (the output's rounding) and half as much for the rest, which is random:
    the score's roundings move an output by about one fp16 step of its size, 2^-10."""
    got = got.double().cpu().numpy()
    err = np.abs(got - want)
    assert np.isfinite(got).all(), what
    assert (err <= bound).all(), (what, float(np.max(err / np.maximum(bound, 1e-300))))
    rel = float(np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-300))
    say("%s: rel %.2e, %.2f of the bound" % (what, rel, float((err / np.maximum(bound, 1e-300)).max())))
    if norm:
        assert rel <= C.UBF + 2.0 ** -9, (what, rel)


# ------------------------------------------------------------------ append, read
def same_pools(cache, want, what):
    """Bytes (NaN with either sign), scales and means equal to the model's pools."""
    def bytes_(t, w):
        t = t.cpu().numpy()
        nan = (t & 127) == 127
        assert (nan == ((w & 127) == 127)).all(), what
        # a zero of either sign is zero
        zero = (t & 127) == 0
        assert ((t == w) | nan | (zero & ((w & 127) == 0))).all(), what
    bytes_(cache.k, want[0])
    bytes_(cache.v, want[1])
    for t, w in zip((cache.k_scale, cache.v_scale, cache.k_mean), want[2:]):
        np.testing.assert_array_equal(t.double().cpu().numpy(), w, err_msg=what)


APPENDS = [  # Hkv, blocks, starts, n, n_new
    (1, 1, [0], 1, None),
    (2, 3, [0, 0, 0], 64, None),
    (1, 3, [63, 64, 65, 1, 0, 127], 1, None),
    (3, 4, [0, 1, 63, 64, 100], 129, None),
    (8, 3, [17, 0, 130], 50, [50, 0, 13]),
    (2, 3, [5, 40, 100, 190], 70, [-3, 99, 1, 70]),  # counts clamped; rows past the capacity
    (1, 2, [-5, 128, 2 ** 31 - 1, -2 ** 31, -70], 20, None),  # partly and wholly outside
    (5, 9, [3, 300], 200, None),
]


@pytest.mark.parametrize("case", range(len(APPENDS)))
@pytest.mark.parametrize("per", [0, 1, 2])  # blocks of a page, 0: dense
def test_append_equals_the_model(case, per):
    Hkv, nb, starts, n, n_new = APPENDS[case]
    B = len(starts)
    rng = np.random.default_rng(100 * case + per)
    table = None
    if per:
        nb = -(-nb // per) * per
        table, n_pages = paged(B, nb // per, 2, case)
    m = filled(rng, B, nb, Hkv, [min(max(s, 0), nb * 64) for s in starts])
    before = C.pools(m, table, *((n_pages, per) if per else ()), fill=0x55 if per else 0)
    cache = upload(before)
    k, v = normals(rng, B, n, Hkv, C.D, size=2.0), normals(rng, B, n, Hkv, C.D, size=0.3)
    say("append", APPENDS[case], "per", per)
    api.cache8_append(cache, dev(k), dev(v), ints(starts), block_table=ints(table) if per else None,
                      n_new=None if n_new is None else ints(n_new))
    torch.cuda.synchronize()
    m.append(k, v, starts, n_new)
    same_pools(cache, C.pools(m, table, *((n_pages, per) if per else ()), fill=0x55 if per else 0),
               "append")


def test_append_values_at_the_edges_of_the_types():
    """Zero rows, infinities, NaN, the largest and smallest bf16, ties, and a scale that grows by
    so much that the earlier rows become subnormal or zero; each block also appended row by row."""
    rng = np.random.default_rng(7)
    tiny, most = 2.0 ** -133, C.BF16_MAX
    x = normals(rng, 9, 64, 1, C.D)
    x[0] = 0
    x[1, :, :, ::3] = math.inf
    x[2, 5, 0, 7], x[2, 6, 0, 8], x[2, :, 0, 9] = math.nan, -math.inf, -0.0
    x[3] = C.to_bf16(rng.uniform(-1, 1, x[3].shape) * tiny * 4)
    x[4, :, :, 0], x[4, :, :, 1] = most, -most
    x[5] = C.to_bf16(rng.choice([1.0625, 1.1875, 448.0, 2.0 ** -7, 3 * 2.0 ** -10, 464.0, 432.0], x[5].shape))
    x[6] = C.to_bf16(x[6] * 2.0 ** (np.arange(64) / 3.0)[:, None, None])
    x[7, 40:] *= 2.0 ** 20
    x[8] = np.nan
    for step in (64, 1, 23):
        m, cache = C.Model(9, 1, 1), api.cache8_alloc(9, 64, 1)
        for s in range(0, 64, step):
            part = x[:, s:s + step]
            api.cache8_append(cache, dev(part), dev(-part), ints([s] * 9))
            m.append(part, -part, [s] * 9)
        torch.cuda.synchronize()
        same_pools(cache, C.pools(m), "step %d" % step)
        k, v = api.cache8_read(cache, 64)
        for got, w in ((k, "k"), (v, "v")):
            np.testing.assert_array_equal(got.double().cpu().numpy(), m.rows(w))


def test_append_drops_pages_outside_the_pool_and_keeps_the_others():
    rng = np.random.default_rng(8)
    m = filled(rng, 2, 4, 2, [70, 10])
    table = np.array([[3, -1, 1, 9], [0, 2 ** 31 - 1, 2, -2 ** 31]], dtype=np.int64)
    bad = {(0, 1), (0, 3), (1, 1), (1, 3)}
    cache = upload(C.pools(m, table, 5, 1, fill=0x33))
    k, v = normals(rng, 2, 180, 2, C.D), normals(rng, 2, 180, 2, C.D)
    say("append with pages outside the pool")
    api.cache8_append(cache, dev(k), dev(v), ints([70, 10]), block_table=ints(table))
    torch.cuda.synchronize()
    m.append(k, v, [70, 10], dropped=bad)
    same_pools(cache, C.pools(m, table, 5, 1, fill=0x33), "dropped pages")


@pytest.mark.parametrize("Hkv,per,start,n", [(1, 0, 0, 1), (2, 0, 63, 2), (3, 2, 5, 300),
                                             (8, 1, 64, 64), (2, 4, 100, 412)])
def test_read_gives_the_exact_rows(Hkv, per, start, n):
    rng = np.random.default_rng(n)
    B, nb = 3, 8
    m = filled(rng, B, nb, Hkv, [512, 300, 1])
    table = None
    if per:
        table, n_pages = paged(B, nb // per, 3, n)
    cache = upload(C.pools(m, table, *((n_pages, per) if per else ())))
    k, v = api.cache8_read(cache, n, start=start, block_table=ints(table) if per else None)
    for got, w in ((k, "k"), (v, "v")):
        assert got.shape == (B, n, Hkv, C.D)
        np.testing.assert_array_equal(got.double().cpu().numpy(), m.rows(w)[:, start:start + n])


# ------------------------------------------------------------------ decode
LENS = [0, 1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 500, 1000, 1023, 1024]


@pytest.mark.parametrize("g,Hkv,per", [(1, 1, 0), (4, 2, 2), (8, 1, 1), (7, 3, 4)])
def test_decode_of_equal_scores_is_the_mean_of_the_values(g, Hkv, per):
    """K = 0: every weight is 1 / n exactly before the division, so the output is the sum of the
    values, which fp32 holds exactly, over n: one key too many or too few, at any border,
    shows.  Everything behind the lengths is NaN."""
    rng = np.random.default_rng(g)
    B, nb = len(LENS), 16
    m = C.Model(B, nb, Hkv)
    v = rng.integers(-8, 9, (B, 1024, Hkv, C.D)).astype(np.float64)
    m.append(np.zeros_like(v), v, [0] * B, LENS)
    for b, n in enumerate(LENS):  # NaN behind the last row, in its block too
        for j in range(nb):
            if j * 64 + 64 > n:
                m.k[b, j, :, max(0, n - j * 64):] = 127
                m.v[b, j, :, max(0, n - j * 64):] = 127
            if j * 64 >= n:
                m.ks[b, j] = m.vs[b, j] = math.nan
    table = None
    if per:
        table, n_pages = paged(B, nb // per, 3, g)
    cache = upload(C.pools(m, table, *((n_pages, per) if per else ())))
    q = dev(normals(rng, B, g * Hkv, C.D))
    kw = dict(block_table=ints(table) if per else None)
    for bif in (True, False):
        say("decode8 uniform g=%d Hkv=%d per=%d bifocal=%s" % (g, Hkv, per, bif))
        out = api.decode8(q, cache, ints(LENS), w_pretrained=300, w_local=70, bifocal=bif, **kw)
        got = out.double().cpu().numpy()
        for b, n in enumerate(LENS):
            want = v[b, :n].sum(0) / max(n, 1)  # [Hkv, 128]
            want = np.repeat(want, g, axis=0)
            # one rounding to bf16 of an fp32 quotient
            assert (np.abs(got[b] - want) <= np.abs(want) * C.UBF * (1 + 2.0 ** -14)).all(), (b, n)


@pytest.mark.parametrize("g,Hkv,per,w0", [(1, 2, 0, 20), (2, 3, 1, 0), (4, 8, 2, 70), (5, 1, 0, 64),
                                          (8, 2, 4, 63), (3, 1, 1, 2 ** 31 - 1)])
def test_decode_matches_the_definition(g, Hkv, per, w0):
    rng = np.random.default_rng(10 * g + Hkv)
    lens = [1, 20, 64, 97, 193, 300, 384, 640]
    B, nb, w_pre = len(lens), 12, 96
    m = filled(rng, B, nb, Hkv, lens)
    table = None
    if per:
        table, n_pages = paged(B, nb // per, 3, g)
    cache = upload(C.pools(m, table, *((n_pages, per) if per else ())))
    q = normals(rng, B, g * Hkv, C.D)
    for bif in (True, False):
        want, bound = C.decode(q, m, lens, w_pre, w0, bif)
        ws = api.decode8_workspace(g * Hkv, Hkv)
        say("decode8 g=%d Hkv=%d per=%d w0=%d bifocal=%s" % (g, Hkv, per, w0, bif))
        kw = dict(w_pretrained=w_pre, w_local=w0, bifocal=bif, workspace=ws,
                  block_table=ints(table) if per else None)
        out = api.decode8(dev(q), cache, ints(lens), **kw)
        check(out, want, bound, "decode8")
        again = api.decode8(dev(q), cache, ints(lens), **kw)
        assert torch.equal(out.view(torch.int16), again.view(torch.int16))
        assert int(ws[:4096].count_nonzero()) == 0


@pytest.mark.parametrize("B,n", [(1, 5000), (3, 2500), (150, 130), (700, 40)])
def test_decode_of_few_long_and_many_short_sequences(B, n):
    """Splits of one sequence over many workgroups, and more sequences than workgroups."""
    rng = np.random.default_rng(B)
    Hkv, g, w_pre, w0 = 2, 2, 700, 100
    lens = [max(1, n - 7 * i % n) for i in range(B)]
    nb = -(-n // 64)
    m = filled(rng, B, nb, Hkv, lens)
    q = normals(rng, B, g * Hkv, C.D)
    want, bound = C.decode(q, m, lens, w_pre, w0)
    say("decode8 B=%d n=%d" % (B, n))
    out = api.decode8(dev(q), upload(C.pools(m)), ints(lens), w_pretrained=w_pre, w_local=w0)
    check(out, want, bound, "decode8 B=%d" % B)


def test_decode_returns_the_value_of_the_one_key_that_matches():
    """A key that only matches the query under the right rotation (remote and band, G = 5), far
    above the others: the softmax is that key alone and its value row comes back."""
    rng = np.random.default_rng(3)
    n, w_pre, w0 = 1000, 220, 100
    G, qp = -(-n // w_pre), n - 1
    for key in (0, 63, 64, 500, qp - w0 - 1, qp - w0, qp):
        q = normals(rng, 1, 1, C.D)
        remote = qp - key > w0
        rel = (qp // G - key // G) if remote else qp - key
        k = C.to_bf16(0.01 * rng.standard_normal((1, n, 1, C.D)))
        k[0, key, 0] = C.to_bf16(C.rope(q[0], [rel])[0] * 8)  # R(q) x_q = R(k) x_k
        v = normals(rng, 1, n, 1, C.D)
        m = C.Model(1, 16, 1)
        m.append(k, v, [0])
        say("decode8 needle at", key)
        out = api.decode8(dev(q), upload(C.pools(m)), ints([n]), w_pretrained=w_pre, w_local=w0)
        want = m.rows("v")[0, key, 0]
        # the others' weight is below exp(-60)
        np.testing.assert_allclose(out[0, 0].double().cpu().numpy(), want, rtol=1e-6, atol=1e-20)


def test_decode_at_extreme_sizes_of_the_operands():
    """Queries beyond fp16's range, values of blocks 2^60 apart, keys whose scale is tiny."""
    rng = np.random.default_rng(4)
    n, w_pre, w0 = 300, 64, 40
    for qs, ks, vs in ((2.0 ** 100, 2.0 ** -100, 1.0), (2.0 ** -90, 2.0 ** 90, 2.0 ** 60),
                       (1.0, 2.0 ** -60, 2.0 ** -90), (2.0 ** 20, 2.0 ** -20, 2.0 ** 110)):
        m = C.Model(1, 5, 2)
        k, v = normals(rng, 1, n, 2, C.D) * ks, normals(rng, 1, n, 2, C.D) * vs
        v[:, 64:128] *= 2.0 ** -30
        m.append(k, v, [0])
        q = normals(rng, 1, 4, C.D) * qs
        want, bound = C.decode(q, m, [n], w_pre, w0)
        say("decode8 sizes", qs, ks, vs)
        out = api.decode8(dev(q), upload(C.pools(m)), ints([n]), w_pretrained=w_pre, w_local=w0)
        check(out, want, bound, "sizes")
    # one block holds all the weight and the others far larger values, times 2^-27 at most
    k, v = np.zeros((1, 128, 1, C.D)), normals(rng, 1, 128, 1, C.D)
    q = np.zeros((1, 1, C.D))
    q[..., 0] = 16.0
    k[0, :, 0, 0] = C.rope(np.eye(C.D)[:1].repeat(128, 0), np.arange(128) - 127)[:, 0] * 0
    m = C.Model(1, 2, 1)
    v[:, 64:] *= 2.0 ** 40
    m.append(C.to_bf16(k), v, [0])
    want, bound = C.decode(q, m, [128], 4096, 4096)
    out = api.decode8(dev(q), upload(C.pools(m)), ints([128]), w_pretrained=4096, w_local=4096)
    check(out, want, bound, "blocks 2^40 apart", norm=False)


def test_nan_and_infinity_reach_only_their_own_rows():
    rng = np.random.default_rng(5)
    lens = [200, 200, 200, 200]
    m = filled(rng, 4, 4, 2, lens)
    m.k[1, 1, 0, 3, 5] = 127  # a NaN key of sequence 1, head 0
    m.v[2, 2, 1, 60, 9] = 127  # a NaN value of sequence 2, head 1, channel 9
    q = normals(rng, 4, 4, C.D)
    q[3, 0, 0] = math.nan
    say("decode8 NaN")
    out = api.decode8(dev(q), upload(C.pools(m)), ints(lens), w_pretrained=64,
                      w_local=20).float().cpu().numpy()
    nan = np.isnan(out)
    want = np.zeros_like(nan)
    want[1, 0:2], want[3, 0], want[2, 2:4, 9] = True, True, True
    assert (nan == want).all()


def test_lengths_are_clamped_and_pages_stay_in_the_pool():
    rng = np.random.default_rng(6)
    m = filled(rng, 4, 2, 1, [128] * 4)
    q = normals(rng, 4, 2, C.D)
    lens = [-5, 2 ** 31 - 1, -2 ** 31, 129]
    want, bound = C.decode(q, m, [0, 128, 0, 128], 50, 10)
    say("decode8 clamped lengths")
    out = api.decode8(dev(q), upload(C.pools(m)), ints(lens), w_pretrained=50, w_local=10)
    check(out, want, bound, "clamped lengths")
    assert bool((out[0] == 0).all()) and bool((out[2] == 0).all())
    table = np.array([[-7, 2 ** 31 - 1], [1, -2 ** 31], [2, 3], [99, 0]])
    cl = np.clip(table, 0, 3)
    pages = C.Model(4, 2, 1)
    for b in range(4):
        for j in range(2):
            for x in ("k", "v", "ks", "vs", "mean"):
                getattr(pages, x)[b, j] = getattr(m, x)[cl[b, j], 0]
    one = C.Model(4, 1, 1)
    for x in ("k", "v", "ks", "vs", "mean"):
        getattr(one, x)[:] = getattr(m, x)[:, :1]
    want, bound = C.decode(q, pages, [100, 128, 65, 1], 50, 10)
    out = api.decode8(dev(q), upload(C.pools(one)), ints([100, 128, 65, 1]), w_pretrained=50,
                      w_local=10, block_table=ints(table))
    check(out, want, bound, "clamped pages")


def test_offsets_past_32_bits():
    """The last pages of pools of 4.3 GB each: byte offsets past 2^32."""
    rng = np.random.default_rng(9)
    n_pages, B = 526000, 2
    table = np.array([[n_pages - 1, 5], [n_pages - 2, n_pages - 3]])
    cache = api.cache8_alloc(n_pages, 64, 1)
    k, v = normals(rng, B, 128, 1, C.D), normals(rng, B, 128, 1, C.D)
    say("pools past 2^32 bytes")
    api.cache8_append(cache, dev(k), dev(v), ints([0, 0]), block_table=ints(table))
    m = C.Model(B, 2, 1)
    m.append(k, v, [0, 0])
    got, _ = api.cache8_read(cache, 128, block_table=ints(table))
    np.testing.assert_array_equal(got.double().cpu().numpy(), m.rows("k"))
    q, lens = normals(rng, B, 2, C.D), [128, 100]
    want, bound = C.decode(q, m, lens, 50, 20)
    kw = dict(w_pretrained=50, block_table=ints(table))
    out = api.decode8(dev(q), cache, ints(lens), w_local=20, **kw)
    check(out, want, bound, "decode past 2^32")
    s = api.block_scores8(dev(q), cache, ints(lens), **kw)
    w, tol = scores_of(q, m, lens, 50, True)
    assert (np.abs(s.double().cpu().numpy() - w) <= tol).all()
    assert int(cache.k[6:n_pages - 3].count_nonzero()) == 0


# ------------------------------------------------------------------ blocks
def scores_of(q, m, lens, w_pre, bifocal):
    """(scores, bound): fp32 rotations of query and mean (cos/sin to half a step each) and 128
    fp32 sums: 140 half-steps of the products' magnitudes at most."""
    B, Hq, _ = q.shape
    g = Hq // m.Hkv
    s = np.full((B, m.Hkv, m.nb), -math.inf)
    tol = np.zeros_like(s)
    for b in range(B):
        n = min(max(int(lens[b]), 0), m.nb * 64)
        G = max(1, -(-n // w_pre)) if bifocal else 1
        j = np.arange(-(-n // 64))
        for h in range(m.Hkv):
            mean = m.mean[b, :len(j), h]
            k = C.rope(mean, (64 * j + 31) // G)
            x = np.stack([k @ C.rope(q[b, h * g + i][None], [(n - 1) // G])[0] for i in range(g)])
            s[b, h, :len(j)] = x.max(0) / math.sqrt(C.D) if len(j) else 0
            mag = (np.abs(mean[:, :64]) + np.abs(mean[:, 64:])) @ np.abs(
                q[b, h * g:(h + 1) * g, :64] + 1j * q[b, h * g:(h + 1) * g, 64:]).max(0) * 1.5
            tol[b, h, :len(j)] = 140 * 2.0 ** -24 * mag / math.sqrt(C.D)
    return s, tol


@pytest.mark.parametrize("g,Hkv,per,nb", [(1, 1, 0, 1), (4, 2, 2, 6), (8, 3, 1, 11), (7, 1, 0, 300),
                                          (2, 8, 4, 8)])
def test_block_scores(g, Hkv, per, nb):
    rng = np.random.default_rng(nb)
    lens = [0, 1, 64, 65, nb * 64, nb * 64 - 1, max(nb * 64 // 3, 1)]
    lens = [min(n, nb * 64) for n in lens]
    B = len(lens)
    m = C.Model(B, nb, Hkv)
    m.mean[:] = C.to_bf16(rng.standard_normal(m.mean.shape))
    table = None
    if per:
        nb = m.nb = -(-nb // per) * per
        full = C.Model(B, nb, Hkv)
        full.mean[:, :m.mean.shape[1]] = m.mean
        m = full
        table, n_pages = paged(B, nb // per, 3, nb)
    cache = upload(C.pools(m, table, *((n_pages, per) if per else ())))
    q = normals(rng, B, g * Hkv, C.D)
    for bif in (True, False):
        say("scores g=%d Hkv=%d per=%d nb=%d bifocal=%s" % (g, Hkv, per, nb, bif))
        out = api.block_scores8(dev(q), cache, ints(lens), w_pretrained=90, bifocal=bif,
                                block_table=ints(table) if per else None).double().cpu().numpy()
        want, tol = scores_of(q, m, lens, 90, bif)
        inf = np.isinf(want)
        assert (np.isinf(out) == inf).all() and (out[inf] < 0).all()
        assert (np.abs(out[~inf] - want[~inf]) <= tol[~inf]).all()
    q[1, 0, 3] = math.nan  # sequence 1 has one block
    out = api.block_scores8(dev(q), cache, ints(lens), w_pretrained=90,
                            block_table=ints(table) if per else None).cpu().numpy()
    assert np.isnan(out).sum() == 1 and np.isnan(out[1, 0, 0])


@pytest.mark.parametrize("nb,n_select,w0,n_first,levels", [
    (1, 1, 0, 0, 5), (1, 7, 1000, 3, 5), (10, 10, 0, 0, 2), (64, 5, 63, 1, 1), (65, 20, 200, 0, 3),
    (300, 40, 64, 2, 50), (300, 299, 0, 0, 4), (2048, 128, 4096, 1, 10 ** 9), (5000, 66, 0, 1, 7),
    (257, 300, 0, 1, 3)])
def test_select_equals_a_sort(nb, n_select, w0, n_first, levels):
    """Few levels make many ties, also at the border; infinities, zeros of both signs and NaN."""
    rng = np.random.default_rng(nb + n_select)
    lens = [nb * 64, nb * 64 - 63, max(nb * 32, 1), 1, 0, 64, -1, 2 ** 31 - 1]
    B, Hkv = len(lens), 2
    s = rng.integers(-levels, levels + 1, (B, Hkv, nb)).astype(np.float32)
    s[0, 0, ::5] = -0.0
    s[1, 0, ::7], s[1, 1, ::3] = np.nan, -np.inf
    s[2, 0, ::6] = np.inf
    s[2, 1] = -np.inf
    s[0, 1, 1::4] = -np.nan
    say("select nb=%d n_select=%d w0=%d n_first=%d" % (nb, n_select, w0, n_first))
    got = api.select_blocks(torch.from_numpy(s).cuda(), ints(lens), n_select, w_local=w0,
                            n_first=n_first)
    np.testing.assert_array_equal(got.cpu().numpy(), C.select(s, lens, n_select, w0, n_first))


@pytest.mark.parametrize("nb", [2047, 2049, 3000, 4096, 4097, 8192, 8193, 16385, 20003])
def test_select_of_rows_of_every_length(nb):
    """Rows that start at any address, with many equal scores; shorter sequences beside long ones."""
    rng = np.random.default_rng(nb)
    lens = [nb * 64, nb * 64 - 1, nb * 37 + 5, 64 * 300]
    s = np.round(rng.standard_normal((4, 2, nb)) * 30).astype(np.float32)
    say("select nb=%d" % nb)
    for n, w0 in ((129, 4096), (nb // 2, 0)):
        got = api.select_blocks(torch.from_numpy(s).cuda(), ints(lens), n, w_local=w0)
        np.testing.assert_array_equal(got.cpu().numpy(), C.select(s, lens, n, w0, 1))


def test_select_of_the_longest_row():
    rng = np.random.default_rng(1)
    nb, n = 131072, 700
    s = np.round(rng.standard_normal((1, 2, nb)) * 500).astype(np.float32)
    got = api.select_blocks(torch.from_numpy(s).cuda(), ints([nb * 64 - 5]), n, w_local=4096)
    np.testing.assert_array_equal(got.cpu().numpy(), C.select(s, [nb * 64 - 5], n, 4096, 1))


@pytest.mark.parametrize("g,Hkv,per", [(1, 1, 0), (4, 2, 2), (8, 3, 1), (5, 2, 4)])
def test_decode_over_listed_blocks(g, Hkv, per):
    """Lists in any order, with entries outside the sequence, one block twice, no entry at all."""
    rng = np.random.default_rng(20 + g)
    lens = [1, 64, 100, 400, 640, 768, 300, 0]
    B, nb, w_pre, w0, n = len(lens), 12, 96, 70, 9
    m = filled(rng, B, nb, Hkv, lens)
    table = None
    if per:
        table, n_pages = paged(B, nb // per, 3, g)
    cache = upload(C.pools(m, table, *((n_pages, per) if per else ())))
    q = normals(rng, B, g * Hkv, C.D)
    blocks = rng.integers(-2, nb + 3, (B, Hkv, n)).astype(np.int32)
    blocks[3, 0] = [2, 2, 0, 5, 0, -1, 2 ** 31 - 1, -2 ** 31, 1]
    blocks[4, :] = -1
    blocks[5, 0, 1:] = 100
    for bif in (True, False):
        want, bound = C.decode(q, m, lens, w_pre, w0, bif, blocks)
        say("decode8_blocks g=%d Hkv=%d per=%d bifocal=%s" % (g, Hkv, per, bif))
        out = api.decode8_blocks(dev(q), cache, ints(lens), ints(blocks), w_pretrained=w_pre,
                                 w_local=w0, bifocal=bif, block_table=ints(table) if per else None)
        check(out, want, bound, "decode8_blocks")
        assert bool((out[4] == 0).all()) and bool((out[7] == 0).all())


@pytest.mark.parametrize("fill", [math.nan, math.inf])
def test_entries_that_name_no_block_take_nothing_from_the_pools(fill):
    """The pools' first page belongs to no sequence and holds no numbers: the same bits as over
    pools in which it holds zeros."""
    rng = np.random.default_rng(31)
    lens = [600, 130, 64, 0]
    m = filled(rng, 4, 10, 2, lens)
    table = np.arange(1, 41, dtype=np.int32).reshape(4, 10)
    pools = C.pools(m, table, 41, 1)
    q, blocks = normals(rng, 4, 8, C.D), rng.integers(-2, 12, (4, 2, 40)).astype(np.int32)
    blocks[0, 0, 1:], blocks[1, 1] = -1, -1
    outs = []
    for x in (0.0, fill):
        for a in pools[2:]:
            a[0] = x
        pools[0][0], pools[1][0] = (127, 127) if x else (0, 0)
        say("decode8_blocks beside a page of", x)
        outs.append(api.decode8_blocks(dev(q), upload(pools), ints(lens), ints(blocks),
                                       w_pretrained=64, w_local=20, block_table=ints(table)))
    assert torch.equal(outs[0], outs[1])
    want, bound = C.decode(q, m, lens, 64, 20, True, blocks)
    check(outs[1], want, bound, "beside a page without numbers")


@pytest.mark.parametrize("B,n_select", [(1, 120), (2, 1000), (90, 3)])
def test_decode_over_long_lists_and_many_sequences(B, n_select):
    rng = np.random.default_rng(B)
    nb, Hkv, g = 130, 2, 2
    lens = [nb * 64 - 13 * i for i in range(B)]
    if B > 2:
        nb, lens = 4, [256 - 2 * i for i in range(B)]
    m = filled(rng, B, nb, Hkv, lens)
    q = normals(rng, B, g * Hkv, C.D)
    blocks = rng.integers(0, nb, (B, Hkv, n_select)).astype(np.int32)
    want, bound = C.decode(q, m, lens, 2000, 300, True, blocks)
    out = api.decode8_blocks(dev(q), upload(C.pools(m)), ints(lens), ints(blocks),
                             w_pretrained=2000, w_local=300)
    check(out, want, bound, "long lists")


def _ones(rng_seed, n_pages, page, Hkv):
    """A dense cache whose keys are zero and whose values are drawn from -1, 0, 1, 2, straight as
    images (random bytes), with unit scales."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rng_seed)
    cache = api.cache8_alloc(n_pages, page, Hkv)
    number = torch.tensor([0xB8, 0, 0x38, 0x40], dtype=torch.uint8, device="cuda")
    for h in range(Hkv):
        for p in range(n_pages):
            pick = torch.randint(0, 4, (page, 128), generator=g, device="cuda", dtype=torch.uint8)
            cache.v[p, h] = number[pick.int()]
    cache.k_scale.fill_(1)
    cache.v_scale.fill_(1)
    return cache


@pytest.mark.parametrize("B,Hkv,n", [(1, 8, 1100000), (2, 1, 4194304), (1, 70, 1000)])
def test_decode_of_millions_of_keys(B, Hkv, n):
    """More steps than a wave looks up at once, in one sequence and in a batch, and one sequence of
    more kv heads than share its workgroups: equal scores, so the output is the values' mean,
    whose sum fp32 holds exactly."""
    page = -(-n // 64) * 64
    cache = _ones(n, B, page, Hkv)
    lens = [n - 70 * b for b in range(B)]
    q = dev(normals(np.random.default_rng(n), B, 2 * Hkv, C.D))
    say("decode8 of %d keys, B=%d Hkv=%d" % (n, B, Hkv))
    out = api.decode8(q, cache, ints(lens), w_pretrained=40000, w_local=5000).double()
    for b in range(B):
        total = torch.zeros((Hkv, C.D), dtype=torch.float64, device="cuda")
        for s in range(0, lens[b], 1 << 18):
            m = min(1 << 18, lens[b] - s)
            _, v = api.cache8_read(cache, m, start=s, B=B)
            total += v[b].double().sum(0)
        want = (total / lens[b]).repeat_interleave(2, 0)
        # the sums exact, one fp32 quotient rounded to bf16
        assert bool(((out[b] - want).abs() <= want.abs() * C.UBF * (1 + 2.0 ** -14)).all())


@pytest.mark.parametrize("lens,Hkv,g", [([70000], 1, 8), ([40001], 2, 7), ([66000], 1, 1),
                                        ([60000, 100, 45000], 1, 8), ([9000, 0, 30000, 64], 2, 5),
                                        ([33000, 20000], 1, 2)])
def test_decode_of_sequences_shared_by_many_workgroups(lens, Hkv, g):
    """Few kv heads and many keys: the states of a head pass through groups of workgroups.  The
    same call gives the same bits, and the arrival counters are zero behind it."""
    rng = np.random.default_rng(len(lens) + g)
    B, nb = len(lens), -(-max(lens) // 64)
    m = filled(rng, B, nb, Hkv, lens)
    cache, q = upload(C.pools(m)), normals(rng, B, g * Hkv, C.D)
    ws = api.decode8_workspace(g * Hkv, Hkv)
    lists = np.tile(np.arange(nb, dtype=np.int32), (B, Hkv, 1))
    lists[:, :, ::9] = -1
    kw = dict(w_pretrained=16384, w_local=1000, workspace=ws)
    for blocks in (None, lists):
        say("decode8", lens, "Hkv=%d g=%d listed=%s" % (Hkv, g, blocks is not None))
        want, bound = C.decode(q, m, lens, 16384, 1000, True, blocks)
        outs = [api.decode8(dev(q), cache, ints(lens), **kw) if blocks is None else
                api.decode8_blocks(dev(q), cache, ints(lens), ints(blocks), **kw) for _ in range(3)]
        check(outs[0], want, bound, "many workgroups")
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        assert bool((ws[:4096] == 0).all())


@pytest.mark.parametrize("B,n_select", [(128, 270), (200, 9), (300, 2)])
def test_decode_over_more_lists_than_workgroups(B, n_select):
    """Lists that a workgroup has for itself, of more entries than a wave looks up at once, and
    more lists than workgroups."""
    Hkv, nb = 4, 6
    cache = _ones(B, B, nb * 64, Hkv)
    rng = np.random.default_rng(B)
    blocks = rng.integers(-1, nb + 1, (B, Hkv, n_select)).astype(np.int32)
    lens = rng.integers(0, nb * 64 + 1, B)
    q = dev(normals(rng, B, 2 * Hkv, C.D))
    say("decode8_blocks B=%d n_select=%d" % (B, n_select))
    out = api.decode8_blocks(q, cache, ints(lens), ints(blocks), w_pretrained=100, w_local=50)
    _, v = api.cache8_read(cache, nb * 64)
    v, got = v.double().cpu().numpy(), out.double().cpu().numpy()
    for b in range(B):
        for h in range(Hkv):
            times = np.zeros(nb * 64)
            for j in blocks[b, h]:
                if 0 <= j < nb:
                    times[64 * j:64 * j + 64] += 1
            times[lens[b]:] = 0
            want = times @ v[b, :, h] / max(times.sum(), 1)
            for i in (2 * h, 2 * h + 1):
                assert (np.abs(got[b, i] - want) <= np.abs(want) * C.UBF * (1 + 2.0 ** -14)).all()


@pytest.mark.parametrize("B,Hkv,g,per,n_select", [(33, 4, 2, 1, 3), (43, 3, 7, 0, 20), (256, 1, 8, 2, 1),
                                                  (64, 4, 1, 0, 9), (64, 4, 4, 2, 70),
                                                  (65, 2, 5, 1, 16)])
def test_decode_over_a_list_for_every_compute_unit(B, Hkv, g, per, n_select):
    """Some 129 to 256 lists: short and long ones, with entries outside the sequences, in both
    rotations."""
    rng = np.random.default_rng(B + g)
    nb = 8
    lens = rng.integers(0, nb * 64 + 1, B)
    lens[:4] = [0, 1, 64, nb * 64]
    m = filled(rng, B, nb, Hkv, list(lens))
    table = None
    if per:
        table, n_pages = paged(B, nb // per, 1, B)
    cache = upload(C.pools(m, table, *((n_pages, per, 0x7f) if per else ())))
    q = normals(rng, B, g * Hkv, C.D)
    blocks = rng.integers(-2, nb + 2, (B, Hkv, n_select)).astype(np.int32)
    blocks[5], blocks[6, 0] = -1, 0
    for bif in (True, False):
        say("decode8_blocks of %d lists of %d, g=%d, per=%d, bifocal=%s" % (B * Hkv, n_select, g, per, bif))
        want, bound = C.decode(q, m, lens, 100, 70, bif, blocks)
        out = api.decode8_blocks(dev(q), cache, ints(lens), ints(blocks), w_pretrained=100,
                                 w_local=70, bifocal=bif, block_table=ints(table) if per else None)
        check(out, want, bound, "lists")
        assert bool((out[0] == 0).all()) and bool((out[5] == 0).all())


# ------------------------------------------------------------------ together
def _serving(Hq=8, Hkv=2, n0=300, steps=5, w_pre=128, w0=64, seed=0):
    rng = np.random.default_rng(seed)
    cap = -(-(n0 + 100 + steps) // 64) * 64
    return rng, cap, dict(w_pretrained=w_pre, w_local=w0)


def test_a_prompt_a_second_chunk_and_decode_steps():
    """As a serving program uses them: prompt appended, a second chunk prefilled over the rows
    read back, then decode steps over all keys and over chosen blocks."""
    Hq, Hkv, n0, n1, steps = 8, 2, 300, 50, 4
    rng, cap, kw = _serving(Hq, Hkv, n0, steps)
    cache = api.cache8_alloc(2, cap, Hkv)
    m = C.Model(2, cap // 64, Hkv)
    n = n0 + n1 + steps
    k, v, q = (normals(rng, 2, n, h, C.D) for h in (Hkv, Hkv, Hq))
    say("prompt")
    api.cache8_append(cache, dev(k[:, :n0]), dev(v[:, :n0]), ints([0, 0]))
    api.cache8_append(cache, dev(k[:, n0:n0 + n1]), dev(v[:, n0:n0 + n1]), ints([n0, n0]))
    m.append(k[:, :n0], v[:, :n0], [0, 0])
    m.append(k[:, n0:n0 + n1], v[:, n0:n0 + n1], [n0, n0])
    kb, vb = api.cache8_read(cache, n0 + n1)
    say("second chunk over the rows read back")
    out = api.prefill_chunk(dev(q[:, n0:n0 + n1]), kb, vb, q_start=n0, **kw)
    last = n0 + n1
    want, bound = C.decode(q[:, last - 1], m, [last, last], kw["w_pretrained"], kw["w_local"])
    err = np.abs(out[:, -1].double().cpu().numpy() - want)
    assert err.max() <= 2e-2  # the prefill's own tolerance (parity_util)
    same = api.decode8(dev(q[:, last - 1]), cache, ints([last, last]), **kw)
    check(same, want, bound, "the chunk's last row")
    ws = api.decode8_workspace(Hq, Hkv)
    for t in range(last, last + steps):
        say("step", t)
        api.cache8_append(cache, dev(k[:, t:t + 1]), dev(v[:, t:t + 1]), ints([t, t]))
        m.append(k[:, t:t + 1], v[:, t:t + 1], [t, t])
        lens = ints([t + 1, t + 1])
        qd = dev(q[:, t])
        full = api.decode8(qd, cache, lens, workspace=ws, **kw)
        want, bound = C.decode(q[:, t], m, [t + 1] * 2, kw["w_pretrained"], kw["w_local"])
        check(full, want, bound, "step %d" % t)
        scores = api.block_scores8(qd, cache, lens, w_pretrained=kw["w_pretrained"])
        blocks = api.select_blocks(scores, lens, 4, w_local=kw["w_local"])
        chosen = blocks.cpu().numpy()
        np.testing.assert_array_equal(
            chosen, C.select(scores.cpu().numpy(), [t + 1] * 2, 4, kw["w_local"], 1))
        some = api.decode8_blocks(qd, cache, lens, blocks, workspace=ws, **kw)
        want, bound = C.decode(q[:, t], m, [t + 1] * 2, kw["w_pretrained"], kw["w_local"],
                               blocks=chosen)
        check(some, want, bound, "step %d, chosen blocks" % t)
        every = api.select_blocks(scores, lens, cap // 64, w_local=kw["w_local"])
        allb = api.decode8_blocks(qd, cache, lens, every, workspace=ws, **kw)
        rel = float((allb.double() - full.double()).norm() / full.double().norm())
        assert rel <= C.UBF  # the same sums in another order, each output rounded once
    same_pools(cache, C.pools(m), "after the steps")


def test_two_captured_steps_replay_beside_eager_calls():
    """A step of append, decode, scores, choice and sparse decode captured twice, each graph with a
    workspace of its own, replayed on two streams and between eager calls: the eager bits."""
    Hq, Hkv, n0 = 8, 2, 700
    rng, cap, kw = _serving(Hq, Hkv, n0)

    def state(seed):
        r = np.random.default_rng(seed)
        cache = api.cache8_alloc(3, cap, Hkv)
        api.cache8_append(cache, dev(normals(r, 3, n0, Hkv, C.D)), dev(normals(r, 3, n0, Hkv, C.D)),
                          ints([0] * 3))
        return dict(cache=cache, ws=api.decode8_workspace(Hq, Hkv), q=dev(normals(r, 3, Hq, C.D)),
                    k=dev(normals(r, 3, 1, Hkv, C.D)), v=dev(normals(r, 3, 1, Hkv, C.D)),
                    at=ints([n0, 100, 639]), lens=ints([n0 + 1, 101, 640]))

    def step(s, ws=None):
        api.cache8_append(s["cache"], s["k"], s["v"], s["at"])
        ws = s["ws"] if ws is None else ws
        full = api.decode8(s["q"], s["cache"], s["lens"], workspace=ws, **kw)
        sc = api.block_scores8(s["q"], s["cache"], s["lens"], w_pretrained=kw["w_pretrained"])
        bl = api.select_blocks(sc, s["lens"], 5, w_local=kw["w_local"])
        return full, sc, bl, api.decode8_blocks(s["q"], s["cache"], s["lens"], bl, workspace=ws,
                                                **kw)

    states = [state(1), state(2)]
    eager = [[x.clone() for x in step(s)] for s in states]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(s))
        graphs.append(g)
    extra = api.decode8_workspace(Hq, Hkv)
    for turn in range(4):
        say("replay", turn)
        for o in outs:
            for x in o:
                x.fill_(0)
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for o, e in zip(outs, eager):
            for x, y in zip(o, e):
                assert torch.equal(x, y)
        again = step(states[turn % 2], ws=extra)
        for x, y in zip(again, eager[turn % 2]):
            assert torch.equal(x, y)


def test_calls_on_a_given_stream():
    rng = np.random.default_rng(2)
    lens = [500, 64]
    m = filled(rng, 2, 8, 2, lens)
    cache, q = upload(C.pools(m)), normals(rng, 2, 8, C.D)
    qd, ld = dev(q), ints(lens)
    kw = dict(w_pretrained=100, w_local=30)
    want, bound = C.decode(q, m, lens, 100, 30)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    for _ in range(3):
        out = api.decode8(qd, cache, ld, stream=st, **kw)
        sc = api.block_scores8(qd, cache, ld, w_pretrained=100, stream=st)
        bl = api.select_blocks(sc, ld, 3, w_local=30, stream=st)
        st.synchronize()
        check(out, want, bound, "stream")
        np.testing.assert_array_equal(bl.cpu().numpy(),
                                      C.select(sc.cpu().numpy(), lens, 3, 30, 1))


def test_calls_on_two_streams_at_once():
    """Each stream has a workspace of its own; every call gives the bits of the call alone."""
    rng = np.random.default_rng(12)
    lens = [3000, 64, 1, 2500, 700]
    m = filled(rng, 5, 48, 2, lens)
    cache, qd, ld = upload(C.pools(m)), dev(normals(rng, 5, 8, C.D)), ints(lens)
    one = upload(C.pools(filled(rng, 1, 48, 2, [3000])))
    lists = ints(np.tile(np.arange(48, dtype=np.int32), (5, 2, 1)))
    kw = dict(w_pretrained=500, w_local=100)

    def calls(ws, st=None):
        return [api.decode8(qd, cache, ld, workspace=ws, stream=st, **kw),
                api.decode8_blocks(qd, cache, ld, lists, workspace=ws, stream=st, **kw),
                api.decode8(qd[:1], one, ld[:1], workspace=ws, stream=st, **kw),
                api.block_scores8(qd, cache, ld, w_pretrained=500, stream=st)]

    alone = calls(api.decode8_workspace(8, 2))
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [api.decode8_workspace(8, 2) for _ in streams]
    torch.cuda.synchronize()
    say("two streams")
    got = [calls(ws, st) for _ in range(8) for ws, st in zip(spaces, streams)]
    torch.cuda.synchronize()
    for outs in got:
        for x, y in zip(outs, alone):
            assert torch.equal(x, y)
    for ws in spaces:
        assert bool((ws[:4096] == 0).all())


def test_refusals_of_the_binding():
    cache = api.cache8_alloc(2, 128, 2)
    q, lens = torch.zeros((2, 4, 128), dtype=BF, device="cuda"), ints([5, 6])
    rows = torch.zeros((2, 3, 2, 128), dtype=BF, device="cuda")
    say("binding refusals")
    for bad, err in (
            (lambda: api.decode8(q.float(), cache, lens), TypeError),
            (lambda: api.decode8(q.cpu(), cache, lens), TypeError),
            (lambda: api.decode8(q[:, :3].contiguous(), cache, lens), api.JetLongError),
            (lambda: api.decode8(q[:, ::2], cache, lens), ValueError),
            (lambda: api.decode8(q, cache, lens[:1]), ValueError),
            (lambda: api.decode8(q, cache, lens.long()), TypeError),
            (lambda: api.decode8(q, cache, lens, out=torch.empty_like(q)[:1]), ValueError),
            (lambda: api.decode8(q, cache, lens, workspace=torch.zeros(64, device="cuda")),
             api.JetLongError),
            (lambda: api.decode8(q, cache.k, lens), TypeError),
            (lambda: api.decode8(torch.cat([q, q]), cache, ints([1] * 4)), ValueError),
            (lambda: api.decode8(q, cache, lens, block_table=ints([[0, 1]])), ValueError),
            (lambda: api.decode8_blocks(q, cache, lens, None), ValueError),
            (lambda: api.decode8_blocks(q, cache, lens, ints([[0], [1]])), ValueError),
            (lambda: api.decode8_blocks(q, cache, lens, torch.zeros((2, 2, 3), device="cuda")),
             TypeError),
            (lambda: api.cache8_append(cache, rows[:, :, :1], rows, lens), ValueError),
            (lambda: api.cache8_append(cache, rows, rows[:, :2].contiguous(), lens), ValueError),
            (lambda: api.cache8_append(cache, rows, rows, lens, n_new=ints([1])), ValueError),
            (lambda: api.cache8_append(cache, rows[:, :0], rows[:, :0], lens), api.JetLongError),
            (lambda: api.cache8_read(cache, 129), api.JetLongError),
            (lambda: api.cache8_read(cache, 64, start=65), api.JetLongError),
            (lambda: api.cache8_read(cache, 64, k_out=rows), ValueError),
            (lambda: api.block_scores8(q, cache, lens, out=torch.zeros((2, 2, 3), device="cuda")),
             ValueError),
            (lambda: api.select_blocks(torch.zeros((2, 2, 9), device="cuda"), lens, 2, w_local=64),
             api.JetLongError),
            (lambda: api.select_blocks(torch.zeros((2, 2, 9)), lens, 5, w_local=0), TypeError),
            (lambda: api.Cache8(cache.k, cache.v[:1], cache.k_scale, cache.v_scale, cache.k_mean),
             ValueError),
            (lambda: api.Cache8(cache.k, cache.v, cache.k_scale.double(), cache.v_scale,
                                cache.k_mean), TypeError),
            (lambda: api.cache8_alloc(2, 100, 2), ValueError)):
        with pytest.raises(err):
            bad()


def test_a_table_without_pages_is_refused():
    cache = api.cache8_alloc(2, 128, 2)
    q, lens = torch.zeros((2, 4, 128), dtype=BF, device="cuda"), ints([5, 6])
    none = torch.zeros((2, 0), dtype=torch.int32, device="cuda")
    rows = torch.zeros((2, 3, 2, 128), dtype=BF, device="cuda")
    say("empty table")
    for call in (lambda: api.decode8(q, cache, lens, block_table=none),
                 lambda: api.block_scores8(q, cache, lens, block_table=none),
                 lambda: api.cache8_append(cache, rows, rows, lens, block_table=none),
                 lambda: api.cache8_read(cache, 1, block_table=none)):
        with pytest.raises(ValueError):
            call()
