"""The 8-bit cache's attentions where numbers, positions or turns of a loop get large: weights,
values and queries far apart in size, positions up to 2^23, several tiles of blocks a wave."""
import math
from types import SimpleNamespace

import numpy as np
import pytest

import cache8_util as C
from paper_2607_07740_amd import api
from parity_util import say
from test_gpu_cache8 import dev, ints, normals, scores_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def attend(q, k, v, pos, kv_len, w_pre, w0, bifocal=True, n_zero=0):
    """One query head over keys k, v [n, 128] at positions pos (whole blocks, in order) and n_zero
    more keys whose K and V are zero -> (o, bound).  The roundings are those of
    cache8_util.attend, but that a weight too small for fp16 errs by at most 2^-40 of the largest
    in its own block of 64: no block's values may be lost beside another's weights."""
    G = max(1, -(-kv_len // w_pre)) if bifocal else 1
    qp = kv_len - 1
    s = C.rope(k, pos) @ C.rope(q[None], [qp])[0]
    if G > 1:
        far = C.rope(k, pos // G) @ C.rope(q[None], [qp // G])[0]
        s = np.where(qp - pos > w0, far, s)
    s = np.where(pos < kv_len, s / math.sqrt(C.D), -math.inf)
    top = max(s.max(), 0.0 if n_zero else -math.inf)
    p = np.exp(s - top)
    rest = n_zero * math.exp(-top)
    total = p.sum() + rest
    p, rest = p / total, rest / total
    o = p @ v
    mag = (np.abs(k[:, :64]) + np.abs(k[:, 64:])) @ (np.abs(q[:64]) + np.abs(q[64:])) / math.sqrt(C.D)
    delta = 4.5 * C.U16 * mag.max()
    small = 2.0 ** -40 * p.reshape(-1, C.BLOCK).max(1).repeat(C.BLOCK)
    moved = p @ np.abs(v - o) + rest * np.abs(o)
    bound = moved * np.expm1(2 * delta) + (C.U16 * p + small) @ np.abs(v) + C.UBF * np.abs(o)
    return o, 1.01 * bound + 1e-37


def within(got, want, bound, what):
    err = np.abs(got - want)
    assert np.isfinite(got).all(), what
    say("%s: %.2f of the bound, rel %.1e" % (what, float((err / np.maximum(bound, 1e-300)).max()),
                                             float(np.linalg.norm(got - want) / np.linalg.norm(want))))
    assert (err <= bound).all(), what


def block_pages(k, v, Hkv):
    """A cache of one-block pages: page 0 is zero, page 1 + i holds rows k[i], v[i] [Hkv, 64, 128]
    (fp64, quantised here) -> (cache, dequantised k, v)."""
    n = len(k)
    cache = api.cache8_alloc(n + 1, C.BLOCK, Hkv)
    out = []
    for rows, pool, scale, pack in ((k, cache.k, cache.k_scale, C.pack_k),
                                    (v, cache.v, cache.v_scale, C.pack_v)):
        sc = C.scale_of(np.abs(rows).max((-2, -1)))
        y = C.e4m3(rows / sc[..., None, None])
        pool[1:] = torch.from_numpy(pack(y).reshape(n, Hkv, C.BLOCK, C.D)).cuda()
        scale[1:] = dev(sc[..., None], torch.float32)
        out.append(C.E4M3[y] * sc[..., None, None])
    mean = C.to_bf16(out[0].mean(-2))
    cache.k_mean[1:] = dev(mean[:, :, None])
    return cache, out[0], out[1], mean


# form: lists per sequence, or None for decode8 over all keys; every wave takes several steps
FORMS = [(1, 64, 600, None), (2, 64, 500, None), (2, 8, 400, 2400), (40, 4, 40, 60), (130, 4, 40, 24)]


@pytest.mark.parametrize("B,Hkv,nb,n_select", FORMS)
def test_small_weights_on_large_values(B, Hkv, nb, n_select):
    """The weights of whole blocks lie up to 2^61 below the largest, and their values as far above
    those of the others: every block counts alike, in whatever order a wave meets them."""
    rng = np.random.default_rng(B + Hkv)
    n_pages = 70
    level = rng.choice([0, 10, 22, 30], n_pages)  # e4m3 numbers
    q = np.zeros((B, Hkv, C.D))
    q[..., 63] = 16.0  # a pair that hardly turns
    k = np.zeros((n_pages, Hkv, C.BLOCK, C.D))
    k[..., 63] = level[:, None, None]
    bits = 16.0 * level / math.sqrt(C.D) / math.log(2.0)
    v = np.abs(normals(rng, n_pages, Hkv, C.BLOCK, C.D)) * 2.0 ** np.round(bits.max() - bits)[:, None, None, None]
    table = rng.integers(0, n_pages, (B, nb))
    cache, kd, vd, _ = block_pages(k, v, Hkv)
    lens = [nb * 64 - 5 * (b % 7) for b in range(B)]
    kw = dict(w_pretrained=700, w_local=500, block_table=ints(table + 1))
    say("small weights B=%d Hkv=%d n_select=%s" % (B, Hkv, n_select))
    if n_select is None:
        lists = np.tile(np.arange(nb), (B, Hkv, 1))
        out = api.decode8(dev(q), cache, ints(lens), **kw)
    else:
        lists = rng.integers(0, nb, (B, Hkv, n_select))
        out = api.decode8_blocks(dev(q), cache, ints(lens), ints(lists), **kw)
    out = out.double().cpu().numpy()
    pairs = [(b, h) for b in range(B) for h in range(Hkv)]
    for b, h in [pairs[i] for i in rng.permutation(len(pairs))[:24]]:
        at = table[b, lists[b, h]]
        pos = (64 * lists[b, h][:, None] + np.arange(64)).ravel()
        want, bound = attend(q[b, h], kd[at, h].reshape(-1, C.D), vd[at, h].reshape(-1, C.D), pos,
                             lens[b], 700, 500)
        within(out[b, h], want, bound, "sequence %d head %d" % (b, h))


@pytest.mark.parametrize("bits", [20, 26])
def test_small_channels_of_a_query_count(bits):
    """One channel of the query is 2^bits above the others, and the keys are zero there: the scores
    come from the others alone."""
    rng = np.random.default_rng(bits)
    B, Hkv, nb = 2, 2, 6
    q = normals(rng, B, Hkv, C.D)
    q[..., 5] = 2.0 ** bits
    k = normals(rng, B * nb, Hkv, C.BLOCK, C.D) * 2.0
    k[..., 5] = k[..., 69] = 0
    v = normals(rng, B * nb, Hkv, C.BLOCK, C.D)
    table = rng.permutation(B * nb).reshape(B, nb)
    cache, kd, vd, _ = block_pages(k, v, Hkv)
    lens = [nb * 64, 201]
    say("small channels", bits)
    out = api.decode8(dev(q), cache, ints(lens), w_pretrained=150, w_local=60,
                      block_table=ints(table + 1)).double().cpu().numpy()
    for b in range(B):
        for h in range(Hkv):
            at = table[b, :-(-lens[b] // 64)]
            want, bound = attend(q[b, h], kd[at, h].reshape(-1, C.D), vd[at, h].reshape(-1, C.D),
                                 np.arange(64 * len(at)), lens[b], 150, 60)
            within(out[b, h], want, bound, "sequence %d head %d" % (b, h))


# ------------------------------------------------------------------ far positions
FAR = [(8388608, 32768, 4096), (8388545, 40001, 5000), (1100003, 32768, 4096), (8388608, 1, 100),
       (8300001, 8388608, 64), (1048577, 1000, 0)]  # length, w_pretrained, w_local


def far_blocks(n, w_pre, w0):
    """Blocks of a sequence of n keys: its ends, both sides of the band's edge, some between."""
    last, edge = (n - 1) // 64, max(n - 1 - w0, 0) // 64
    js = {0, 1, last, max(last - 1, 0), edge, max(edge - 1, 0), last // 3, 2 * last // 3,
          min(last, (1 << 20) // 64)}
    return np.array(sorted(js))


def far_cache(rng, cases, Hkv):
    """Sequences whose tables name one of 12 pages for each of their far_blocks, and page 0, of
    zeros, for every other block -> (blocks and pages of each sequence, table, cache, k, v, mean)."""
    table = np.zeros((len(cases), 131072), dtype=np.int32)
    found = []
    for b, c in enumerate(cases):
        js = far_blocks(*c)
        at = rng.permutation(12)[:len(js)]
        table[b, js] = 1 + at
        found.append((js, at))
    k, v = (normals(rng, 12, Hkv, C.BLOCK, C.D) for _ in range(2))
    return (found, ints(table)) + block_pages(k, v, Hkv)


@pytest.mark.parametrize("n,w_pre,w0", FAR)
@pytest.mark.parametrize("B,Hkv,listed", [(1, 1, False), (1, 65, False), (3, 2, False), (2, 3, True),
                                          (66, 2, True), (257, 2, True)])
def test_decode_at_far_positions(B, Hkv, listed, n, w_pre, w0):
    """Positions up to 2^23, groups of 1 to 2^23: the keys of a few far blocks, beside millions of
    zero ones where all are read, against the definition.  Scores differ by several units there,
    so a view or a rotation that is off by one shows."""
    rng = np.random.default_rng(B + Hkv)
    size = 1.0 if listed else 5.0  # of a query: beside millions of zero keys the others must count
    mine, g = [(n - 64001 * i, w_pre, w0) for i in range(min(B, 16))], 2
    mine = (mine * B)[:B]
    found, table, cache, kd, vd, _ = far_cache(rng, mine, Hkv)
    q = normals(rng, B, g * Hkv, C.D, size=size)
    lens = [c[0] for c in mine]
    lists = np.full((B, Hkv, max(len(js) for js, _ in found)), -1, dtype=np.int32)
    for b, (js, _) in enumerate(found):
        lists[b, :, :len(js)] = js
    for bif in (True, False):
        kw = dict(w_pretrained=w_pre, w_local=w0, bifocal=bif, block_table=table)
        say("far decode8 n=%d w_pre=%d B=%d Hkv=%d listed=%s" % (n, w_pre, B, Hkv, listed))
        out = (api.decode8_blocks(dev(q), cache, ints(lens), ints(lists), **kw) if listed else
               api.decode8(dev(q), cache, ints(lens), **kw)).double().cpu().numpy()
        some = [(b, i) for b in range(B) for i in range(g * Hkv)]
        for b, i in [some[x] for x in rng.permutation(len(some))[:16]]:
            js, at = found[b]
            pos = (64 * js[:, None] + np.arange(64)).ravel()
            zero = 0 if listed else lens[b] - int((pos < lens[b]).sum())
            want, bound = attend(q[b, i], kd[at, i // g].reshape(-1, C.D),
                                 vd[at, i // g].reshape(-1, C.D), pos, lens[b], w_pre, w0, bif, zero)
            within(out[b, i], want, bound, "sequence %d head %d" % (b, i))


def needles(n, w0):
    """Positions of a key: the ends, borders of blocks far out, both sides of the band's edge."""
    mid = n // 64 // 2 * 64
    return [0, 63, 64, mid, mid + 63, max(n - 2 - w0, 0), max(n - 1 - w0, 0), n - 1]


def needle(rng, n, key, w_pre, w0, bifocal, n_keys):
    """(q, k): a query of the fastest pair alone, and the key that meets it at position `key` under
    the right rotation.  Its score is 6 above the logarithm of the keys whose score is zero: off by
    one position, cos(1) = 0.54 of the score is left, and the others count as much or more."""
    G = max(1, -(-n // w_pre)) if bifocal else 1
    rel = (n - 1) // G - key // G if n - 1 - key > w0 and G > 1 else n - 1 - key
    q = np.zeros(C.D)
    turn = rng.uniform(0, 2 * math.pi)
    q[0], q[64] = C.to_bf16(4 * math.cos(turn)), C.to_bf16(4 * math.sin(turn))
    k = C.rope(q[None], [rel])[0]  # R(q) x_q = R(k) x_k
    return q, C.to_bf16(k * (math.log(n_keys) + 6) * math.sqrt(C.D) / (k @ k))


@pytest.mark.parametrize("n,w_pre,w0", FAR)
@pytest.mark.parametrize("B,Hkv,listed", [(1, 1, False), (8, 2, False), (8, 1, True), (72, 2, True),
                                          (264, 2, True)])
def test_decode_finds_the_one_key_at_a_far_position(B, Hkv, listed, n, w_pre, w0):
    """A wrong view, or a rotation that is off by one position, loses the key's value."""
    rng = np.random.default_rng(B)
    for bif in (True, False):
        for turn in range(8 if B == 1 else 1):
            lens = [n - 1 - 7 * (b // 8) for b in range(B)]
            keys = [needles(lens[b], w0)[(b + turn) % 8] for b in range(B)]
            table = np.zeros((B, 131072), dtype=np.int32)
            q = np.zeros((B, Hkv, C.D))
            k, v = np.zeros((B, Hkv, C.BLOCK, C.D)), normals(rng, B, Hkv, C.BLOCK, C.D)
            lists = np.full((B, Hkv, 9), 2, dtype=np.int32)  # 9 blocks, with the key's among them
            for b in range(B):
                table[b, keys[b] // 64] = 1 + b
                lists[b] += np.arange(9) * 5
                if keys[b] // 64 not in lists[b, 0]:
                    lists[b, :, b % 9] = keys[b] // 64
                for h in range(Hkv):
                    q[b, h], k[b, h, keys[b] % 64] = needle(rng, lens[b], keys[b], w_pre, w0, bif,
                                                            9 * 64 if listed else lens[b])
            cache, kd, vd, _ = block_pages(k, v, Hkv)
            say("far needle n=%d w_pre=%d B=%d Hkv=%d listed=%s at %s" % (n, w_pre, B, Hkv, listed,
                                                                          keys[:8]))
            kw = dict(w_pretrained=w_pre, w_local=w0, bifocal=bif, block_table=ints(table))
            out = (api.decode8_blocks(dev(q), cache, ints(lens), ints(lists), **kw) if listed else
                   api.decode8(dev(q), cache, ints(lens), **kw)).double().cpu().numpy()
            for b in rng.permutation(B)[:16]:
                pos = keys[b] // 64 * 64 + np.arange(64)
                live = int((pos < lens[b]).sum())
                for h in range(Hkv):
                    # of a list's blocks only the key's own may hold the end of the sequence
                    want, bound = attend(q[b, h], kd[b, h], vd[b, h], pos, lens[b], w_pre, w0, bif,
                                         8 * 64 if listed else lens[b] - live)
                    within(out[b, h], want, bound, "sequence %d key %d" % (b, keys[b]))


@pytest.mark.parametrize("n,w_pre,w0", FAR)
def test_block_scores_at_far_positions(n, w_pre, w0):
    rng = np.random.default_rng(n)
    mine, Hkv, g = [(n, w_pre, w0), (n - 64001, w_pre, w0)], 2, 3
    found, table, cache, _, _, mean = far_cache(rng, mine, Hkv)
    q, lens = normals(rng, 2, g * Hkv, C.D), [c[0] for c in mine]
    for bif in (True, False):
        say("far scores", mine, bif)
        out = api.block_scores8(dev(q), cache, ints(lens), w_pretrained=w_pre, bifocal=bif,
                                block_table=table).double().cpu().numpy()
        for b, (js, at) in enumerate(found):
            nb = -(-lens[b] // 64)
            assert np.isneginf(out[b, :, nb:]).all()
            assert (np.delete(out[b, :, :nb], js, 1) == 0).all()
            G = max(1, -(-lens[b] // w_pre)) if bif else 1
            for h in range(Hkv):
                m, qs = mean[at, h], q[b, h * g:(h + 1) * g]
                k = C.rope(m, (64 * js + 31) // G)
                x = np.stack([k @ C.rope(a[None], [(lens[b] - 1) // G])[0] for a in qs]).max(0)
                # as scores_of: 140 half-steps of fp32 of the products' magnitudes
                mag = ((np.abs(m[:, :64]) + np.abs(m[:, 64:])) @
                       (np.abs(qs[:, :64]) + np.abs(qs[:, 64:])).max(0))
                tol = 140 * 2.0 ** -24 * mag / math.sqrt(C.D)
                assert (np.abs(out[b, h, js] - x / math.sqrt(C.D)) <= tol).all()


# ------------------------------------------------------------------ several turns
@pytest.mark.parametrize("g,Hkv,per,nb,B", [(4, 8, 0, 260, 64), (8, 8, 1, 260, 64), (1, 5, 2, 130, 128),
                                            (5, 1, 0, 77, 300)])
def test_block_scores_of_several_tiles_a_wave(g, Hkv, per, nb, B):
    """More tiles of 16 blocks than a wave takes at once: a workgroup goes through its loop three
    times and more, and its sequences end after different numbers of turns."""
    rng = np.random.default_rng(nb + B)
    lens = [int(x) for x in rng.integers(0, nb * 64 + 1, B)]
    lens[:6] = [0, nb * 64, 1, 16 * 64, 16 * 64 + 1, nb * 64 - 63]
    mean = normals(rng, B, nb, Hkv, C.D)
    if per:
        table = rng.permutation(B * (nb // per) + 3)[:B * (nb // per)].reshape(B, -1)
        cache = api.cache8_alloc(B * (nb // per) + 3, 64 * per, Hkv)
        cache.k_mean.fill_(math.nan)
        cache.k_mean[torch.from_numpy(table).cuda()] = dev(
            mean.reshape(B, nb // per, per, Hkv, C.D).transpose(0, 1, 3, 2, 4))
    else:
        table, cache = None, api.cache8_alloc(B, 64 * nb, Hkv)
        cache.k_mean.copy_(dev(mean.transpose(0, 2, 1, 3)))
    q = normals(rng, B, g * Hkv, C.D)
    for bif in (True, False):
        say("scores g=%d Hkv=%d per=%d nb=%d B=%d bifocal=%s" % (g, Hkv, per, nb, B, bif))
        out = api.block_scores8(dev(q), cache, ints(lens), w_pretrained=3000, bifocal=bif,
                                block_table=None if table is None else ints(table))
        out = out.double().cpu().numpy()
        want, tol = scores_of(q, SimpleNamespace(mean=mean, nb=nb, Hkv=Hkv), lens, 3000, bif)
        inf = np.isinf(want)
        assert (np.isinf(out) == inf).all() and (out[inf] < 0).all()
        assert (np.abs(out[~inf] - want[~inf]) <= tol[~inf]).all()
