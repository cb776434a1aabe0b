"""The 8-bit cache's attentions where numbers, positions or turns of a loop get large: weights,
values and queries far apart in size, positions up to 2^23, several tiles of blocks a wave."""
import math

import numpy as np
import pytest

import cache8_util as C
from paper_2607_07740_amd import api
from parity_util import say
from test_gpu_cache8 import dev, ints, normals

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
