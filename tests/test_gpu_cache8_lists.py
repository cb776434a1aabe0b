"""Decode over some 129 to 511 lists of the 8-bit cache, by how long they are: a workgroup for each,
several, or equal ranges of all."""
import numpy as np
import pytest

from paper_2607_07740_amd import api
from parity_util import say
from test_gpu_cache8 import dev, ints, normals
from test_gpu_cache8_ranges import attend, block_pages, within

import cache8_util as C

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Hkv,g,n_select", [
    (34, 4, 4, 170), (34, 4, 4, 171), (40, 4, 1, 300), (34, 5, 8, 239), (43, 4, 2, 400),
    (86, 3, 3, 81), (66, 4, 4, 84), (257, 1, 8, 90), (64, 5, 5, 106), (64, 5, 5, 108),
    (96, 4, 2, 200), (100, 4, 2, 200), (73, 7, 4, 1000), (128, 4, 2, 150)])
def test_decode_over_lists_by_their_number_and_length(B, Hkv, g, n_select):
    """Lists with entries outside the sequences and with none at all, lengths from zero on, in both
    rotations; the same call gives the same bits and leaves its counters zero."""
    rng = np.random.default_rng(B + n_select)
    n_pages, nb = 60, 50
    k = normals(rng, n_pages, Hkv, C.BLOCK, C.D)
    v = normals(rng, n_pages, Hkv, C.BLOCK, C.D) * 2.0 ** rng.uniform(-3, 3, (n_pages, Hkv, 1, 1))
    cache, kd, vd, _ = block_pages(k, v, Hkv)
    table = rng.integers(0, n_pages, (B, nb))
    lens = rng.integers(0, nb * 64 + 1, B)
    lens[:4] = [0, 1, 64, nb * 64]
    lists = rng.integers(-3, nb + 3, (B, Hkv, n_select))
    lists[4], lists[5, 0], lists[6, :, 1:] = -1, 0, nb
    q = normals(rng, B, g * Hkv, C.D)
    ws = api.decode8_workspace(g * Hkv, Hkv)
    pairs = [(b, i) for b in range(7, B) for i in range(g * Hkv)]
    some = [pairs[x] for x in rng.permutation(len(pairs))[:20]] + [(b, 0) for b in range(7)]
    for bif in (True, False):
        say("decode8_blocks of %d lists of %d, g=%d, bifocal=%s" % (B * Hkv, n_select, g, bif))
        out, again = (api.decode8_blocks(dev(q), cache, ints(lens), ints(lists), w_pretrained=700,
                                         w_local=300, bifocal=bif, block_table=ints(table + 1),
                                         workspace=ws) for _ in range(2))
        assert torch.equal(out.view(torch.int16), again.view(torch.int16))
        assert int(ws[:4096].count_nonzero()) == 0
        out = out.double().cpu().numpy()
        for b, i in some:
            h = i // g
            js = lists[b, h][(lists[b, h] >= 0) & (lists[b, h] < -(-lens[b] // 64))]
            if len(js) == 0:
                assert (out[b, i] == 0).all(), (b, i)
                continue
            pos = (64 * js[:, None] + np.arange(64)).ravel()
            want, bound = attend(q[b, i], kd[table[b, js], h].reshape(-1, C.D),
                                 vd[table[b, js], h].reshape(-1, C.D), pos, lens[b], 700, 300, bif)
            within(out[b, i], want, bound, "list %d %d" % (b, i))
