"""Packed chunks behind paged caches against the fp64 oracle's prefill of each whole sequence.

Tolerances: the parity bounds of the prefill tests, whose roundings these are (rotated queries and
keys, cos and sin of the keys, softmax weights in bf16 at worst, u = 2^-8): scores of unit normals are off
by 0.007 rms at most, which moves an output, a weighted mean of values of size 1, by less than
0.004 rms; with its own rounding 2e-2 at most and 2e-3 in the mean.  The row sums carry the scores' errors averaged
over the weights: 2e-2."""
import numpy as np
import pytest

from oracle import oracle as O
from paper_2607_07740_amd import api, synth
from parity_util import assert_close, say, to_dev, to_f64

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NAN = np.uint16(0x7FC0)


def _i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


class Chunks:
    """Sequences of `lens` keys on shuffled pages, the last n[b] positions of each in the call; rows
    and pages that none has hold NaN."""

    def __init__(self, lens, n, Hq, Hkv, page, seed, spare=1):
        rng = np.random.default_rng(seed)
        self.lens, self.n, self.Hq, self.Hkv, self.page = list(lens), list(n), Hq, Hkv, page
        self.max_pages = -(-max(max(lens), 1) // page) + spare
        n_pages = sum(-(-x // page) for x in lens) + 2
        deal = iter(rng.permutation(n_pages))
        self.kp = np.full((n_pages, page, Hkv, 128), NAN, np.uint16)
        self.vp = np.full_like(self.kp, NAN)
        self.table = np.full((len(lens), self.max_pages), -1, np.int32)
        self.seqs, rows = [], []
        for b, L in enumerate(lens):
            q, k, v = synth.prefill_inputs(1, Hq, Hkv, max(L, 1), 128, seed=seed + 1 + b,
                                           outlier_channels=8)
            self.seqs.append((q, k, v))
            rows.append(q[0, L - n[b]:L] if n[b] <= L else
                        np.concatenate([np.full((n[b] - L, Hq, 128), NAN, np.uint16), q[0, :L]]))
            for j in range(-(-L // page)):
                p = next(deal)
                self.table[b, j] = p
                part = slice(j * page, min((j + 1) * page, L))
                m = part.stop - part.start
                self.kp[p, :m], self.vp[p, :m] = k[0, part], v[0, part]
        self.q = np.concatenate(rows)
        self.cu = np.concatenate([[0], np.cumsum(n)])

    def run(self, w_pre=1, w0=0, bifocal=True, **kw):
        r = api.prefill_varlen_paged(to_dev(self.q), to_dev(self.kp), to_dev(self.vp),
                                     _i32(self.table), _i32(self.cu), _i32(self.lens),
                                     w_pretrained=w_pre, w_local=w0, bifocal=bifocal, **kw)
        torch.cuda.synchronize()
        return r

    def want(self, w_pre=1, w0=0, bifocal=True):
        outs, lses = [], []
        for (q, k, v), L, n in zip(self.seqs, self.lens, self.n):
            if L == 0 or n == 0:
                continue
            o, lse = O.prefill(q, k, v, theta=1e6, w_pretrained=w_pre if bifocal else 1 << 30,
                               w_local=w0)[:2]
            m = min(n, L)
            outs.append(o[0, L - m:])
            lses.append(lse[0, :, L - m:])
        return np.concatenate(outs), np.concatenate(lses, 1)


# lens, rows: single tokens, whole prompts, blocks of one and of several, lengths beside tile and
# page ends, sequences without rows or without keys
SHAPES = [([1], [1]), ([5, 64, 65, 200], [5, 64, 1, 33]), ([300, 0, 129, 31, 700], [0, 0, 129, 30, 65]),
          ([640] * 3, [8, 1, 640]), ([97, 96, 33, 32, 17, 16], [1, 2, 3, 4, 5, 6]),
          ([500], [300])]


@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("bifocal", [True, False])
def test_matches_oracle(shape, page, bifocal):
    Hq, Hkv = [(4, 2), (8, 2), (6, 2), (16, 2), (8, 1), (32, 2)][shape]
    c = Chunks(*SHAPES[shape], Hq, Hkv, page, seed=shape + page)
    say("varlen_paged", shape, page, bifocal)
    out, lse = c.run(96, 40, bifocal, want_lse=True)
    o, l = c.want(96, 40, bifocal)
    assert_close(to_f64(out), o, what="out")
    assert_close(lse.cpu().numpy(), l, what="lse")


@pytest.mark.parametrize("w_pre,w0", [(1, 0), (50, 0), (64, 7), (300, 33), (10, 2147483647)])
def test_windows(w_pre, w0):
    c = Chunks([640, 100, 333, 64], [70, 100, 3, 1], 8, 2, 64, seed=w_pre)
    say("windows", w_pre, w0)
    assert_close(to_f64(c.run(w_pre, w0)), c.want(w_pre, w0)[0], what="w_pre %d w0 %d" % (w_pre, w0))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 1), (7, 1), (20, 2), (16, 1), (64, 1), (256, 1), (8, 8)])
def test_groups_of_heads(Hq, Hkv):
    """Any number of query heads for a kv head, up to a block's rows."""
    c = Chunks([200, 90, 40], [100, 2, 40], Hq, Hkv, 32, seed=Hq)
    say("heads", Hq, Hkv)
    assert_close(to_f64(c.run(64, 20)), c.want(64, 20)[0], what="heads %d/%d" % (Hq, Hkv))


@pytest.mark.parametrize("lens,n,w_pre,w0,page", [
    ([6000, 900, 40, 3000], [300, 1, 40, 70], 2000, 500, 64),  # blocks in parts, beside few rows
    ([5000, 4999], [260, 4], 1 << 20, 9, 128),                 # every G 1
    ([2500, 1300, 260], [65, 400, 260], 600, 0, 1024),         # a block that ends the chunk, a page of all
    ([300] * 12, [30] * 12, 100, 50, 64)])                     # no sequence has a block's rows
def test_long_chunks_in_blocks(lens, n, w_pre, w0, page):
    """Enough rows that longer chunks run as whole blocks, whose key ranges are cut."""
    c = Chunks(lens, n, 8, 2, page, seed=len(lens))
    say("blocks", lens, n)
    for bifocal in (True, False):
        out, lse = c.run(w_pre, w0, bifocal, want_lse=True)
        at = 0
        for (q, k, v), L, m in zip(c.seqs, c.lens, c.n):
            rows = np.asarray([(0, h, L - m + i) for h in range(8) for i in range(m)], np.int64)
            o, l, _ = O.prefill_rows(q, k, v, rows, theta=1e6, w_pretrained=w_pre, w_local=w0,
                                     bifocal=bifocal, want_lse=True)
            got = to_f64(out[at:at + m]).transpose(1, 0, 2).reshape(8 * m, 128)
            assert_close(got, o, what="L %d n %d" % (L, m))
            assert_close(lse[:, at:at + m].reshape(-1).cpu().numpy(), l, what="lse")
            at += m


def test_scores_far_from_the_first_reference():
    """Keys whose scores lie hundreds of log2 units apart, rising and falling: the references move."""
    for n, sign in ((3, 1), (3, -1), (150, 1), (300, -1)):
        c = Chunks([700, 64], [n, 5], 8, 2, 64, seed=n)
        for b, (q, k, v) in enumerate(c.seqs):
            big = synth.bf16_bits(np.full(q.shape, 20.0, np.float32))
            ramp = np.linspace(-sign, sign, c.lens[b], dtype=np.float32)[None, :, None, None]
            kk = synth.bf16_bits(np.broadcast_to(20 * ramp, k.shape).copy())
            c.seqs[b] = (big, kk, v)
            for j in range(-(-c.lens[b] // 64)):
                part = slice(64 * j, min(64 * j + 64, c.lens[b]))
                c.kp[c.table[b, j], :part.stop - part.start] = kk[0, part]
        c.q = np.concatenate([s[0][0, L - m:] for s, L, m in zip(c.seqs, c.lens, c.n)])
        say("far scores", n, sign)
        # a weight of size 1 over scores of this size keeps no better than their own rounding, 2^-8
        # of about 2000: the mean over few keys, values of size 1
        out = c.run(256, 90)
        assert torch.isfinite(out.float()).all()
        want = c.want(256, 90)[0]
        assert np.abs(to_f64(out) - want).mean() < 1.0


def test_agrees_with_the_chunk_of_one_start_and_repeats_its_bits():
    c = Chunks([900, 900], [130, 130], 8, 2, 64, seed=3)
    say("one start")
    one, two = c.run(256, 100), c.run(256, 100)
    q = to_dev(c.q).view(2, 130, 8, 128)
    ref = api.prefill_chunk_paged(q, to_dev(c.kp), to_dev(c.vp), _i32(c.table), q_start=770,
                                  w_pretrained=256, w_local=100)
    torch.cuda.synchronize()
    assert torch.equal(one, two)
    assert_close(to_f64(one), to_f64(ref.view(260, 8, 128)), what="chunk of one start")


def test_rows_of_no_sequence_and_before_the_first_position_stay():
    c = Chunks([40, 3, 70], [10, 5, 7], 4, 2, 16, seed=9)
    out = torch.full((24, 4, 128), 3.0, device="cuda").to(torch.bfloat16)
    lse = torch.full((4, 24), 5.0, device="cuda")
    q = torch.cat([to_dev(c.q), torch.full((2, 4, 128), float("nan"), device="cuda").to(torch.bfloat16)])
    say("rows that stay")
    api.prefill_varlen_paged(q, to_dev(c.kp), to_dev(c.vp), _i32(c.table), _i32(c.cu), _i32(c.lens),
                             w_pretrained=30, w_local=9, out=out, lse=lse)
    torch.cuda.synchronize()
    o, l = c.want(30, 9)
    left = [10, 11, 22, 23]  # two rows more than keys, two of no sequence
    done = [i for i in range(24) if i not in left]
    assert (out[left] == 3.0).all() and (lse[:, left] == 5.0).all()
    assert_close(to_f64(out[done]), o, what="out")
    assert_close(lse[:, done].cpu().numpy(), l, what="lse")


def test_bad_lists_do_not_leave_the_arrays():
    c = Chunks([40, 30, 70], [10, 5, 7], 4, 2, 16, seed=10)
    table = c.table.copy()
    table[0, :2] = [1 << 30, -(1 << 31)]
    for cu, lens in (([-9, 2147483647, 3, 22], [40, 30, 70]), ([22, 11, 5, 0], [2147483647, -9, 1]),
                     ([0, 0, 0, 0], [0, 0, 0]), ([5, 6, 6, 22], [2147483647] * 3)):
        say("bad lists", cu)
        api.prefill_varlen_paged(to_dev(c.q), to_dev(c.kp), to_dev(c.vp), _i32(table), _i32(cu),
                                 _i32(lens), w_pretrained=30, w_local=9)
        torch.cuda.synchronize()


def test_captured_on_a_stream_of_its_own():
    c = Chunks([500, 90], [3, 40], 8, 2, 64, seed=13)
    q, k, v, t, cu, lens = (to_dev(c.q), to_dev(c.kp), to_dev(c.vp), _i32(c.table), _i32(c.cu),
                            _i32(c.lens))
    out = torch.empty_like(q)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        api.prefill_varlen_paged(q, k, v, t, cu, lens, w_pretrained=100, w_local=30, out=out)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            api.prefill_varlen_paged(q, k, v, t, cu, lens, w_pretrained=100, w_local=30, out=out)
    want = c.want(100, 30)[0]
    for i in range(4):
        if i == 2:  # other lengths in the same arrays
            cu.copy_(_i32([0, 1, 43]))
            lens.copy_(_i32([498, 90]))
        say("replay", i)
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = api.prefill_varlen_paged(q, k, v, t, cu, lens, w_pretrained=100, w_local=30)
        torch.cuda.synchronize()
        if i < 2:
            assert_close(to_f64(out), want, what="replay %d" % i)
        rows = slice(0, 43) if i < 2 else slice(1 - 1, 43)
        assert torch.equal(out[rows], eager[rows])


def test_the_rows_of_a_forked_batch_from_prompt_to_tokens():
    """What a server does: prompts enter forked pages in packed rows, are prefilled behind what they
    share, and every sequence decodes a token over the shared prefix."""
    rng = np.random.default_rng(1)
    Hq, Hkv, page, w_pre, w0 = 8, 2, 16, 100, 30
    pages = api.pages_alloc(4, 20, 70, page)
    kp = torch.zeros((70, page, Hkv, 128), device="cuda", dtype=torch.bfloat16)
    vp = torch.zeros_like(kp)
    hist = [np.zeros((3, 0, Hq, 128), np.uint16) for _ in range(4)]

    def turn(n):
        """n[b] more tokens of every sequence; the outputs of their rows, packed."""
        x = [synth.prefill_inputs(1, Hq, Hq, max(m, 1), 128, seed=int(rng.integers(1 << 30))) for m in n]
        for b, m in enumerate(n):
            hist[b] = np.concatenate([hist[b], np.stack([t[0, :m] for t in x[b]])], 1)
        rows = [np.concatenate([t[i][0, :m] for t, m in zip(x, n)]) for i in range(3)]
        cu = _i32(np.concatenate([[0], np.cumsum(n)]))
        starts, granted, moves, info = api.pages_reserve(pages, _i32(n))
        api.copy_pages([kp, vp], moves, info)
        q, k, v = to_dev(rows[0]), to_dev(rows[1][:, :Hkv]), to_dev(rows[2][:, :Hkv])
        api.cache_append(kp, vp, k, v, starts, n_new=granted, block_table=pages.table, cu_seqlens=cu)
        return q, cu

    def want(b, m):
        q, k, v = hist[b]
        o = O.prefill(q[None], k[None, :, :Hkv], v[None, :, :Hkv], theta=1e6, w_pretrained=w_pre,
                      w_local=w0)[0]
        return o[0, -m:]

    say("server: prompt")
    q, cu = turn([140, 0, 0, 9])
    out = api.prefill_varlen_paged(q, kp, vp, pages.table, cu, pages.lens, w_pretrained=w_pre,
                                   w_local=w0)
    torch.cuda.synchronize()
    assert_close(to_f64(out), np.concatenate([want(0, 140), want(3, 9)]), what="prompt")
    say("server: forks and their turns")
    api.pages_fork(pages, _i32([0, 0, 0, 3]))
    hist[1], hist[2] = hist[0].copy(), hist[0].copy()
    q, cu = turn([5, 33, 1, 60])
    out = api.prefill_varlen_paged(q, kp, vp, pages.table, cu, pages.lens, w_pretrained=w_pre,
                                   w_local=w0)
    torch.cuda.synchronize()
    assert_close(to_f64(out), np.concatenate([want(0, 5), want(1, 33), want(2, 1), want(3, 60)]),
                 what="turns")
    for i in range(3):
        say("server: token", i)
        q, _ = turn([1, 1, 1, 1])
        plan = api.shared_plan(pages.lens, _i32([0, 3, 4]), _i32([140, 0]), Hq=Hq, Hkv=Hkv,
                               page_size=page, max_pages=20, w_pretrained=w_pre, w_local=w0)
        out = api.decode_shared(q, kp, vp, pages.table, plan)
        torch.cuda.synchronize()
        assert_close(to_f64(out), np.concatenate([want(b, 1) for b in range(4)]), what="token %d" % i)


@pytest.mark.parametrize("n", [[3, 70, 1], [30, 33, 20], [300, 260, 200]])
def test_keys_and_queries_of_any_magnitude(n):
    """Keys times 2^e, their queries times 2^-e, another e for each sequence: the same scores."""
    c = Chunks([400, 300, 260], n, 8, 2, 64, seed=51)
    want = c.want(150, 60)[0]
    on = lambda x: ((x & 0x7F80) != 0) & ((x & 0x7F80) != 0x7F80)  # noqa: E731
    times = lambda x, e: np.where(on(x), x + (e << 7), x).astype(np.uint16)  # noqa: E731
    for b, e in enumerate((18, 0, -20)):
        c.q[c.cu[b]:c.cu[b + 1]] = times(c.q[c.cu[b]:c.cu[b + 1]].astype(np.int32), -e)
        for j in c.table[b][c.table[b] >= 0]:
            c.kp[j] = times(c.kp[j].astype(np.int32), e)
    say("magnitudes", n)
    assert_close(to_f64(c.run(150, 60)), want, what="magnitudes")


def test_two_graphs_and_an_eager_call_at_once():
    """Calls of different sizes on three streams, two of them replays of graphs that one stream captured:
    none sees another's workspace."""
    cs = [Chunks([900, 300], [260, 200], 8, 2, 64, seed=61), Chunks([400, 77, 500], [3, 70, 130], 8, 2, 64, seed=62),
          Chunks([1200], [700], 8, 2, 64, seed=63)]
    data = [(to_dev(c.q), to_dev(c.kp), to_dev(c.vp), _i32(c.table), _i32(c.cu), _i32(c.lens)) for c in cs]
    run = lambda i, **kw: api.prefill_varlen_paged(*data[i], w_pretrained=150, w_local=60, **kw)  # noqa: E731
    say("at once")
    want = [run(i) for i in range(3)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(i))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for turn in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        with torch.cuda.stream(streams[2]):
            outs[2:] = [run(2)]
        torch.cuda.synchronize()
        for i in range(3):
            assert torch.equal(outs[i], want[i]), (turn, i)


def test_the_workspace_is_the_callers():
    c = Chunks([300, 90], [150, 2], 8, 2, 64, seed=65)
    data = (to_dev(c.q), to_dev(c.kp), to_dev(c.vp), _i32(c.table), _i32(c.cu), _i32(c.lens))
    n = api.varlen_paged_workspace_bytes(2, 152, 8, 2, c.max_pages, 64)
    say("workspace")
    ws = torch.full((n + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    one = api.prefill_varlen_paged(*data, w_pretrained=100, w_local=30, workspace=ws[:n])
    torch.cuda.synchronize()
    assert (ws[n:] == 0xFF).all()
    assert torch.equal(one, api.prefill_varlen_paged(*data, w_pretrained=100, w_local=30))
    with pytest.raises(api.JetLongError) as e:
        api.prefill_varlen_paged(*data, w_pretrained=100, w_local=30, workspace=ws[:n - 16])
    assert e.value.status == api.JL_ERR_WORKSPACE


@pytest.mark.parametrize("n", [3, 100, 300])
@pytest.mark.parametrize("shape", ["rising", "falling", "zigzag", "one peak"])
def test_references_follow_exact_scores(n, shape):
    """One slow channel holds whole numbers: its rotation is the identity to 1e-3 and to 1e-6 in the
    scores, 4.08 log2 units a step, whose differences bf16 holds to 2^-8: the weight of a step, 0.06, is
    off by 0.0007.  The references move by hundreds; tolerances as above."""
    c = Chunks([700, 300], [n, 5], 8, 2, 64, seed=70)
    for b, (q, k, v) in enumerate(c.seqs):
        L = c.lens[b]
        x = {"rising": np.linspace(-120, 120, L), "falling": np.linspace(120, -120, L),
             "zigzag": 100 * np.cos(np.arange(L) / 9.0),
             "one peak": np.where(np.arange(L) == L // 3, 110, -110)}[shape].round()
        qq, kk = np.zeros(q.shape, np.float32), np.zeros(k.shape, np.float32)
        qq[..., 63], kk[..., 63] = 32.0, x.astype(np.float32)[None, :, None]
        c.seqs[b] = (synth.bf16_bits(qq), synth.bf16_bits(kk), v)
        for j in range(-(-L // 64)):
            part = slice(64 * j, min(64 * j + 64, L))
            c.kp[c.table[b, j], :part.stop - part.start] = c.seqs[b][1][0, part]
    c.q = np.concatenate([s[0][0, L - m:] for s, L, m in zip(c.seqs, c.lens, c.n)])
    say("exact scores", n, shape)
    for bifocal in (True, False):
        out, lse = c.run(256, 90, bifocal, want_lse=True)
        o, l = c.want(256, 90, bifocal)
        assert_close(to_f64(out), o, what="out")
        # row sums of 340 at most, by a query that is rounded to half a step of bf16, 2^-8 of itself:
        # 4.0803 to 4.09375
        assert np.abs(lse.cpu().numpy() - l).max() < 340 * 2.0 ** -8 + 2e-2


@pytest.mark.parametrize("lens,n,w_pre,w0", [
    ([30], [4], 16, 8), ([60], [16], 32, 20), ([80], [16], 64, 40),
    ([80, 30, 40, 60], [16, 1, 3, 16], 16, 8)])
@pytest.mark.parametrize("exp", [18, -30])
def test_short_sequences_of_any_magnitude(lens, n, w_pre, w0, exp):
    """As above, where a few rows of a short sequence are whole in one workgroup and two pairs of waves
    take its visits: the second run's result has to stand, its row sums too.  The softmax has 27 keys
    at least, so its weights' squares sum to 0.16 at most, and the scores' 0.007 rms move outputs and row
    sums by 0.0028 rms, 0.0025 in the mean with the outputs' and the weights' own rounding; 3e-3, and ten
    times that for the largest.  The run in fp16 gives NaN (exp 18) or equal weights (-30)."""
    c = Chunks(lens, n, 8, 2, 16, seed=sum(lens))
    o, l = c.want(w_pre, w0)
    on = lambda x: ((x & 0x7F80) != 0) & ((x & 0x7F80) != 0x7F80)  # noqa: E731
    times = lambda x, e: np.where(on(x), x + (e << 7), x).astype(np.uint16)  # noqa: E731
    c.q, c.kp = times(c.q.astype(np.int32), -exp), times(c.kp.astype(np.int32), exp)
    say("short magnitudes", lens, exp)
    out, lse = c.run(w_pre, w0, want_lse=True)
    assert_close(to_f64(out), o, 3e-2, 3e-3, what="out")
    assert_close(lse.cpu().numpy(), l, 3e-2, 3e-3, what="lse")


@pytest.mark.parametrize("page", [16, 64])
def test_the_largest_batch(page):
    """2048 sequences of a token each, every hundredth a prompt, which with the larger pages run as
    blocks."""
    b = np.arange(2048)
    lens = np.where(b % 100 == 7, 90, 1 + b % 37).tolist()
    n = np.where(b % 100 == 7, 85, 1).tolist()
    c = Chunks(lens, n, 2, 1, page, seed=71)
    say("largest batch", page)
    out, lse = c.run(40, 30, want_lse=True)
    o, l = c.want(40, 30)
    assert_close(to_f64(out), o, what="out")
    # the row sum of a single key carries its score's error, in fp16 an eighth of 0.007 rms
    assert_close(lse.cpu().numpy(), l, what="lse")


@pytest.mark.parametrize("page", [16, 64])
def test_as_many_sequences_and_rows_as_a_call_takes(page):
    """2048 whole prompts of 1.3 million rows in all, against the packed prefill without pages."""
    g = torch.Generator(device="cuda").manual_seed(page)
    B, most = 2048, 256
    n = 128 + np.arange(B) % 63
    T, per = int(n.sum()), most // page
    assert api.varlen_paged_workspace_bytes(B, T, 4, 1, per, page) > 0
    assert api.varlen_paged_workspace_bytes(B, T + 6000, 4, 1, per, page) == 0
    table = torch.randperm(B * per, generator=g, device="cuda").view(B, per)
    q, k, v = (torch.randn((T, h, 128), generator=g, device="cuda").to(torch.bfloat16) for h in (4, 1, 1))
    cu = np.concatenate([[0], np.cumsum(n)])
    kp, vp = (torch.zeros((B * per, page, 1, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = table.to(torch.int32)
    say("most rows", page, T)
    api.cache_append(kp, vp, k, v, torch.zeros(B, dtype=torch.int32, device="cuda"), block_table=table,
                     cu_seqlens=_i32(cu))
    out = api.prefill_varlen_paged(q, kp, vp, table, _i32(cu), _i32(n), w_pretrained=100, w_local=40)
    want = api.prefill_varlen(q, k, v, _i32(cu), max_seqlen=int(n.max()), w_pretrained=100, w_local=40)
    torch.cuda.synchronize()
    off = (out.float() - want.float()).abs()  # each is within half of these bounds of 64 bits
    assert off.max().item() <= 4e-2 and off.mean().item() <= 4e-3


def test_more_parts_than_a_launch_has_threads():
    """A prompt beside a thousand tokens, of so many kv heads that the blocks' parts pass 2^32 threads:
    the last heads are right too."""
    Hkv, B, L, page = 4096, 1013, 1100, 64
    g = torch.Generator(device="cuda").manual_seed(9)
    kp, vp = (torch.randn((18, page, Hkv, 128), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = torch.zeros((B, 18), dtype=torch.int32, device="cuda")
    table[0] = torch.arange(18)
    T = L + B - 1
    q = torch.randn((T, Hkv, 128), generator=g, device="cuda", dtype=torch.bfloat16)
    cu = torch.cat([_i32([0]), L + torch.arange(B, device="cuda", dtype=torch.int32)])
    lens = _i32([L] + [3] * (B - 1))
    say("parts past 32 bits")
    out = torch.full_like(q, float("nan"))
    api.prefill_varlen_paged(q, kp, vp, table, cu, lens, w_pretrained=600, w_local=300, out=out)
    few = [0, 1, Hkv // 2, Hkv - 1]
    pools = [x[:, :, few].contiguous() for x in (kp, vp)]
    want = api.prefill_varlen_paged(q[:, few].contiguous(), *pools, table, cu, lens, w_pretrained=600,
                                    w_local=300)
    torch.cuda.synchronize()
    off = (out[:, few].float() - want.float()).abs()  # each is within half of these bounds of 64 bits
    assert off.max().item() <= 4e-2 and off.mean().item() <= 4e-3
    del out, q, kp, vp
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [[3, 70, 1], [300, 260, 200]])
@pytest.mark.parametrize("small", [1e-5, 1e-30, 0.0])
def test_a_few_small_channels_in_a_normal_row(n, small):
    """Every ninth key of one sequence and every fifth query of another have eight channels and their
    partners, and half of them, near nothing, below fp16's normal values: blocks take their second
    run, the rows' kernel does not."""
    c = Chunks([400, 300, 260], n, 8, 2, 64, seed=81)
    tiny = np.concatenate([np.arange(24, 32), np.arange(88, 96)])
    some = np.concatenate([np.arange(8, 128, 16) + i for i in range(8)])
    q, k, v = c.seqs[0]
    k = k.copy()
    x = small * np.random.default_rng(1).standard_normal(k[:, ::9][..., tiny].shape)
    for i, ch in enumerate(tiny):
        k[:, ::9, :, ch] = synth.bf16_bits(x[..., i].astype(np.float32))
    c.seqs[0] = (q, k, v)
    for j in range(-(-400 // 64)):
        part = slice(64 * j, min(64 * j + 64, 400))
        c.kp[c.table[0, j], :part.stop - part.start] = k[0, part]
    q, k, v = c.seqs[1]
    q = q.copy()
    for ch in some:
        q[:, ::5, :, ch] = synth.bf16_bits(np.full(q[:, ::5, :, ch].shape, small, np.float32))
    c.seqs[1] = (q, k, v)
    c.q = np.concatenate([s[0][0, L - m:] for s, L, m in zip(c.seqs, c.lens, c.n)])
    say("small channels", n, small)
    out, lse = c.run(150, 60, want_lse=True)
    o, l = c.want(150, 60)
    assert_close(to_f64(out), o, what="out")
    assert_close(lse.cpu().numpy(), l, what="lse")


def test_pools_past_32_bits():
    """The same pages at the end of pools of 4.7 GB: appended, copied, decoded over and behind chunks,
    the same bits as in small ones."""
    Hq, Hkv, page, far = 16, 8, 64, 36000
    lens, n = [700, 640, 300], [300, 90, 1]
    c = Chunks(lens, n, Hq, Hkv, page, seed=91)
    kp, vp, q, cu, L = to_dev(c.kp), to_dev(c.vp), to_dev(c.q), _i32(c.cu), _i32(lens)
    table = _i32(c.table)
    big = [torch.zeros((far, page, Hkv, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    at = torch.where(table >= 0, far - 1 - table, table)
    say("pools past 32 bits")
    for b, m in enumerate(lens):  # through the append, but the last page, which a copy brings
        rows = [torch.cat([x[p] for p in c.table[b][c.table[b] >= 0]])[:m] for x in (kp, vp)]
        api.cache_append(*big, *[x[None].contiguous() for x in rows], _i32([0]),
                         block_table=at[b:b + 1].contiguous())
    p = int(c.table[0, 2])
    for x in big:
        x[5] = x[far - 1 - p]
        x[far - 1 - p] = 0
    api.copy_pages(big, _i32([[5, far - 1 - p]]), _i32([1]))
    for x, small in zip(big, (kp, vp)):
        for b, m in enumerate(lens):
            for j in range(-(-m // page)):
                e, k = int(c.table[b, j]), min(page, m - j * page)
                assert torch.equal(x[far - 1 - e, :k], small[e, :k])
    for kw in (dict(w_pretrained=200, w_local=70), dict(bifocal=False)):
        for rows in (c.cu[-1], 6):  # blocks and the rows' kernel, the latter alone
            cut = cu if rows == c.cu[-1] else _i32([0, 2, 5, 6])
            a, z = (api.prefill_varlen_paged(q[:rows].contiguous(), *pools, t, cut, L, **kw)
                    for pools, t in (((kp, vp), table), (big, at)))
            assert torch.equal(a, z)
        plan = api.shared_plan(L, _i32([0, 1, 2, 3]), _i32([0, 0, 0]), Hq=Hq, Hkv=Hkv, page_size=page,
                               max_pages=c.max_pages, **kw)
        a, z = (api.decode_shared(q[:3].contiguous(), *pools, t, plan)
                for pools, t in (((kp, vp), table), (big, at)))
        assert torch.equal(a, z) and torch.isfinite(a.float()).all()
    del big
    torch.cuda.empty_cache()
