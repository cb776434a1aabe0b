"""Decode over shared prefixes against the fp64 oracle, which reads every sequence's keys from a
dense cache of its own.

Tolerances: the parity bounds of the decode and prefill tests.  With u = 2^-8 the unit roundoff of
bf16, a score <q, k> / sqrt(128) of unit normals carries the roundings of the rotated query, of
cos and sin and of the rotated key (where they are not in fp16): three of relative size u / sqrt(3) in the mean square on
products whose root sum of squares is 1, so 0.004 to 0.007 rms.  That shifts an output,
a weighted mean of values of size 1, by less than its own size times the root of the
sum of the squared weights: below 0.004 rms, 0.02 at five times that with the output's own
rounding (u |o| / 2 at most 0.008 for |o| < 4).  2e-2 and 2e-3 in the mean."""
import ctypes

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


class Batch:
    """Groups (n sequences, common tokens, own lengths behind them) on shuffled pages: whole pages of
    a prefix are named by all of its group.  Unused pages and rows hold NaN.  order: where the
    groups' sequences lie in the batch."""

    def __init__(self, groups, Hq, Hkv, page, seed, shuffle=False, spare=2):
        rng = np.random.default_rng(seed)
        self.Hq, self.Hkv, self.page = Hq, Hkv, page
        lens, share, fork = [], [], []
        for pre, own in groups:
            share.append(pre)
            fork.append(len(own))
            lens += [pre + x for x in own]
        B = len(lens)
        self.B = B
        self.order = rng.permutation(B) if shuffle else np.arange(B)
        cap = -(-max(max(lens), 1) // page) + spare
        self.max_pages = cap
        q, k, v, _ = synth.decode_inputs(B, Hq, Hkv, max(max(lens), 1), lens, seed=seed + 1,
                                         nan_tail=True, outlier_channels=8)
        at = 0
        for pre, own in groups:
            for b in range(at + 1, at + len(own)):
                k[b, :pre], v[b, :pre] = k[at, :pre], v[at, :pre]
            at += len(own)
        n_pages = sum(-(-x // page) for x in lens) + 3
        deal = iter(rng.permutation(n_pages))
        kp = np.full((n_pages, page, Hkv, 128), NAN, np.uint16)
        vp = np.full_like(kp, NAN)
        table = np.full((B, cap), -1, np.int32)
        at = 0
        for pre, own in groups:
            for b in range(at, at + len(own)):
                for j in range(-(-lens[b] // page)):
                    if b > at and j < pre // page:
                        table[b, j] = table[at, j]
                        continue
                    p = next(deal)
                    table[b, j] = p
                    lo, hi = j * page, min((j + 1) * page, lens[b])
                    kp[p, :hi - lo], vp[p, :hi - lo] = k[b, lo:hi], v[b, lo:hi]
            at += len(own)
        # member i of the groups is sequence order[i] of the batch
        back = np.argsort(self.order)
        self.q, self.k, self.v = q[back], k[back], v[back]
        self.lens = np.asarray(lens, np.int32)[back]
        self.table, self.kp, self.vp = table[back], kp, vp
        self.starts = np.concatenate([[0], np.cumsum(fork)])
        self.share = np.asarray(share)

    def plan(self, w_pre, w0, bifocal, **kw):
        kw.setdefault("members", _i32(self.order))
        return api.shared_plan(_i32(self.lens), _i32(self.starts), _i32(self.share), Hq=self.Hq,
                               Hkv=self.Hkv, page_size=self.page, max_pages=self.max_pages,
                               w_pretrained=w_pre, w_local=w0, bifocal=bifocal, **kw)

    def run(self, plan, theta=1e6, **kw):
        return api.decode_shared(to_dev(self.q), to_dev(self.kp), to_dev(self.vp),
                                 _i32(self.table), plan, rope_theta=theta, **kw)

    def want(self, w_pre, w0, bifocal, theta=1e6):
        one = np.maximum(self.lens, 1)
        o, _, _ = O.decode(self.q, self.k, self.v, one, theta=theta, w_pretrained=w_pre, w_local=w0,
                           bifocal=bifocal)
        o[self.lens == 0] = 0
        return o


# (prefix, own lengths): forks of one length, ragged ones, several groups, single sequences,
# prefixes that end inside a page or hold no whole one, sequences that end with the prefix
GROUPS = [
    [(0, [1])],
    [(0, [77, 1, 300])],
    [(128, [5, 5])],
    [(130, [1, 40, 7, 200, 33]), (0, [60]), (65, [3, 3, 90])],
    [(300, [0, 1, 64, 129])],
    [(700, list(range(1, 72)))],
    [(15, [40, 50]), (16, [1, 1]), (31, [2, 3]), (32, [1, 9]), (33, [4, 4])],
]


@pytest.mark.parametrize("groups", range(len(GROUPS)))
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("bifocal", [True, False])
def test_matches_oracle(groups, page, bifocal):
    Hq, Hkv = [(8, 2), (4, 4), (16, 2), (6, 2), (5, 1), (8, 2), (14, 2)][groups]
    b = Batch(GROUPS[groups], Hq, Hkv, page, seed=10 * groups + page, shuffle=groups % 2 == 1)
    say("decode_shared", groups, page, bifocal)
    out = b.run(b.plan(96, 40, bifocal))
    torch.cuda.synchronize()
    assert_close(to_f64(out), b.want(96, 40, bifocal), what="groups %d page %d" % (groups, page))


@pytest.mark.parametrize("w_pre,w0", [(1, 0), (64, 0), (100, 7), (128, 300), (333, 31),
                                      (1000, 2147483647), (7, 1 << 20)])
def test_views_that_differ_inside_a_group(w_pre, w0):
    """Sequences of one prefix whose G and local windows differ."""
    b = Batch([(640, [1, 30, 64, 100, 199, 350, 351, 640]), (64, [10, 700])], 8, 2, 64, seed=w_pre)
    say("views", w_pre, w0)
    out = b.run(b.plan(w_pre, w0, True))
    torch.cuda.synchronize()
    assert_close(to_f64(out), b.want(w_pre, w0, True), what="w_pre %d w0 %d" % (w_pre, w0))


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 1), (7, 1), (32, 8), (64, 8), (28, 4), (3, 3)])
def test_head_layouts_and_many_rows(Hq, Hkv):
    """More rows than one block holds, for every group size of query heads."""
    n = 300 * Hkv // Hq + 3
    b = Batch([(200, [(7 * i) % 90 + 1 for i in range(n)])], Hq, Hkv, 32, seed=Hq, shuffle=True)
    say("heads", Hq, Hkv, n)
    out = b.run(b.plan(150, 60, True))
    torch.cuda.synchronize()
    assert_close(to_f64(out), b.want(150, 60, True), what="heads %d/%d" % (Hq, Hkv))


def test_long_prefix_in_parts():
    """Ranges of more tiles than one list holds, one kv head, and a far position."""
    b = Batch([(70001, [3, 500, 1500])], 4, 1, 64, seed=3)
    say("long prefix")
    for bif in (True, False):
        out = b.run(b.plan(16384, 1000, bif))
        torch.cuda.synchronize()
        assert_close(to_f64(out), b.want(16384, 1000, bif), what="long prefix")


def test_many_kv_heads_leave_few_workgroups():
    b = Batch([(20000, [100, 2000])], 128, 128, 64, seed=5)
    say("128 kv heads")
    out = b.run(b.plan(8192, 1000, True))
    torch.cuda.synchronize()
    assert_close(to_f64(out), b.want(8192, 1000, True), what="128 kv heads")


def test_agrees_with_the_paged_decode_and_gives_the_same_bits_twice():
    b = Batch([(512, [9, 100, 30]), (0, [800])], 8, 2, 64, seed=11)
    plan = b.plan(300, 50, True)
    say("same bits")
    one, two = b.run(plan), b.run(plan)
    ws = torch.full((api.decode_shared_workspace_bytes(b.B, 8, 2),), 0xFF, dtype=torch.uint8,
                    device="cuda")  # NaN
    three = b.run(plan, workspace=ws)
    ref = api.decode_paged(to_dev(b.q), to_dev(b.kp), to_dev(b.vp), _i32(b.table), _i32(b.lens),
                           w_pretrained=300, w_local=50)
    torch.cuda.synchronize()
    assert torch.equal(one, two) and torch.equal(one, three)
    assert_close(to_f64(one), to_f64(ref), what="paged decode")


def test_empty_sequences_and_rows_of_no_group():
    b = Batch([(128, [4, 9, 70]), (0, [50]), (0, [40])], 8, 2, 64, seed=17)
    lens = b.lens.copy()
    lens[1] = 0
    out = torch.full((5, 8, 128), 3.0, device="cuda").to(torch.bfloat16)
    say("empty ones")
    plan = api.shared_plan(_i32(lens), _i32([0, 3, 4]), _i32([128, 0]), Hq=8, Hkv=2, page_size=64,
                           max_pages=b.max_pages, members=_i32([0, 1, 2, 3, 77]), w_pretrained=90,
                           w_local=30)
    b.run(plan, out=out)
    torch.cuda.synchronize()
    want = b.want(90, 30, True)
    want[1] = 0
    assert (out[4] == 3.0).all() and (out[1] == 0).all()
    assert_close(to_f64(out[:4]), want[:4], what="empty ones")
    say("nothing at all")
    plan = api.shared_plan(_i32([0] * 5), _i32([0, 5]), _i32([64]), Hq=8, Hkv=2, page_size=64,
                           max_pages=b.max_pages)
    assert (b.run(plan) == 0).all()


def test_bad_lists_do_not_leave_the_arrays():
    """Members, starts, lengths and pages far outside: wrong values at most."""
    b = Batch([(128, [4, 9, 70]), (0, [50]), (0, [40])], 8, 2, 64, seed=19)
    for starts, share, members, lens in (
            ([-5, 9, 2, 2147483647], [1 << 30, -7, 64], [4, -1, 2147483647, 0, 1], b.lens),
            ([3, 1, 0, 5], [64, 64, 64], [0, 1, 2, 3, 4], [2147483647, -9, 1, 100, 5]),
            ([0, 5, 5, 5], [2147483647] * 3, [-2147483648] * 5, b.lens)):
        say("bad lists", starts)
        plan = api.shared_plan(_i32(lens), _i32(starts), _i32(share), Hq=8, Hkv=2, page_size=64,
                               max_pages=b.max_pages, members=_i32(members), w_pretrained=90,
                               w_local=30)
        table = b.table.copy()
        table[0, :2] = [1 << 30, -(1 << 31)]
        api.decode_shared(to_dev(b.q), to_dev(b.kp), to_dev(b.vp), _i32(table), plan)
        torch.cuda.synchronize()


def test_a_plan_of_other_sizes_is_refused():
    b = Batch([(128, [4, 9, 70])], 8, 2, 64, seed=23)
    plan = b.plan(90, 30, True)
    with pytest.raises(ValueError):
        api.decode_shared(to_dev(b.q), to_dev(b.kp), to_dev(b.vp), _i32(b.table[:, :-1].copy()), plan)
    with pytest.raises(ValueError):
        api.decode_shared(to_dev(b.q[:2]), to_dev(b.kp), to_dev(b.vp), _i32(b.table), plan)
    with pytest.raises(ValueError):
        b.plan(91, 30, True, out=plan)
    with pytest.raises(TypeError):
        api.decode_shared(to_dev(b.q), to_dev(b.kp), to_dev(b.vp), _i32(b.table), plan.buf)
    with pytest.raises(api.JetLongError) as e:
        b.run(plan, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert e.value.status == api.JL_ERR_WORKSPACE
    # through the C entry a plan of other windows computes nothing
    out = torch.full((3, 8, 128), 5.0, device="cuda").to(torch.bfloat16)
    q, k, v, t = to_dev(b.q), to_dev(b.kp), to_dev(b.vp), _i32(b.table)
    ws = torch.empty(api.decode_shared_workspace_bytes(3, 8, 2), dtype=torch.uint8, device="cuda")
    p = lambda x: ctypes.c_void_p(x.data_ptr())  # noqa: E731
    say("plan of other windows")
    st = api.lib().jl_bifocal_decode_shared(
        p(q), p(k), p(v), p(t), b.max_pages, 64, b.kp.shape[0], plan.ptr, plan.nbytes, p(out), 3, 1,
        8, 2, 128, 1e6, 91, 30, p(ws), ws.nbytes, None)
    torch.cuda.synchronize()
    assert st == api.JL_OK and (out == 5.0).all()


def test_a_captured_step_follows_the_lengths():
    """Plan and decode captured, replayed for growing sequences, on another stream than the inputs'."""
    b = Batch([(192, [1, 20, 64]), (64, [5, 5])], 8, 2, 64, seed=29, spare=3)
    full = b.lens.copy()
    q, k, v, t = to_dev(b.q), to_dev(b.kp), to_dev(b.vp), _i32(b.table)
    lens = _i32(full)
    kw = dict(Hq=8, Hkv=2, page_size=64, max_pages=b.max_pages, w_pretrained=100, w_local=40)
    starts, share = _i32(b.starts), _i32(b.share)
    plan = api.shared_plan(lens, starts, share, **kw)
    ws = torch.empty(api.decode_shared_workspace_bytes(b.B, 8, 2), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    api.decode_shared(q, k, v, t, plan, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.shared_plan(lens, starts, share, out=plan, **kw)
        api.decode_shared(q, k, v, t, plan, out=out, workspace=ws)
    for i in range(6):
        now = np.maximum(full - 11 * i, 1) if i != 3 else np.asarray([193, 0, 1, 69, 2])
        lens.copy_(_i32(now))
        say("replay", i)
        graph.replay()
        torch.cuda.synchronize()
        eager = api.decode_shared(q, k, v, t, api.shared_plan(lens, starts, share, **kw))
        torch.cuda.synchronize()
        assert torch.equal(out, eager), i
        b.lens = now.astype(np.int32)
        assert_close(to_f64(out), b.want(100, 40, True), what="replay %d" % i)


def test_two_plans_on_two_streams():
    bs = [Batch([(256, [3, 50, 70]), (0, [300])], 8, 2, 64, seed=s) for s in (31, 37)]
    want = [b.want(120, 30, True) for b in bs]
    data = [(to_dev(b.q), to_dev(b.kp), to_dev(b.vp), _i32(b.table), _i32(b.lens), _i32(b.starts),
             _i32(b.share)) for b in bs]
    streams = [torch.cuda.Stream() for _ in bs]
    torch.cuda.synchronize()
    say("two streams")
    outs = []
    for _ in range(5):
        for b, s, d in zip(bs, streams, data):
            plan = api.shared_plan(d[4], d[5], d[6], Hq=8, Hkv=2, page_size=64,
                                   max_pages=b.max_pages, w_pretrained=120, w_local=30, stream=s)
            outs.append(api.decode_shared(*d[:4], plan, stream=s))
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        assert_close(to_f64(o), want[i % 2], what="stream %d" % (i % 2))


@pytest.mark.parametrize("B,n", [(2048, 2048), (2048, 1), (1, 2048), (1500, 700)])
def test_the_largest_batches(B, n):
    """As many sequences and groups as a plan takes: every sequence of a few tokens, every tenth long."""
    page, Hkv = 16, 1
    g = torch.Generator(device="cuda").manual_seed(B + n)
    starts = np.minimum(np.arange(n + 1) * -(-B // n), B)
    share = np.full(n, 16)
    lens = np.where(np.arange(B) % 10 == 0, 90, 20) + np.arange(B) % 5
    first = starts[np.searchsorted(starts, np.arange(B), side="right") - 1]
    table = 8 * np.arange(B)[:, None] + np.arange(8)
    table[:, 0] = 8 * first  # the prefix page is the first one's
    kp = torch.randn((8 * B, page, Hkv, 128), generator=g, device="cuda").to(torch.bfloat16)
    vp = torch.randn((8 * B, page, Hkv, 128), generator=g, device="cuda").to(torch.bfloat16)
    q = torch.randn((B, 2, 128), generator=g, device="cuda").to(torch.bfloat16)
    say("largest batches", B, n)
    plan = api.shared_plan(_i32(lens), _i32(starts), _i32(share), Hq=2, Hkv=Hkv, page_size=page,
                           max_pages=8, w_pretrained=40, w_local=30)
    out = api.decode_shared(q, kp, vp, _i32(table), plan)
    ref = api.decode_paged(q, kp, vp, _i32(table), _i32(lens), w_pretrained=40, w_local=30)
    torch.cuda.synchronize()
    assert_close(to_f64(out), to_f64(ref), what="largest batches")


def _times(bits, e):
    """bf16 bit patterns times 2^e; zeros and NaN stay."""
    x = bits.astype(np.int32)
    on = ((x & 0x7F80) != 0) & ((x & 0x7F80) != 0x7F80)
    assert (((x >> 7 & 255) + e)[on] > 0).all() and (((x >> 7 & 255) + e)[on] < 255).all()
    return np.where(on, x + (e << 7), x).astype(np.uint16)


@pytest.mark.parametrize("group", [False, True])
@pytest.mark.parametrize("exps", [[17, 0, 0, 0], [0, -14, 40, -40], [15, 16, -7, -9]])
def test_keys_and_queries_of_any_magnitude(group, exps):
    """Keys times 2^e, their queries times 2^-e: the scores of the same values, for single
    sequences and a group's, beside others."""
    sizes = [(0, [300]), (0, [70]), (0, [129]), (0, [33])]
    if group:
        sizes = [(130, [3, 40, 1 + i]) for i in range(4)]
    b = Batch(sizes, 8, 2, 32, seed=41)
    want = b.want(100, 40, True)
    per = len(sizes[0][1])
    for s in range(b.B):
        e = exps[s // per]
        b.q[s] = _times(b.q[s], -e)
        for j in set(b.table[s][b.table[s] >= 0]):
            if s % per == 0 or j not in b.table[s - 1]:
                b.kp[j] = _times(b.kp[j], e)
    say("magnitudes", group, exps)
    out = b.run(b.plan(100, 40, True))
    torch.cuda.synchronize()
    assert_close(to_f64(out), want, what="magnitudes")


def test_zero_keys_and_queries():
    b = Batch([(64, [40, 9])], 8, 2, 32, seed=43)
    b.kp[b.table[0, 0], 3:20] = 0
    b.k[:, 3:20] = 0
    b.q[1] = 0
    say("zeros")
    out = b.run(b.plan(50, 20, True))
    torch.cuda.synchronize()
    assert_close(to_f64(out), b.want(50, 20, True), what="zeros")


def test_distance_from_64_bits():
    """Rounded to bf16 are the weights and the output, each by 0.42 of 2^-8 of its size in the root
    mean square; the weights' errors reach an output, a mean of independent values, undiminished.
    Together 0.0024 of the output's size; the scores, in fp16, add a tenth: 0.003."""
    b = Batch([(2000, [1, 30, 300, 700]), (0, [900])], 8, 2, 64, seed=47)
    for w_pre in (600, 4096):
        out = b.run(b.plan(w_pre, 200, True))
        torch.cuda.synchronize()
        want = b.want(w_pre, 200, True)
        off = np.linalg.norm(to_f64(out) - want) / np.linalg.norm(want)
        say("distance", w_pre, off)
        assert off < 3e-3


def test_two_graphs_at_once():
    """Steps captured on one stream, plan and workspace their own, replayed on two at once."""
    bs = [Batch([(256, [3, 50, 70]), (0, [300])], 8, 2, 64, seed=71), Batch([(640, [9, 1]), (64, [64] * 5)], 8, 2, 64, seed=72)]
    data = [(to_dev(b.q), to_dev(b.kp), to_dev(b.vp), _i32(b.table), _i32(b.lens), _i32(b.starts), _i32(b.share)) for b in bs]

    def step(b, d):
        plan = api.shared_plan(d[4], d[5], d[6], Hq=8, Hkv=2, page_size=64, max_pages=b.max_pages,
                               w_pretrained=120, w_local=30)
        return api.decode_shared(*d[:4], plan)

    say("two graphs")
    want = [step(b, d) for b, d in zip(bs, data)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for b, d in zip(bs, data):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(b, d))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in bs]
    for turn in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i], want[i]), (turn, i)
            assert_close(to_f64(outs[i]), bs[i].want(120, 30, True), what="graph %d" % i)


def test_one_sequence_of_large_keys_leaves_the_others_right():
    """Its ranges run in bf16; what stands beside them is right too, and the same twice."""
    b = Batch([(192, [40, 9]), (0, [700]), (0, [100])], 8, 2, 64, seed=73)
    want = b.want(100, 40, True)
    b.q[2] = _times(b.q[2], -30)
    for j in b.table[2][b.table[2] >= 0]:
        b.kp[j] = _times(b.kp[j], 30)
    plan = b.plan(100, 40, True)
    say("large keys of one")
    one, two = b.run(plan), b.run(plan)
    torch.cuda.synchronize()
    assert torch.equal(one, two)
    assert_close(to_f64(one), want, what="large keys of one")
