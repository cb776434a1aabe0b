"""Pages of a batch on the GPU against a plain model that takes one entry after another:
whole numbers are equal, copied bytes are equal."""
import numpy as np
import pytest

from pages_util import Model, filled, n_pages_of, same, to_device
from parity_util import say
from paper_2607_07740_amd import api

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# sequences, entries of a row, pages, tokens of a page: a single one of each; odd ones; more pages
# than one strip of counts; more sequences than threads
SIZES = [(1, 1, 1, 1), (3, 7, 19, 5), (33, 40, 700, 16), (64, 33, 2000, 64), (7, 130, 16384, 64),
         (20, 500, 40001, 3), (1500, 9, 9000, 4), (2048, 3, 5000, 64)]


def _i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


@pytest.mark.parametrize("size", SIZES)
def test_fork_takes_all_rows_at_once(size):
    rng = np.random.default_rng(sum(size))
    m = filled(rng, *size)
    pages = to_device(m, torch)
    B = size[0]
    for kind in ("any", "beams", "stay", "free", "swap"):
        say("pages_fork", size, kind)
        parent = {"any": rng.integers(-2, B + 2, B), "beams": rng.integers(0, B, B),
                  "stay": np.arange(B), "swap": np.arange(B)[::-1],
                  "free": np.where(rng.random(B) < 0.5, np.arange(B), -1)}[kind]
        api.pages_fork(pages, _i32(parent))
        m.fork(parent.tolist())
        same(pages, m)


@pytest.mark.parametrize("size", SIZES)
def test_reserve_deals_the_lowest_free_pages_in_order(size):
    rng = np.random.default_rng(7 + sum(size))
    B, max_pages, n_pages, page = size
    for most in (0, 1, page, 3 * page + 1):
        m = filled(rng, B, max_pages, n_pages - n_pages // 3, page)
        m.n_pages = n_pages
        m.refs += [0] * (n_pages // 3)
        room = [max_pages * page - x for x in m.lens]
        n_new = [int(min(r, x)) for r, x in zip(room, rng.integers(-1, most + 1, B))]
        pages = to_device(m, torch)
        say("pages_reserve", size, most)
        starts, granted, moves, info = api.pages_reserve(pages, _i32(n_new))
        want = m.reserve(n_new)
        assert info.tolist() == want[3]
        assert starts.tolist() == want[0] and granted.tolist() == want[1]
        assert moves.tolist() == [list(x) for x in want[2]] + [[-1, -1]] * (B - len(want[2]))
        same(pages, m)


def test_writers_of_a_shared_page_part_but_for_the_last():
    """Four rows name one partly filled page.  Where all of them write, the last one keeps it;
    where one does not, all writers part; a sequence whose page is full takes a new one."""
    for writing, copies in (([1, 1, 1, 1], 3), ([1, 0, 1, 1], 3), ([0, 0, 1, 0], 1), ([9, 1, 0, 0], 2)):
        m = Model(5, 8, 20, 8)
        m.lens, m.table[4][:2] = [13] * 4 + [16], [3, 9]
        for b in range(4):
            m.table[b][:2] = [5, 7]
        m.count()
        pages = to_device(m, torch)
        say("writers", writing)
        _, granted, moves, info = api.pages_reserve(pages, _i32(writing + [1]))
        want = m.reserve(writing + [1])
        assert info.tolist() == want[3] and want[3][0] == copies
        assert moves.tolist()[:copies] == [list(x) for x in want[2]]
        assert granted.tolist() == writing + [1]
        same(pages, m)


def test_reserve_changes_nothing_where_pages_do_not_suffice():
    m = Model(3, 4, 6, 8)
    for b in range(3):
        m.lens[b], m.table[b][0] = 5, 4
    m.count()
    for n_new, missing, over in (([8, 8, 17], 2, 0), ([1, 1, 28], 0, 1), ([30, 1, 0], 0, 1)):
        pages = to_device(m, torch)
        say("reserve", n_new)
        starts, granted, moves, info = api.pages_reserve(pages, _i32(n_new))
        got = info.tolist()
        assert got[0] == got[1] == 0 and got[3] == over and (got[2] > 0 or over)
        assert granted.tolist() == [0] * 3 and starts.tolist() == [5] * 3
        assert (moves == -1).all()
        same(pages, m)
    # what is just enough is dealt
    pages = to_device(m, torch)
    _, granted, _, info = api.pages_reserve(pages, _i32([8, 8, 9]))
    assert info.tolist() == list(m.reserve([8, 8, 9])[3]) and info.tolist()[1] == 5
    same(pages, m)


@pytest.mark.parametrize("size", SIZES)
def test_compact_numbers_the_pages_in_use_from_zero(size):
    rng = np.random.default_rng(13 + sum(size))
    m = filled(rng, *size)
    m.fork([b if rng.random() < 0.6 else -1 for b in range(size[0])])
    pages = to_device(m, torch)
    say("pages_compact", size)
    moves, info = api.pages_compact(pages)
    want, winfo = m.compact()
    assert info.tolist() == winfo
    assert moves.tolist() == [list(x) for x in want] + [[-1, -1]] * (size[2] // 2 - len(want))
    same(pages, m)
    moves, info = api.pages_compact(pages)  # nothing is left to move
    assert info.tolist() == [0, winfo[1], 0, 0] and (moves == -1).all()
    same(pages, m)


def test_bad_entries_are_not_followed():
    """Table entries outside the pool, lengths below zero and parents far outside."""
    B, n_pages = 6, 40
    table = torch.full((B, 5), -1, dtype=torch.int32, device="cuda")
    table[0] = _i32([3, 1 << 30, -7, 39, 40])
    table[1] = _i32([-2147483648, 2147483647, 5, 6, 7])
    lens = _i32([37, -5, 3, 2147483647, 0, 9])
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[[3, 39, 5, 6, 7]] = 1
    guard = refs.clone()
    pages = api.PageTable(lens, refs, table, 8)
    say("bad entries: fork")
    api.pages_fork(pages, _i32([0, 1, 2147483647, -2147483648, 0, 1]))
    assert refs.tolist()[3] == 2 and refs.tolist()[5] == 2 and int((refs - guard).sum()) == 5
    say("bad entries: reserve")
    api.pages_reserve(pages, _i32([1, 1, 1, 0, 1, 1]))
    say("bad entries: compact")
    moves, info = api.pages_compact(pages)
    assert info.tolist()[0] >= 0


@pytest.mark.parametrize("n_pools,shape,dtype", [
    (1, (3,), "float32"), (2, (64, 8, 128), "bfloat16"), (3, (5, 7, 1), "int32"),
    (70, (6,), "int32"), (2, (16, 1, 128), "bfloat16"), (1, (40, 3, 100), "float32")])
def test_copies_move_whole_pages(n_pools, shape, dtype):
    n_pages = 50
    g = torch.Generator(device="cuda").manual_seed(n_pools)
    pools = [torch.randint(-30000, 30000, (n_pages, *shape), generator=g, device="cuda").to(
        getattr(torch, dtype)) for _ in range(n_pools)]
    want = [p.clone() for p in pools]
    moves = _i32([[4, 9], [49, 0], [-1, 3], [5, 50], [7, 8], [11, 12]])
    for p in want:
        p[9], p[0], p[8] = p[4].clone(), p[49].clone(), p[7].clone()
    say("copy_pages", n_pools, shape)
    api.copy_pages(pools, moves, _i32([5]))  # the sixth is behind the count
    for p, w in zip(pools, want):
        assert torch.equal(p, w)
    api.copy_pages(pools, moves, _i32([0]))
    api.copy_pages(pools, moves[:0].contiguous(), _i32([7]))
    for p, w in zip(pools, want):
        assert torch.equal(p, w)


def test_copies_of_an_8_bit_cache_keep_what_it_reads():
    cache = api.cache8_alloc(12, 128, 3)
    x = torch.randn((1, 300, 3, 128), device="cuda").to(torch.bfloat16)
    table = _i32([[7, 2, 9]])
    api.cache8_append(cache, x, x, _i32([0]), block_table=table)
    before = api.cache8_read(cache, 300, block_table=table)
    say("copy_pages of a Cache8")
    api.copy_pages(cache, _i32([[7, 1], [2, 4], [9, 0]]), _i32([3]))
    after = api.cache8_read(cache, 300, block_table=_i32([[1, 4, 0]]))
    assert all(torch.equal(a, b) for a, b in zip(before, after))


@pytest.mark.parametrize("Hkv,page", [(1, 16), (8, 64), (3, 7), (8, 256)])
@pytest.mark.parametrize("packed", [False, True])
def test_append_puts_rows_where_they_belong(Hkv, page, packed):
    rng = np.random.default_rng(Hkv * page + packed)
    B, max_pages, n_pages = 70, 6, 430
    table = rng.permutation(n_pages)[:B * max_pages].reshape(B, max_pages)
    table[3, 2], table[5, 0] = -1, n_pages  # rows for these are dropped
    starts = rng.integers(0, max_pages * page, B)
    starts[:4] = [0, page - 1, page, 2 * page]
    n = rng.integers(0, 3 * page, B)
    n[1], n[2] = 0, 1
    cap = rng.integers(0, 3 * page, B)
    k = torch.full((n_pages, page, Hkv, 128), 7.0, device="cuda").to(torch.bfloat16)
    v = torch.full_like(k, -7.0)
    wk, wv = k.clone(), v.clone()
    rows = int(n.sum()) if packed else B * int(n.max())
    x = torch.randn((2, rows, Hkv, 128), device="cuda").to(torch.bfloat16)
    cu = np.concatenate([[0], np.cumsum(n)])
    for b in range(B):
        for i in range(int(min(n[b] if packed else n.max(), cap[b]))):
            pos = starts[b] + i
            if pos >= max_pages * page:
                break
            p = table[b, pos // page]
            if 0 <= p < n_pages:
                r = (cu[b] if packed else b * int(n.max())) + i
                wk[p, pos % page], wv[p, pos % page] = x[0, r], x[1, r]
    if not packed:
        x = x.view(2, B, -1, Hkv, 128)
    say("cache_append", Hkv, page, packed)
    api.cache_append(k, v, x[0], x[1], _i32(starts), n_new=_i32(cap), block_table=_i32(table),
                     cu_seqlens=_i32(cu) if packed else None)
    assert torch.equal(k, wk) and torch.equal(v, wv)


def test_append_to_a_dense_cache_and_bad_offsets():
    k = torch.zeros((3, 20, 2, 128), device="cuda", dtype=torch.bfloat16)
    v = torch.zeros_like(k)
    x = torch.randn((2, 3, 4, 2, 128), device="cuda").to(torch.bfloat16)
    say("append dense")
    api.cache_append(k, v, x[0], x[1], _i32([0, 18, -2]))
    wk = torch.zeros_like(k)
    wk[0, :4], wk[1, 18:], wk[2, :2] = x[0, 0], x[0, 1, :2], x[0, 2, 2:]
    assert torch.equal(k, wk)
    say("append, offsets that decrease and run past the rows")
    y = x[:, 0].contiguous()
    api.cache_append(k, v, y[0], y[1], _i32([0, 0, 0]), cu_seqlens=_i32([2, 900, -5, 3]))


def test_steps_of_forked_sequences_keep_their_contents():
    """Growing, forking, ending and compacting in turn: every sequence reads back the rows that it
    and its forebears were given.  On a side stream, captured and replayed."""
    rng = np.random.default_rng(5)
    B, max_pages, n_pages, page, Hkv = 12, 8, 80, 16, 2
    pages = api.pages_alloc(B, max_pages, n_pages, page)
    k = torch.zeros((n_pages, page, Hkv, 128), device="cuda", dtype=torch.bfloat16)
    v = torch.zeros_like(k)
    held = [torch.zeros((0, Hkv, 128), dtype=torch.bfloat16) for _ in range(B)]
    n_new, parent = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    rows = torch.zeros((2, B, 20, Hkv, 128), device="cuda", dtype=torch.bfloat16)

    def step():
        api.pages_fork(pages, parent)
        starts, granted, moves, info = api.pages_reserve(pages, n_new)
        api.copy_pages([k, v], moves, info)
        api.cache_append(k, v, rows[0], rows[1], starts, n_new=granted, block_table=pages.table)
        moves, info2 = api.pages_compact(pages)
        api.copy_pages([k, v], moves, info2)
        return info, info2

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        parent.copy_(torch.arange(B))
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        infos = step()
    for i in range(25):
        up = np.where(rng.random(B) < 0.3, rng.integers(-1, B, B), np.arange(B))
        if i % 6 == 5:
            up[rng.integers(0, B, 7)] = -1
        left = [held[p].shape[0] if p >= 0 else 0 for p in up]
        new = [int(min(x, max_pages * page - y)) for x, y in zip(rng.integers(0, 21, B), left)]
        x = torch.randn((2, B, 20, Hkv, 128)).to(torch.bfloat16)
        parent.copy_(torch.from_numpy(up.astype(np.int32)))
        n_new.copy_(torch.tensor(new, dtype=torch.int32))
        rows.copy_(x)
        say("step", i)
        if i % 2:
            graph.replay()
            info = infos[0]
        else:
            info = step()[0]
        held = [held[p] if p >= 0 else held[0][:0] for p in up]
        if info.tolist()[2] == 0:
            held = [torch.cat([h, x[0, b, :new[b]]]) for b, h in enumerate(held)]
        lens, table, refs = pages.lens.tolist(), pages.table.cpu(), pages.refs.tolist()
        used = [p for r in table.tolist() for p in r if p >= 0]
        assert all(refs[p] == used.count(p) for p in range(n_pages))
        assert sorted(set(used)) == list(range(len(set(used))))
        kh = k.cpu()
        for b in range(B):
            assert lens[b] == held[b].shape[0]
            own = table[b, :n_pages_of(lens[b], page)].long()
            assert (table[b, len(own):] == -1).all()
            assert torch.equal(kh[own].reshape(-1, Hkv, 128)[:lens[b]], held[b]), (i, b)


def test_calls_on_two_streams_do_not_meet():
    rng = np.random.default_rng(3)
    ms = [filled(rng, 64, 33, 2000, 64) for _ in range(2)]
    tables = [to_device(m, torch) for m in ms]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    up = [rng.integers(-1, 64, 64) for _ in range(2)]
    ups = [_i32(u) for u in up]
    torch.cuda.synchronize()
    say("two streams")
    for _ in range(3):
        for s, t, u in zip(streams, tables, ups):
            api.pages_fork(t, u, stream=s)
    torch.cuda.synchronize()
    for m, t, u in zip(ms, tables, up):
        for _ in range(3):
            m.fork(u.tolist())
        same(t, m)


def test_more_rows_than_a_launch_has_waves():
    """2^26 rows and a few, of which the last three have a place."""
    n = (1 << 26) + 5
    k, v = (torch.empty((1, n, 1, 128), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    x = torch.randn((2, 3, 1, 128), device="cuda").to(torch.bfloat16)
    k[0, n - 3:], v[0, n - 3:] = x[0], x[1]
    kc, vc = (torch.zeros((1, 8, 1, 128), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    say("append", n)
    api.cache_append(kc, vc, k, v, _i32([3 - n]))
    torch.cuda.synchronize()
    for c, rows in ((kc, x[0]), (vc, x[1])):
        assert torch.equal(c[0, :3], rows) and (c[0, 3:] == 0).all()
    del k, v
    torch.cuda.empty_cache()


def test_a_table_row_of_more_entries_than_a_launch_has_threads():
    cols = (1 << 29) + 9
    table = torch.full((1, cols), -1, dtype=torch.int32, device="cuda")
    table[0, :2], table[0, cols - 2:] = _i32([3, 1]), _i32([0, 2])
    pages = api.PageTable(_i32([cols]), _i32([1, 1, 1, 1, 0]), table, 1)
    say("fork", cols)
    api.pages_fork(pages, _i32([-1]))
    torch.cuda.synchronize()
    assert pages.refs.tolist() == [0] * 5 and pages.lens.tolist() == [0]
    assert (table[0, :2] == -1).all() and (table[0, cols - 2:] == -1).all()
    del pages, table
    torch.cuda.empty_cache()
