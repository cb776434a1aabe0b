"""Rows that are taken back: the caller lowers lens, as after rejected drafts, and the next
pages_reserve frees the pages behind."""
import numpy as np
import pytest

from pages_util import Model, filled, n_pages_of, same, to_device
from parity_util import say
from paper_2607_07740_amd import api

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.tensor(np.asarray(x, np.int32), device="cuda")


def _release(m):
    for b in range(m.B):
        had = n_pages_of(m.lens[b], m.page)
        m.table[b][had:] = [-1] * (m.max_pages - had)
    m.count()


# sequences, entries of a row, pages, tokens of a page: as for the other page calls
@pytest.mark.parametrize("size", [(1, 1, 1, 1), (3, 7, 19, 5), (33, 40, 700, 16), (7, 130, 16384, 64),
                                  (20, 500, 40001, 3), (3, 9000, 30000, 2), (1500, 9, 9000, 4),
                                  (2048, 3, 5000, 64)])
@pytest.mark.parametrize("some", [0.2, 1.0])
def test_reserve_frees_what_lies_behind(size, some):
    rng = np.random.default_rng(int(10 * some) + sum(size))
    B, max_pages, n_pages, page = size
    m = filled(rng, B, max_pages, n_pages, page, share=0.7)
    m.lens = [int(rng.integers(0, x + 1)) if rng.random() < some else x for x in m.lens]
    pages = to_device(m, torch)
    _release(m)
    room = [max_pages * page - x for x in m.lens]
    n_new = [int(min(r, x)) for r, x in zip(room, rng.integers(-1, 2 * page + 1, B))]
    say("taken back", size, some)
    starts, granted, moves, info = api.pages_reserve(pages, _i32(n_new))
    want = m.reserve(n_new)
    assert info.tolist() == want[3]
    assert starts.tolist() == want[0] and granted.tolist() == want[1]
    assert moves.tolist() == [list(x) for x in want[2]] + [[-1, -1]] * (B - len(want[2]))
    same(pages, m)


def test_pages_behind_are_free_in_the_same_call_and_if_it_grants_nothing():
    m = Model(2, 4, 4, 8)
    m.lens, m.table = [9, 8], [[2, 3, 1, -1], [0, -1, -1, -1]]  # the first had 17 to 24 tokens
    m.count()
    pages = to_device(m, torch)
    say("taken back: the pool's last page")
    starts, granted, moves, info = api.pages_reserve(pages, _i32([8, 0]))
    assert info.tolist() == [0, 1, 0, 0] and granted.tolist() == [8, 0]
    assert pages.table.tolist()[0] == [2, 3, 1, -1] and pages.refs.tolist() == [1] * 4
    pages.lens.copy_(_i32([2, 8]))
    starts, granted, moves, info = api.pages_reserve(pages, _i32([1, 24]))
    assert info.tolist() == [0, 0, 1, 0] and granted.tolist() == [0, 0]
    assert pages.table.tolist() == [[2, -1, -1, -1], [0, -1, -1, -1]]
    assert pages.refs.tolist() == [1, 0, 1, 0] and pages.lens.tolist() == [2, 8]


def test_drafts_that_are_rejected_lose_no_page():
    """Eight drafts for every sequence and step, of which some are kept, beside forks, ends and
    compactions, captured and replayed: the counts are those of the table, and what was kept
    reads back."""
    rng = np.random.default_rng(2)
    B, max_pages, n_pages, page, Hkv = 10, 6, 62, 16, 1
    pages = api.pages_alloc(B, max_pages, n_pages, page)
    k = torch.zeros((n_pages, page, Hkv, 128), device="cuda", dtype=torch.bfloat16)
    v = torch.zeros_like(k)
    n_new, parent, kept = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(3))
    rows = torch.zeros((2, B, 8, Hkv, 128), device="cuda", dtype=torch.bfloat16)

    def step():
        api.pages_fork(pages, parent)
        starts, granted, moves, info = api.pages_reserve(pages, n_new)
        api.copy_pages([k, v], moves, info)
        api.cache_append(k, v, rows[0], rows[1], starts, n_new=granted, block_table=pages.table)
        pages.lens.copy_(starts + kept)
        moves, info2 = api.pages_compact(pages)
        api.copy_pages([k, v], moves, info2)
        return info

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        parent.copy_(torch.arange(B))
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        caught = step()
    held = [torch.zeros((0, Hkv, 128), dtype=torch.bfloat16)] * B
    for i in range(60):
        up = np.where(rng.random(B) < 0.15, rng.integers(0, B, B), np.arange(B))
        up[[b for b in range(B) if held[up[b]].shape[0] + 8 > max_pages * page]] = -1
        held = [held[p] if p >= 0 else held[0][:0] for p in up]
        keep = rng.integers(0, 9, B)
        x = torch.randn((2, B, 8, Hkv, 128)).to(torch.bfloat16)
        parent.copy_(torch.from_numpy(up.astype(np.int32)))
        n_new.fill_(8)
        kept.copy_(torch.from_numpy(keep.astype(np.int32)))
        rows.copy_(x)
        say("drafts", i)
        if i % 2:
            graph.replay()
            info = caught
        else:
            info = step()
        # 60 pages hold ten sequences of 6 each
        assert info.tolist()[2:] == [0, 0]
        held = [torch.cat([h, x[0, b, :keep[b]]]) for b, h in enumerate(held)]
        lens, table, refs = pages.lens.tolist(), pages.table.cpu(), pages.refs.tolist()
        used = [p for r in table.tolist() for p in r if p >= 0]
        assert all(refs[p] == used.count(p) for p in range(n_pages))
        kh = k.cpu()
        for b in range(B):
            assert lens[b] == held[b].shape[0]
            own = table[b, :n_pages_of(lens[b], page)].long()
            assert torch.equal(kh[own].reshape(-1, Hkv, 128)[:lens[b]], held[b]), (i, b)
