"""The Python side of the 8-bit calls, on the CPU: tensors of host memory, and a library that only
notes which entry point it was given what."""
import pytest

from paper_2607_07740_amd import api

torch = pytest.importorskip("torch")
BF = torch.bfloat16


class Noting:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def entry(*args):
            self.calls.append((name, args))
            return 4096 if name.endswith("_bytes") else api.JL_OK
        return entry

    def launches(self):
        return [c for c in self.calls if not c[0].endswith("_bytes")]


@pytest.fixture
def library(monkeypatch):
    note = Noting()
    monkeypatch.setattr(api, "lib", lambda: note)
    monkeypatch.setattr(api, "_dev", lambda t, *a: t.data_ptr())
    monkeypatch.setattr(api, "_queue", lambda *a: 0)
    return note


def ints(*x):
    return torch.tensor(x, dtype=torch.int32)


def calls(cache, kw=None):
    """Every call on a cache, by name; kw changes arguments of those that have them."""
    rows, q, lens = torch.zeros((2, 3, 2, 128), dtype=BF), torch.zeros((2, 4, 128), dtype=BF), ints(5, 6)
    blocks = torch.zeros((2, 2, 3), dtype=torch.int32)
    kw = kw or {}

    def args(*names, **own):
        return dict(own, **{n: kw[n] for n in names if n in kw})
    return {
        "append": lambda: api.cache8_append(cache, rows, rows, lens),
        "read": lambda: api.cache8_read(cache, **args("n", "start", n=7)),
        "decode": lambda: api.decode8(q, cache, lens, **args("w_pretrained", "w_local")),
        "blocks": lambda: api.decode8_blocks(q, cache, lens, blocks,
                                             **args("w_pretrained", "w_local")),
        "scores": lambda: api.block_scores8(q, cache, lens, **args("w_pretrained")),
    }


def test_a_cache_cannot_be_changed(library):
    cache = api.cache8_alloc(2, 128, 2, device="cpu")
    for name in ("k", "v", "k_scale", "v_scale", "k_mean", "n_pages", "page_size", "Hkv", "head_dim",
                 "device", "index", "other"):
        with pytest.raises(AttributeError):
            setattr(cache, name, None)
    with pytest.raises(AttributeError):
        del cache.k
    assert (cache.n_pages, cache.page_size, cache.Hkv, cache.head_dim) == (2, 128, 2, 128)
    for name, call in calls(cache).items():
        call()
    assert [c[0] for c in library.launches()] == [
        "jl_cache8_append", "jl_cache8_read", "jl_bifocal_decode8", "jl_bifocal_decode8_blocks",
        "jl_bifocal_block_scores8"]


@pytest.mark.parametrize("name", ["k", "v", "k_scale", "v_scale", "k_mean"])
@pytest.mark.parametrize("how", ["resize", "set", "data", "freed"])
def test_a_cache_whose_tensors_moved_is_refused(library, name, how):
    cache = api.cache8_alloc(2, 128, 2, device="cpu")
    t = getattr(cache, name)
    if how == "resize":
        t.resize_((100, *t.shape[1:]))
    elif how == "set":
        t.set_(torch.zeros_like(t))
    elif how == "data":
        t.data = torch.zeros_like(t)
    else:
        t.untyped_storage().resize_(0)
    for call in calls(cache).values():
        with pytest.raises(ValueError, match="moved"):
            call()
    assert library.launches() == []


@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32, 2 ** 32 + 5, 1 << 40, -2 ** 31 - 1])
def test_integers_past_32_bits_are_refused(library, value):
    """The library's are 32 bits: 2^32 + 5 would arrive as 5."""
    cache = api.cache8_alloc(2, 128, 2, device="cpu")
    for names, arg in ((("read",), "n"), (("read",), "start"), (("decode", "blocks"), "w_local"),
                       (("decode", "blocks", "scores"), "w_pretrained")):
        for name in names:
            with pytest.raises(ValueError, match="32 bits"):
                calls(cache, {arg: value})[name]()
    scores, lens = torch.zeros((2, 2, 9)), ints(5, 6)
    for kw in (dict(n_select=value), dict(w_local=value), dict(n_first=value)):
        with pytest.raises(ValueError, match="32 bits"):
            api.select_blocks(scores, lens, **dict(dict(n_select=5, w_local=0), **kw))
    assert library.launches() == []


def test_dimensions_past_32_bits_are_refused(library):
    """Tensors of 2^32 + 5 entries in a dimension, which a card's memory can hold."""
    long = 2 ** 32 + 5
    cache = api.cache8_alloc(2, 128, 2, device="cpu")
    q, lens = torch.zeros((1, 4, 128), dtype=BF), ints(5)
    wide = torch.zeros((1, 1, 1), dtype=torch.int32).expand(1, 2, long)  # takes no memory
    with pytest.raises(ValueError, match="32 bits"):
        api.decode8_blocks(q, cache, lens, wide)
    with pytest.raises(ValueError, match="32 bits"):
        api.decode8(q, cache, lens, block_table=wide[:, 0])
    with pytest.raises(ValueError, match="32 bits"):
        api.select_blocks(torch.zeros(1, 1, 1).expand(1, 2, long), lens, 5, w_local=0)
    assert library.launches() == []


def test_integers_of_32_bits_arrive(library):
    cache = api.cache8_alloc(2, 128, 2, device="cpu")
    calls(cache, dict(w_local=2 ** 31 - 1, w_pretrained=2 ** 31 - 1))["decode"]()
    name, args = library.launches()[0]
    assert name == "jl_bifocal_decode8" and args.count(2 ** 31 - 1) == 2
