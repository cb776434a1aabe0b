"""Calls of the 8-bit entry points whose sizes multiply past 64 bits are refused, on the CPU."""
import ctypes

import pytest

from paper_2607_07740_amd import api
from test_cache8_model import A, A2, ALL, DECODE, _cache, _entries, _refused, _select

BIG = 2 ** 30


def test_pools_whose_blocks_multiply_to_2_to_the_64():
    c = _cache(n_pages=BIG, Hkv=BIG, page_size=16 * 64)  # 2^64 blocks: none in 64 bits
    _refused(_entries(c, Hq=BIG, max_pages=1), ALL, api.JL_ERR_UNSUPPORTED)
    one = api.lib().jl_cache8_append(ctypes.byref(c), A, 1, A, A, A2, None, 1, 1, None)
    assert one == api.JL_ERR_UNSUPPORTED


@pytest.mark.parametrize("max_pages,names", [(10, DECODE), (16, ("scores", "rope_scores"))])
def test_batches_whose_steps_multiply_past_64_bits(max_pages, names):
    c = _cache(n_pages=1, Hkv=BIG, page_size=64)
    # 2^30 sequences of 2^30 heads of 16 steps: a decode counts 6 more for each head
    _refused(_entries(c, max_pages=max_pages, B=BIG, Hq=BIG, n_select=max_pages), names,
             api.JL_ERR_INVALID_ARG)


def test_lists_that_multiply_past_64_bits():
    assert _select(B=BIG, Hkv=BIG, n_blocks=16, n_select=16) == api.JL_ERR_INVALID_ARG
    assert _select(B=BIG, Hkv=BIG, n_blocks=3, n_select=16) == api.JL_ERR_INVALID_ARG
