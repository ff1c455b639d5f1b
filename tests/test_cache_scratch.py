"""Scratch that attention over the cache asks for, and what it refuses for its size (no GPU needed: the pointers are no memory)."""
import ctypes

import pytest

from test_decode_refusals import P, _attend, _handle

ESHAPE = 3


@pytest.fixture()
def tw():
    import paper_2511_03983_amd as tw
    return tw


def _floats(tw, h, T, Hs, max_len, n_seqs=1, page=16):
    """(status, floats) of T rows of Hs heads over max_len tokens, through a table of n_seqs sequences."""
    n, room = ctypes.c_size_t(7), -(-max_len // page)
    pages = tw.binding.PagesC(P, room, n_seqs, room, room, page)
    return tw.lib.twist_cache_attention_floats(h, ctypes.byref(pages), T, Hs, max_len, ctypes.byref(n)), n.value


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_fill_the_gpu_uncut(tw, dtype):
    """Thousands of rows are workgroups enough: no part of a sequence is left to be joined, and none of it asks for memory."""
    h = _handle(tw, d_head=128, dtype=dtype)
    for T, Hs, top in [(4096, 32, 4096), (4096, 8, 4096), (2000, 16, 8000), (8192, 2, 8192), (4096, 32, 16384), (2000, 16, 16384), (1000, 8, 7000), (16384, 32, 16384)]:
        for n_seqs in (1, 2, 16):
            assert _floats(tw, h, T, Hs, top, n_seqs) == (0, 0), (T, Hs, top, n_seqs)
    assert _floats(tw, h, 4096, 32, 4096, 256) == (0, 0)              # (a table of more sequences than the prompt's)
    # few rows of long sequences are cut, whatever their form
    for T, n_seqs in ((1, 1), (8, 1), (16, 16), (180, 36)):
        status, n = _floats(tw, h, T, 3, 16384, n_seqs)
        assert status == 0 and n >= T * 3 * 2 * 130, (T, n_seqs)
    tw.lib.twist_destroy(h)


def test_long_prompts_are_refused_for_the_launch_that_they_get_alone(tw):
    """A launch has less than 2^22 workgroups.  Tiles take 16 or 32 rows each: what a workgroup a row would pass, they do not."""
    h = _handle(tw, d_head=128)
    for T, Hs, top, page in [(16384, 32, 16384, 16), (8192, 32, 32768, 16), (65536, 32, 131072, 16), (16384, 32, 16384, 1), (100000, 40, 131072, 16)]:
        status, n = _floats(tw, h, T, Hs, top, page=page)
        assert status == 0, (T, Hs, top, page)
        assert n == 0 or top > 2047 * page                            # (a part lies on 2048 pages at most)
    # without a list of sequences every row has a workgroup of its own
    pages = ctypes.byref(tw.binding.PagesC(P, 16384, 1, 16384, 16384, 1))
    assert _attend(tw, h, pages, T=16384, Hs=32, stride=32 * 128, ldq=32 * 128, ldo=32 * 128, max_len=16384, floats=2 ** 40) == ESHAPE
    assert b"too many" in tw.lib.twist_last_error(h)
    assert _floats(tw, h, 131071, 32, 2 ** 20, page=1)[0] == ESHAPE
    tw.lib.twist_destroy(h)
    h = _handle(tw, d_head=36)                                         # rows of 72 bytes: no tiles
    assert _floats(tw, h, 16384, 32, 16384, page=1) == (ESHAPE, 7)
    tw.lib.twist_destroy(h)
