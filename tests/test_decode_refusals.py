"""What the entry points of token generation refuse, before any device work (no GPU needed: the pointers are no memory)."""
import ctypes

import pytest

import synth_inputs as si

P = 4096            # stands for a device pointer
EINVAL, ESHAPE = 1, 3


@pytest.fixture()
def tw():
    import paper_2511_03983_amd as tw
    return tw


def _handle(tw, **kw):
    h = ctypes.c_void_p()
    cfg = si.ModelCfg(arch="llama", **{**dict(d_model=64, n_heads=2, d_head=64, d_ff=64, vocab=100, rope=True, act="swiglu", norm="rms", has_bias=False, tied_head=False,
                                              dtype="bf16"), **kw})
    assert tw.lib.twist_create(ctypes.byref(tw.desc_from_cfg(cfg)), None, ctypes.byref(h)) == 0
    return h


def _pages(tw, **kw):
    c = tw.binding.PagesC(P, 8, 2, 8, 16, 16)
    for k, v in kw.items():
        setattr(c, k, v)
    return ctypes.byref(c)


BAD_PAGES = [(dict(table=None), EINVAL), (dict(n_seqs=0), EINVAL), (dict(max_pages=0), EINVAL), (dict(n_pages=0), EINVAL), (dict(n_pages=-1), EINVAL),
             (dict(ld_table=7), ESHAPE), (dict(page_tokens=0), ESHAPE), (dict(page_tokens=-16), ESHAPE), (dict(page_tokens=24), ESHAPE),
             (dict(page_tokens=8192), ESHAPE), (dict(page_tokens=4096, max_pages=2 ** 20, ld_table=2 ** 20), ESHAPE)]
S = 2 * 64 * 16     # elements of a page of two heads


def _append(tw, h, pages, k=P, v=P, stride=S, qkv=P, ld=3 * 128, T=4, Hs=2, lens=P, q_out=P, ldq=128):
    return tw.lib.twist_cache_append_raw(h, pages, k, v, stride, qkv, ld, T, Hs, None, lens, q_out, ldq)


def _attend(tw, h, pages, k=P, v=P, stride=S, q=P, ldq=128, T=4, Hs=2, lens=P, max_len=64, o=P, ldo=128, scratch=P, floats=2 ** 30):
    return tw.lib.twist_cache_attention_raw(h, pages, k, v, stride, q, ldq, T, Hs, None, lens, max_len, o, ldo, P, scratch, floats)


def test_append_refusals(tw):
    h = _handle(tw)
    for kw, status in BAD_PAGES:
        assert _append(tw, h, _pages(tw, **kw)) == status, kw
        assert b"twist_cache_append_raw" in tw.lib.twist_last_error(h)
    for kw, status in [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(qkv=None), EINVAL), (dict(lens=None), EINVAL), (dict(T=0), EINVAL), (dict(T=-1), EINVAL),
                       (dict(Hs=0), EINVAL), (dict(stride=S - 1), ESHAPE), (dict(ld=383), ESHAPE), (dict(ldq=127), ESHAPE), (dict(T=2 ** 24), ESHAPE), (dict(T=2 ** 21), ESHAPE), (dict(stride=2 ** 60), ESHAPE)]:
        assert _append(tw, h, _pages(tw), **kw) == status, kw
    assert _append(tw, h, None) == EINVAL
    assert tw.lib.twist_cache_append_raw(None, _pages(tw), P, P, S, P, 384, 4, 2, None, P, P, 128) == EINVAL
    tw.lib.twist_destroy(h)
    h = _handle(tw, d_head=258)
    assert _append(tw, h, _pages(tw), stride=2 ** 20, ld=2 ** 12, ldq=2 ** 12) == ESHAPE and b"d_head" in tw.lib.twist_last_error(h)
    tw.lib.twist_destroy(h)


def test_attention_refusals(tw):
    h = _handle(tw)
    n = ctypes.c_size_t(77)
    for kw, status in BAD_PAGES:
        assert _attend(tw, h, _pages(tw, **kw)) == status, kw
        assert tw.lib.twist_cache_attention_floats(h, _pages(tw, **kw), 4, 2, 64, ctypes.byref(n)) == status, kw
    for kw, status in [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(q=None), EINVAL), (dict(lens=None), EINVAL), (dict(o=None), EINVAL), (dict(T=0), EINVAL),
                       (dict(Hs=-2), EINVAL), (dict(max_len=0), EINVAL), (dict(max_len=-5), EINVAL), (dict(stride=S - 1), ESHAPE), (dict(ldq=127), ESHAPE),
                       (dict(ldo=127), ESHAPE), (dict(Hs=2 ** 20, stride=2 ** 50, ldq=2 ** 30, ldo=2 ** 30), ESHAPE), (dict(stride=2 ** 62), ESHAPE),
                       (dict(scratch=P + 4), ESHAPE)]:
        assert _attend(tw, h, _pages(tw), **kw) == status, kw
    assert _attend(tw, h, None) == EINVAL
    assert tw.lib.twist_cache_attention_floats(h, _pages(tw, max_pages=2 ** 10, ld_table=2 ** 10), 1, 2, 2 ** 14, ctypes.byref(n)) == 0 and n.value not in (0, 77)
    need = n.value
    n.value = 77
    long = _pages(tw, max_pages=2 ** 10, ld_table=2 ** 10)             # a long sequence is cut: scratch
    assert _attend(tw, h, long, T=1, max_len=2 ** 14, scratch=None) == EINVAL
    assert _attend(tw, h, long, T=1, max_len=2 ** 14, floats=need - 1) == ESHAPE
    for args in ((h, _pages(tw), 0, 2, 64), (h, _pages(tw), 4, 0, 64), (h, _pages(tw), 4, 2, 0), (None, _pages(tw), 4, 2, 64), (h, None, 4, 2, 64)):
        assert tw.lib.twist_cache_attention_floats(*args, ctypes.byref(n)) == EINVAL
    assert tw.lib.twist_cache_attention_floats(h, _pages(tw), 4, 2, 64, None) == EINVAL
    # more parts than can be joined: single-token pages, eight million of them
    long = _pages(tw, page_tokens=1, max_pages=2 ** 23, ld_table=2 ** 23)
    assert tw.lib.twist_cache_attention_floats(h, long, 1, 2, 2 ** 23, ctypes.byref(n)) == ESHAPE
    assert n.value == 77                                               # an error leaves the out-parameters alone
    tw.lib.twist_destroy(h)


@pytest.mark.parametrize("page", [1, 64, 256, 4096])
def test_a_part_of_a_sequence_lies_on_2048_pages_at_most(tw, page):
    """Wherever it begins: the kernels keep the places of that many.  Narrow heads have the longest parts; lengths at which a part is no whole number of pages."""
    n = ctypes.c_size_t()
    for kw in (dict(d_head=1, rope=False), dict(d_head=2), dict(d_head=2, dtype="f32"), dict(d_head=64)):
        h = _handle(tw, **kw)
        for top in [1048448, 2 ** 20 - 128] + [2 ** e - 64 * i for e in range(17, 31) for i in (0, 1, 3, 1027)] + [1024 * (2047 * page + 64 * i) for i in (-1, 0, 1, page // 64)]:
            pages = -(-top // page)
            if not 0 < pages * page <= 2 ** 30:
                continue
            for units in (1, 2, 64, 128, 300):
                if tw.lib.twist_cache_attention_floats(h, _pages(tw, page_tokens=page, max_pages=pages, ld_table=pages, n_pages=pages), units, 1, top, ctypes.byref(n)) == 0:
                    parts = max(1, n.value // (units * (kw["d_head"] + 2)))
                    assert -(-top // parts) <= 2047 * page, (kw, top, units, parts)
        tw.lib.twist_destroy(h)


def test_logits_refusals(tw):
    h = _handle(tw)
    good = dict(history=P, ld_history=8, hist_cap=8, bias_ids=P, bias_values=P, ld_bias=4, bias_cap=4, allowed=P, ld_allowed=4)

    def call(h=h, logits=P, ld=100, T=2, out=2 * P, ldo=100, **kw):
        c = tw.binding.LogitRulesC()
        for k, v in {**good, **kw}.items():
            setattr(c, k, v)
        return tw.lib.twist_logits_raw(h, logits, ld, T, ctypes.byref(c), out, ldo)

    for kw, status in [(dict(logits=None), EINVAL), (dict(out=None), EINVAL), (dict(T=0), EINVAL), (dict(T=65536), ESHAPE), (dict(ld=99), ESHAPE), (dict(ldo=99), ESHAPE),
                       (dict(ld_history=7), ESHAPE), (dict(hist_cap=-1), ESHAPE), (dict(bias_values=None), EINVAL), (dict(ld_bias=3), ESHAPE), (dict(bias_cap=-1), ESHAPE),
                       (dict(ld_allowed=3), ESHAPE), (dict(out=P), EINVAL), (dict(hist_cap=2 ** 30, ld_history=2 ** 30), ESHAPE), (dict(bias_cap=2 ** 30, ld_bias=2 ** 30), ESHAPE)]:
        assert call(**kw) == status, kw
        assert b"twist_logits_raw" in tw.lib.twist_last_error(h)
    assert tw.lib.twist_logits_raw(h, P, 100, 2, None, 2 * P, 100) == EINVAL
    assert tw.lib.twist_logits_raw(None, P, 100, 2, None, 2 * P, 100) == EINVAL
    tw.lib.twist_destroy(h)
    h = _handle(tw, dtype="f32")
    assert call(h=h, out=P, ldo=104) == EINVAL                         # in place only with the same rows
    tw.lib.twist_destroy(h)
    h = _handle(tw, vocab=0)
    assert call(h=h) == ESHAPE
    tw.lib.twist_destroy(h)


def test_holders_refuse_what_is_not_on_a_gpu(tw):
    import torch
    with pytest.raises(tw.TwistError):
        tw.Pages(torch.zeros((2, 2), dtype=torch.int32), 4, 16)
    with pytest.raises(tw.TwistError):
        tw.LogitRules(history=torch.zeros((2, 2), dtype=torch.int32))
    with pytest.raises(tw.TwistError):
        tw.PagedCache(torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 32), torch.zeros((2, 2), dtype=torch.int32))
