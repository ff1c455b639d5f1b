"""What the entry points behind a model's logits refuse, before any device work (no GPU needed: the pointers are no memory)."""
import ctypes

import pytest
import torch

import synth_inputs as si

P = 4096            # stands for a device pointer
EINVAL, ESHAPE = 1, 3


@pytest.fixture()
def tw():
    import paper_2511_03983_amd as tw
    return tw


def _handle(tw, vocab=100, dtype="bf16"):
    h = ctypes.c_void_p()
    cfg = si.ModelCfg(arch="llama", d_model=64, n_heads=2, d_head=64, d_ff=64, vocab=vocab, rope=True, act="swiglu", norm="rms", has_bias=False, tied_head=False, dtype=dtype)
    assert tw.lib.twist_create(ctypes.byref(tw.desc_from_cfg(cfg)), None, ctypes.byref(h)) == 0
    return h


def _refused(tw, h, who, call, cases):
    for kw, status in cases:
        assert call(tw, h, **kw) == status, kw
        assert who in tw.lib.twist_last_error(h), kw
    assert call(tw, None) == EINVAL
    for vocab in (0, 2 ** 20):
        other = _handle(tw, vocab)
        assert call(tw, other, ld=2 ** 20) == ESHAPE
        tw.lib.twist_destroy(other)
    tw.lib.twist_destroy(h)


ROWS = [(dict(logits=None), EINVAL), (dict(T=0), EINVAL), (dict(T=-3), EINVAL), (dict(T=2 ** 22), ESHAPE), (dict(ld=99), ESHAPE), (dict(ld=0), ESHAPE), (dict(ld=-100), ESHAPE)]


def _draw(tw, h, logits=P, ld=100, T=4, uniform=P, tokens=P):
    return tw.lib.twist_draw_raw(h, logits, ld, 0, T, uniform, None, tokens, None, None)


def test_draw_refusals(tw):
    _refused(tw, _handle(tw), b"twist_draw_raw", _draw, ROWS + [(dict(uniform=None), EINVAL), (dict(tokens=None), EINVAL)])


def _top(tw, h, logits=P, ld=100, T=4, k=5, temperature=1.0, ids=P, values=P, ldk=5):
    return tw.lib.twist_top_logits_raw(h, logits, ld, 0, T, k, temperature, ids, values, ldk, None)


def test_top_logits_refusals(tw):
    _refused(tw, _handle(tw), b"twist_top_logits_raw", _top,
             ROWS + [(dict(ids=None), EINVAL), (dict(values=None), EINVAL), (dict(k=0), ESHAPE), (dict(k=-1), ESHAPE), (dict(k=1025, ldk=1025), ESHAPE), (dict(ldk=4), ESHAPE),
                     (dict(temperature=0.0), EINVAL), (dict(temperature=-1.0), EINVAL), (dict(temperature=float("nan")), EINVAL), (dict(temperature=float("inf")), EINVAL)])


def _distill(tw, h, logits=P, ld=100, T=4, targets=P, grad=2 * P, ldg=100, rowloss=P, loss=P, ids=P, values=P, lde=5, k=5, temperature=1.0, weight=0.5, teacher=True):
    t = tw.binding.TeacherC(ids, values, None, lde, k, temperature, weight)
    return tw.lib.twist_distill_raw(h, logits, ld, targets, T, ctypes.byref(t) if teacher else None, grad, ldg, rowloss, loss)


TEACHERS = [(dict(ids=None), EINVAL), (dict(values=None), EINVAL), (dict(k=0), ESHAPE), (dict(k=1025, lde=1025), ESHAPE), (dict(lde=4), ESHAPE), (dict(temperature=0.0), EINVAL),
            (dict(temperature=float("nan")), EINVAL), (dict(temperature=float("inf")), EINVAL), (dict(weight=-0.1), EINVAL), (dict(weight=1.1), EINVAL), (dict(weight=float("nan")), EINVAL)]


def test_distill_refusals(tw):
    _refused(tw, _handle(tw), b"twist_distill_raw", _distill,
             ROWS + TEACHERS + [(dict(teacher=False), EINVAL), (dict(grad=None), EINVAL), (dict(rowloss=None), EINVAL), (dict(loss=None), EINVAL), (dict(targets=None), EINVAL),
                                (dict(ldg=99), ESHAPE), (dict(grad=P, ldg=104), EINVAL)])


def test_holders_refuse_what_is_not_on_a_gpu_or_not_of_its_type(tw):
    z, i = torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    for kw in (dict(temperature=z), dict(top_k=i), dict(top_p=z), dict(min_p=z)):
        with pytest.raises(tw.TwistError):
            tw.DrawRules(**kw)
    with pytest.raises(tw.TwistError):
        tw.Teacher(i.view(1, 3), z.view(1, 3))
    assert tw.DrawRules().T is None


class _NoGPU:
    """What the binding looks at of a context, with no memory to be had."""

    def __new__(cls, tw, vocab=8):
        class Bare(tw.Context):
            def __init__(self):
                self.gpu, self.device, self.torch_dtype, self.desc = -1, "cpu", torch.bfloat16, tw.ModelDesc(vocab=vocab)

            def _empty(self, *a, **kw):
                raise AssertionError("asks for memory")

            def _call(self, *a):
                raise AssertionError("calls the library")
        return Bare()


@pytest.mark.parametrize("T", [2 ** 31, 2 ** 32 + 3])
def test_rows_that_the_library_counts_otherwise_are_refused(tw, T):
    """Its numbers of rows have 32 bits: of 2^32 + 3 rows it would see 3."""
    ctx = _NoGPU(tw)
    x = torch.empty((T, 8), dtype=torch.bfloat16, device="meta")       # (no memory)
    for call in (lambda: ctx._rows(x, T, 8, "logits", torch.bfloat16), lambda: ctx._logits(x), lambda: ctx._batch(torch.empty((T, 8), dtype=torch.int32, device="meta"), "inputs"),
                 lambda: ctx._batch(torch.empty((8, T), dtype=torch.int32, device="meta"), "inputs")):
        with pytest.raises(tw.TwistError, match="logits|inputs"):
            call()
    assert ctx._rows(x[:5], 5, 8, "logits", torch.bfloat16) == 8


@pytest.mark.parametrize("k", [-2 ** 32 + 5, -1, 0, 1025, 2 ** 31, 2 ** 32 + 5])
def test_lists_of_a_length_that_there_is_not_ask_for_no_memory(tw, k):
    ctx = _NoGPU(tw)
    x, i = torch.empty((4, 8), dtype=torch.bfloat16, device="meta"), torch.empty((4, 8), dtype=torch.int32, device="meta")
    given = torch.empty((4, 5), dtype=torch.int32, device="meta")
    for call in (lambda: ctx.twist_top_logits_raw(x, k), lambda: ctx.twist_top_logits_raw(x, k, ids=given), lambda: ctx.twist_subnet_top_logits(None, i, k, None)):
        with pytest.raises(tw.TwistError, match="entries"):
            call()
