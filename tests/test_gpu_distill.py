"""The loss against a teacher's top logits and its gradient, against the formula in 64 bits, in which it is also compared with differences and with the cross-entropy.

Tolerances, with u = 2^-24 and r = u (2 ln V + 4 + V / 256 + 16) what a sum of exponentials in 32 bits is off, relative to itself (the rounding of an exponent d against the largest
and of its division, u 2 E[d], E[d] <= ln V; two steps of the exponential; the additions in one chain):
  rowloss   a rounding; of the cross-entropy r; of the teacher's part r |P - Q|, the derivative by the logarithm of the others' sum, and beside them 64-bit sums: 1e-13 of its terms;
  grad      a rounding of the type; outside the list its share of the others (r, and u (2 d + 4) of its own exponential) times |P - Q|, which is off by r P (1 - P); in it r of the probability;
            of the cross-entropy's part likewise; every sum of two parts a rounding of each.
"""
import math

import numpy as np
import pytest
import torch

import synth_inputs as si
from test_gpu_draw import U, _ctx, _gen, _logits

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _lse(a):
    m = np.max(a) if len(a) else -np.inf
    return m if not np.isfinite(m) else m + math.log(np.exp(a - m).sum())


def _want(x, y, ids, values, rest, tau, weight):
    """(loss, its error, gradient, its error) of one row, in 64 bits, by sets of columns."""
    V = len(x)
    r = U * (2 * math.log(V) + 4 + V / 256 + 16)
    loss = off = 0.0
    g, e = np.zeros(V), np.zeros(V)
    on = (ids >= 0) & (ids < V)
    theirs = {}
    for c, v in zip(ids[on], values[on]):
        theirs.setdefault(int(c), []).append(v / tau)
    t = np.array([_lse(np.array(v)) for v in theirs.values()] + [-np.inf if rest is None else rest])
    if weight > 0 and t.max() > -np.inf:
        cols = np.array(list(theirs), dtype=int)
        out = np.ones(V, bool)
        out[cols] = False
        z = x / tau
        mine = np.append(z[cols], _lse(z[out])) - _lse(z)
        log_q = t - _lse(t)
        q, p = np.exp(log_q), np.exp(mine)
        P, Q = p[-1], q[-1]
        more = P - Q if Q < 0.5 else q[:-1].sum() - p[:-1].sum()
        some = q > 0
        loss += weight * tau ** 2 * (q[some] * (log_q[some] - mine[some])).sum()
        off += weight * tau ** 2 * (r * abs(more) + 1e-13 * (q[some] * (np.abs(log_q[some]) + np.abs(mine[some]) + np.abs(x).max(initial=0, where=np.isfinite(x)) / tau + 1)).sum())
        if out.any() and np.isfinite(z[out].max()):
            d = z[out].max() - z[out]
            share = np.exp(z[out] - _lse(z[out]))
            g[out] += weight * tau * share * more
            e[out] += weight * tau * share * (abs(more) * (r + U * (4 + 2 * np.where(share > 0, d, 0.0))) + r * P * max(1 - P, 0.0) + U * abs(more))
        g[cols] += weight * tau * (p[:-1] - q[:-1])
        e[cols] += weight * tau * ((r + U) * p[:-1] + U * q[:-1])
    if weight < 1 and 0 <= y < V:
        z = _lse(x)
        p = np.exp(x - z)
        loss += (1 - weight) * (z - x[y])
        off += (1 - weight) * (r + U)
        g += (1 - weight) * p
        e += (1 - weight) * p * (r + U * (5 + 2 * np.where(p > 0, x.max() - x, 0.0)))
        g[y] -= 1 - weight
        e[y] += 2 * U * (1 - weight)
    return loss, off + U * abs(loss), g, e


def _check(ctx, lib, x, y, ids, values, rest, tau=1.0, weight=1.0, rows=None, grad=None):
    T, V = x.shape
    xs = x.double().cpu().numpy()
    teacher = lib.Teacher(ids, values, rest=rest, temperature=tau, weight=weight)
    loss, rowloss, out = ctx.twist_distill_raw(x, y, teacher, grad=grad)
    tau, weight = float(np.float32(tau)), float(np.float32(weight))
    ys = np.full(T, -1) if y is None else y.cpu().numpy()
    i, v, s = ids.cpu().numpy(), values.double().cpu().numpy(), [None] * T if rest is None else rest.double().tolist()
    got, gloss = out.double().cpu().numpy() * T, rowloss.double().cpu().numpy()
    half = U if out.dtype == torch.float32 else 2.0 ** -8
    tiny = T * (2.0 ** -149 if out.dtype == torch.float32 else 2.0 ** -133)   # below the smallest steps of the type nothing is promised
    sums = 0.0
    for t in range(T) if rows is None else rows:
        want, off, g, e = _want(xs[t], ys[t], i[t], v[t], s[t], tau, weight)
        assert gloss[t] == want or abs(gloss[t] - want) <= off, (t, gloss[t], want, off)
        d = np.abs(got[t] - g) - (half * np.abs(g) + (1 + half) * (e + 2 * U * np.abs(g)) + tiny)
        c = int(np.argmax(np.where(np.isnan(d), np.inf, d)))
        assert d[c] <= 0, (t, c, got[t][c], g[c], e[c])
    if np.isfinite(gloss).all():
        assert abs(float(loss) - gloss.mean()) <= U * (T / 256 + 16) * np.abs(gloss).mean()
    return loss, rowloss, out


def _teacher(g, x, k, tau, rest=True, noise=1.5):
    """A teacher's list, made from logits near the student's."""
    z = x.float() + noise * torch.randn(x.shape, generator=g, device="cuda")
    values, at = torch.topk(z, k, dim=1)
    others = torch.logsumexp(z.double().scatter(1, at, -math.inf) / tau, 1).float() if rest else None
    return at.to(torch.int32), values, others


def _targets(g, ids, V):
    T = ids.shape[0]
    return torch.where(torch.rand(T, generator=g, device="cuda") < 0.5, ids[:, 0].long(), torch.randint(0, V, (T,), generator=g, device="cuda")).to(torch.int32)


@pytest.mark.parametrize("V", [1, 2, 9, 130, 1003, 4100, 16391, 32000, 50257, 65537, 131072])
@pytest.mark.parametrize("dtype", list(DT))
def test_distill(lib, dtype, V):
    ctx, g = _ctx(lib, V, dtype), _gen(V)
    for kind in ("model", "flat", "steps"):
        for k, tau, weight, rest in ((1, 1.0, 1.0, True), (8, 2.0, 0.5, True), (64, 4.0, 0.3, False), (200, 0.7, 1.0, True), (1000, 1.0, 0.0, True)):
            T, k = 3, min(k, V)
            x = _logits(g, T, V, kind).to(DT[dtype])
            ids, values, others = _teacher(g, x, k, tau, rest)
            _check(ctx, lib, x, None if weight == 1.0 else _targets(g, ids, V), ids, values, others, tau, weight)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [25, 29, 31, 63, 95, 1023, 8191, 32767, 65535, 65563])
def test_distill_last_columns(lib, dtype, V):
    """A row's last columns in a list, then in none: nothing of a list stays for the next one."""
    ctx, g = _ctx(lib, V, dtype), _gen(V + 7)
    T, k = 4, min(V, 40)
    for _ in range(2):
        x = _logits(g, T, V).to(DT[dtype])
        for ids in (torch.arange(V - k, V), torch.arange(1)):
            ids = ids.to(torch.int32).expand(T, -1).contiguous().cuda()
            values = torch.randn(ids.shape, generator=g, device="cuda")
            _check(ctx, lib, x, _targets(g, ids, V), ids, values, torch.zeros(T, device="cuda"), 2.0, 0.5)


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [7, 1003, 50257, 70000])
def test_distill_lists(lib, dtype, V):
    """Entries that are not there, tokens that are named twice and more often, lists of whole vocabularies, entries of no probability, rows without a teacher, a target or both."""
    ctx, g = _ctx(lib, V, dtype), _gen(V + 1)
    T, k = 8, min(V, 40)
    x = _logits(g, T, V).to(DT[dtype])
    ids, values, rest = _teacher(g, x, k, 2.0)
    y = _targets(g, ids, V)
    holes = torch.where(torch.rand((T, k), generator=g, device="cuda") < 0.4, torch.tensor([-1, V, -2 ** 31, 2 ** 31 - 1], device="cuda")[torch.arange(k, device="cuda") % 4], ids.long()).to(torch.int32)
    twice = ids.clone()
    twice[:, 1::2] = twice[:, ::2][:, : k // 2]
    same = ids[:, :1].expand(T, k).contiguous()
    never = torch.where(torch.rand((T, k), generator=g, device="cuda") < 0.5, -math.inf, values)
    none = ids.clone()
    none[::2] = -1
    gone = rest.clone()
    gone[::2] = -math.inf
    off = y.clone()
    off[::3] = torch.tensor([-1, V, -100], dtype=torch.int32, device="cuda")
    for weight in (1.0, 0.4):
        for i, v, s, yy in ((holes, values, rest, y), (twice, values, rest, y), (same, values, rest, off), (ids, never, None, y), (ids, never, rest, off), (none, values, gone, off),
                            (none, values, None, off), (ids, values, torch.full_like(rest, -math.inf), y), (ids, torch.full_like(values, -math.inf), rest, y),
                            (twice, values, None, off), (torch.full_like(ids, -1), values, None, torch.full_like(y, -1)), (torch.full_like(ids, -1), values, rest, y)):
            _check(ctx, lib, x, yy, i, v, s, 2.0, weight)


@pytest.mark.parametrize("dtype", list(DT))
def test_distill_far_apart(lib, dtype):
    """Students that are sure of what the teacher is not and the other way round: shares of next to nothing on either side; logits that are masked out; nearly equal distributions at a high
    temperature."""
    V, T = 2500, 6
    ctx, g = _ctx(lib, V, dtype), _gen(4)
    base = _logits(g, T, V).to(DT[dtype])
    ids, values, rest = _teacher(g, base, 20, 1.0)
    at = ids.long()
    sure = base.clone().scatter_(1, at, base.gather(1, at) + 300.0)             # of the list
    away = base.clone().scatter_(1, at, base.gather(1, at) - 300.0)             # of anything else
    masked = torch.where(torch.rand((T, V), generator=g, device="cuda") < 0.9, -math.inf, base.float()).to(base.dtype).scatter_(1, at, base.gather(1, at))
    only = torch.full_like(base, -math.inf).scatter_(1, at, base.gather(1, at))  # nothing outside the list
    y = ids[:, 3].clone()
    for x, s in ((sure, rest), (sure, rest - 40), (sure, rest + 40), (away, rest), (away, rest + 300), (away, rest - 300), (masked, rest), (only, None), (only, torch.full_like(rest, -math.inf))):
        for weight in (1.0, 0.5):
            _check(ctx, lib, x, y, ids, values, s, 1.0, weight)
    for tau in (8.0, 50.0):
        ids, values, rest = _teacher(g, base, 2, tau, noise=0.5)
        _check(ctx, lib, base, y, ids, values, rest, tau, 1.0)
    # a token that the student excludes and the teacher does not: an infinite loss, in its own row alone
    x = base.clone()
    x[2, at[2, 0]] = -math.inf
    ids, values, rest = _teacher(g, base, 20, 1.0)
    ids[2, 0] = at[2, 0]
    loss, rowloss, grad = ctx.twist_distill_raw(x, None, lib.Teacher(ids, values, rest=rest))
    assert rowloss[2] == math.inf and torch.isfinite(rowloss[[0, 1, 3, 4, 5]]).all() and loss == math.inf and torch.isfinite(grad.float()).all()


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("V", [1003, 70003])
def test_distill_values_and_temperatures_near_their_ends(lib, dtype, V):
    """Logits of the type's lowest value on either side, and values that fp32 does not hold once they are divided by the temperature: a teacher all the same.  An exponential below 2^-126, the least
    that the instruction forms, counts as nothing: with a temperature of at most 1 that is 2^-126 of a row's gradient."""
    ctx, g = _ctx(lib, V, dtype), _gen(V + 19)
    T, k = 6, 20
    low = torch.finfo(DT[dtype]).min
    x = _logits(g, T, V).to(DT[dtype])
    ids, values, rest = _teacher(g, x, k, 1.0)
    y = _targets(g, ids, V)
    masked = torch.where(torch.rand((T, V), generator=g, device="cuda") < 0.5, low, x.float()).to(x.dtype).scatter_(1, ids.long(), x.gather(1, ids.long()))
    masked.scatter_(1, y.long()[:, None], x.gather(1, y.long()[:, None]))
    some = torch.where(torch.rand((T, k), generator=g, device="cuda") < 0.5, low, values)
    some[::2] = low                                                    # (rows of nothing else: all as probable)
    high = 1e38 * (1.0 + torch.randint(0, 3, (T, k), generator=g, device="cuda") * 1e-3)
    half, tiny = (U, 2.0 ** -149) if dtype == "f32" else (2.0 ** -8, 2.0 ** -133)
    for xx, v, s, tau, weight in [(*c, w) for w in (1.0, 0.5) for c in (
            (x, some, None, 0.5), (x, some, None, 0.01), (x, some, rest, 0.5), (masked, values, rest, 1.0), (masked, some, None, 0.5), (x, high, None, 0.1), (x, -high, None, 0.1),
            (x, high, torch.full_like(rest, 3e38), 0.1), (x, values, None, 1e-30), (masked, some, None, 1e-30))] + [(x, values, None, 1e-40, 0.5)]:
        loss, rowloss, grad = ctx.twist_distill_raw(xx, y, lib.Teacher(ids, v, rest=s, temperature=tau, weight=weight))
        tau = float(np.float32(tau))
        for t in range(T):
            # the same teacher with its largest value taken off the others, in 64 bits: of numbers of 1e38 and more their log-sum-exp would leave nothing of the logarithms
            theirs = v[t].double().cpu().numpy()
            m = theirs.max()
            want, off, e, err = _want(xx[t].double().cpu().numpy(), int(y[t]), ids[t].cpu().numpy(), theirs - m, None if s is None else float(s[t]) - m / tau, tau, weight)
            got = grad[t].double().cpu().numpy() * T
            assert abs(float(rowloss[t]) - want) <= off + 2.0 ** -149, (t, tau, weight, float(rowloss[t]), want, off)
            over = np.abs(got - e) - (half * np.abs(e) + (1 + half) * (err + 2 * U * np.abs(e)) + T * tiny + 2.0 ** -126)
            c = int(np.argmax(np.where(np.isnan(over), np.inf, over)))
            assert over[c] <= 0, (t, tau, weight, c, got[c], e[c], err[c])
        assert torch.isfinite(loss)


@pytest.mark.parametrize("dtype", list(DT))
def test_distill_places(lib, dtype):
    """Rows of any stride from any element on, the gradient in other memory or in the logits' place; nothing else is written."""
    for V, pad, first, gpad in ((1003, 0, 1, 0), (1003, 5, 0, 0), (4100, 4, 3, 12), (50257, 7, 0, 0), (50257, 0, 0, 7), (70003, 1, 5, 1)):
        ctx, g = _ctx(lib, V, dtype), _gen(V + pad)
        T, k = 4, 12
        whole = torch.full((T * (V + pad) + first + 3,), 3.0, dtype=DT[dtype], device="cuda")
        x = whole[first: first + T * (V + pad)].view(T, V + pad)[:, :V]
        x.copy_(_logits(g, T, V))
        before = whole.clone()
        ids, values, rest = _teacher(g, x, k, 2.0)
        wide_ids, wide_values = torch.full((T, k + 3), 5, dtype=torch.int32, device="cuda"), torch.full((T, k + 3), 50.0, device="cuda")
        wide_ids[:, 2: 2 + k], wide_values[:, 2: 2 + k] = ids, values
        y = _targets(g, ids, V)
        out = torch.full((T, V + gpad), 9.0, dtype=DT[dtype], device="cuda")
        _check(ctx, lib, x, y, wide_ids[:, 2: 2 + k], wide_values[:, 2: 2 + k], rest, 2.0, 0.5, grad=out[:, :V])
        assert (whole == before).all() and (out[:, V:] == 9.0).all()
        assert _check(ctx, lib, x, y, ids, values, rest, 2.0, 0.5, grad=x)[2] is x
        whole[first: first + T * (V + pad)].view(T, V + pad)[:, :V] = before[first: first + T * (V + pad)].view(T, V + pad)[:, :V]
        assert (whole == before).all()


def test_distill_gradient_against_differences(lib):
    """Central differences of the row losses, which are 32 bits: h = 0.02 leaves h^2 / 6 of the third derivative (at most 1 for a softmax, (1 / tau)^3 tau^2 with tau >= 1) and two roundings of a
    loss below 16 (2^-21 each with what the sums are off) over 2 h."""
    V, T, k, h = 33, 4, 6, 0.02
    ctx, g = _ctx(lib, V), _gen(6)
    x = torch.randn((T, V), generator=g, device="cuda")
    ids, values, rest = _teacher(g, x, k, 1.5)
    y = _targets(g, ids, V)
    teacher = lib.Teacher(ids, values, rest=rest, temperature=1.5, weight=0.6)
    grad = ctx.twist_distill_raw(x, y, teacher)[2].double() * T
    for c in range(V):
        up, down = x.clone(), x.clone()
        up[:, c] += h
        down[:, c] -= h
        step = (up[:, c].double() - down[:, c].double())
        a, b = (ctx.twist_distill_raw(z, y, teacher)[1].double() for z in (up, down))
        assert (a.max() < 16) and ((a - b) / step - grad[:, c]).abs().max() <= h * h / 6 + 2 * 2.0 ** -21 / (2 * h)


@pytest.mark.parametrize("dtype", list(DT))
def test_distill_is_the_cross_entropy_where_the_teacher_names_the_target(lib, dtype):
    """A list of one token that is all of the teacher's distribution, at temperature 1: the loss of twist_ce_raw, whose sums are as exact."""
    V, T = 1003, 50
    ctx, g = _ctx(lib, V, dtype), _gen(8)
    x = _logits(g, T, V).to(DT[dtype])
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    padded = torch.full((T, 1008), 7.0, dtype=DT[dtype], device="cuda")
    padded[:, :V] = x
    _, ce = ctx.twist_ce_raw(padded, y)
    _, rowloss, grad = _check(ctx, lib, x, None, y.view(T, 1).clone(), torch.zeros((T, 1), device="cuda"), None)
    r = U * (2 * math.log(V) + 4 + V / 256 + 16)
    assert ((rowloss - ce).abs() <= 2 * (r + U * ce.abs())).all()
    half = U if dtype == "f32" else 2.0 ** -8
    assert ((grad.float() - padded[:, :V].float()).abs() <= 2 * (half + r + 40 * U) * (grad.float().abs() + 2 * U / T)).all()


def test_distill_many_rows(lib):
    V, T = 1003, 3000
    ctx, g = _ctx(lib, V, "bf16"), _gen(2)
    x = _logits(g, T, V).bfloat16()
    ids, values, rest = _teacher(g, x, 9, 1.0)
    _check(ctx, lib, x, _targets(g, ids, V), ids, values, rest, 1.0, 0.5, rows=range(0, T, 61))


def test_distill_refuses_what_does_not_fit(lib):
    V, T, k = 100, 4, 5
    ctx = _ctx(lib, V, "bf16")
    x = torch.zeros((T, V), dtype=torch.bfloat16, device="cuda")
    y, ids, values, rest = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros((T, k), dtype=torch.int32, device="cuda"), torch.zeros((T, k), device="cuda"), torch.zeros(T, device="cuda")
    ok = lib.Teacher(ids, values, rest, weight=0.5)
    for call in (lambda: ctx.twist_distill_raw(x.float(), y, ok), lambda: ctx.twist_distill_raw(x[:, 1:], y, ok), lambda: ctx.twist_distill_raw(x[:3], y[:3], ok),
                 lambda: ctx.twist_distill_raw(x, None, ok), lambda: ctx.twist_distill_raw(x, y.long(), ok), lambda: ctx.twist_distill_raw(x, y[:3], ok),
                 lambda: ctx.twist_distill_raw(x, y, ok, grad=x.float()), lambda: ctx.twist_distill_raw(x, y, ok, grad=x[:, :99]), lambda: lib.Teacher(ids.long(), values),
                 lambda: lib.Teacher(ids, values.double()), lambda: lib.Teacher(ids, values[:, :4]), lambda: lib.Teacher(ids, values.t().contiguous().t()),
                 lambda: lib.Teacher(ids, values, rest[:3]), lambda: lib.Teacher(ids, torch.zeros((T, 8), device="cuda")[:, :k]),
                 lambda: ctx.twist_distill_raw(x, y, lib.Teacher(ids, values, weight=1.5)), lambda: ctx.twist_distill_raw(x, y, lib.Teacher(ids, values, temperature=0.0))):
        with pytest.raises(lib.TwistError):
            call()


@pytest.mark.parametrize("dtype", list(DT))
def test_distill_largest_vocabulary(lib, dtype):
    V, T = 2 ** 20 - 1, 2
    ctx, g = _ctx(lib, V, dtype), _gen(23)
    x = _logits(g, T, V).to(DT[dtype])
    ids, values, rest = _teacher(g, x, 300, 2.0)
    _check(ctx, lib, x, _targets(g, ids, V), ids, values, rest, 2.0, 0.5)


def test_distill_rows_beyond_32_bits(lib):
    """Rows of logits and gradient so far apart that the last begin behind 2^32 elements."""
    V, T, ld = 1003, 5, 2 ** 30 + 8
    ctx, g = _ctx(lib, V, "bf16"), _gen(24)
    x, grad = (torch.empty((T - 1) * ld + V, dtype=torch.bfloat16, device="cuda").as_strided((T, V), (ld, 1)) for _ in range(2))
    x.copy_(_logits(g, T, V))
    ids, values, rest = _teacher(g, x, 30, 2.0)
    _check(ctx, lib, x, _targets(g, ids, V), ids, values, rest, 2.0, 0.5, grad=grad)
