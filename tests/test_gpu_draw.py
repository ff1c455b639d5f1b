"""Drawing tokens from logits and taking the largest of them, each against the formula in 64 bits.

What is drawn, kept or listed is compared as it is: whole numbers.  Floating results, with u = 2^-24:
  logprobs  a rounding, and the quantum of the probabilities' sums: V 2^-(bits + 1) of the largest, bits of them as the header has it;
  rest      m / tau, the logarithm and their sum: a rounding of each; the sum of exponentials is off, relative to itself, by u times
            2 E[d] (the rounding of an exponent d against the largest, and of its division: E[d] <= ln V, since the entropy of the distribution is
            ln sum + E[d] <= ln V), 4 (two steps of the exponential) and the additions in one chain (V / 256 + 16).
"""
import math

import numpy as np
import pytest
import torch

import synth_inputs as si

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _ctx(lib, V, dtype="f32", stream=None):
    return lib.Context(lib.desc_from_cfg(si.ModelCfg(arch="llama", d_model=64, n_heads=1, d_head=64, d_ff=8, vocab=V, max_seq=1, act="swiglu", norm="rms", has_bias=False,
                                                     tied_head=False, rope=True, dtype=dtype)), stream)


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _order(x):
    """(columns, logits) of a row, largest first, equal ones by column; what holds no number counts as -infinity."""
    x = np.where(np.isnan(x), -np.inf, x)
    at = np.lexsort((np.arange(len(x)), -x))
    return at, x[at]


def _draw_want(x, u, temp=None, k=None, p=None, m=None):
    """(token, logprob, kept) of one row in 64 bits."""
    at, z = _order(x)
    n = int((z > -np.inf).sum())
    if n == 0:
        return -1, -math.inf, 0
    if temp is not None and not temp > 0:
        return int(at[0]), 0.0, 1
    with np.errstate(invalid="ignore"):
        d = np.where(z[:n] == z[0], 0.0, z[:n] - z[0]) / (1.0 if temp is None else temp)
    w = np.exp(np.where(np.isnan(d), -np.inf, d))
    if k is not None and k > 0:
        n = min(n, k)
    if p is not None and p < 1:
        s = np.cumsum(w[:n])
        n = min(n, 1 + int((s[:-1] < p * s[-1]).sum()))
    if m is not None and m > 0:
        n = min(n, int((w[:n] >= min(m, 1.0)).sum()))
    s = np.cumsum(w[:n])
    j = min(int((s <= max(u if u == u else 0.0, 0.0) * s[-1]).sum()), int((w[:n] > 0).sum()) - 1)
    return int(at[j]), float(d[j] - math.log(s[-1])), n


def _check(ctx, lib, x, u, temperature=None, top_k=None, top_p=None, min_p=None, rows=None, **kw):
    T, V = x.shape
    rules = None if all(r is None for r in (temperature, top_k, top_p, min_p)) else lib.DrawRules(temperature, top_k, top_p, min_p)
    tokens, logprobs, kept = ctx.twist_draw_raw(x, u, rules, **kw)
    xs, us = x.double().cpu().numpy(), u.double().tolist()
    of = [None if r is None else r.tolist() for r in (temperature, top_k, top_p, min_p)]
    bits = max(42, min(51, 62 - math.ceil(math.log2(V))))
    for t in range(T) if rows is None else rows:
        token, logprob, n = _draw_want(xs[t], us[t], *(None if r is None else r[t] for r in of))
        got = (int(tokens[t]), int(kept[t]))
        assert got == (token, n), (t, got, (token, n), [None if r is None else r[t] for r in of], us[t])
        lp = float(logprobs[t])
        assert lp == logprob or abs(lp - logprob) <= U * abs(logprob) + V * 2.0 ** -(bits + 1) + 1e-12, (t, lp, logprob)
    return tokens, logprobs, kept


def _logits(g, T, V, kind="model"):
    x = 2.0 * torch.randn((T, V), generator=g, device="cuda")
    if kind == "model":
        n = min(V, 40)
        at = torch.randint(0, V // n, (T, n), generator=g, device="cuda") + torch.arange(n, device="cuda") * (V // n)
        x.scatter_(1, at, 6.0 + 3.0 * torch.randn((T, n), generator=g, device="cuda"))
    elif kind == "flat":
        x *= 0.05
    elif kind == "steps":                   # few different values
        x = x.round()
    elif kind == "masked":
        x = torch.where(torch.rand((T, V), generator=g, device="cuda") < 0.03, x, -math.inf)
    elif kind == "wide":
        x = x * 40
    return x


def _rules(g, T, V, which):
    r = lambda: torch.rand(T, generator=g, device="cuda")  # noqa: E731
    pick = lambda *v: torch.tensor(v, device="cuda")[torch.randint(0, len(v), (T,), generator=g, device="cuda")]  # noqa: E731
    return dict(temperature=pick(0.0, 0.1, 0.7, 1.0, 1.3, 5.0, -1.0) if "t" in which else None,
                top_k=pick(0, 1, 2, 5, 50, 300, 1024, 1500, 5000, V - 1, V, V + 7, -4).to(torch.int32) if "k" in which else None,
                top_p=pick(0.0, 0.05, 0.5, 0.9, 0.95, 0.999, 1.0, 1.5) if "p" in which else None,
                min_p=torch.where(r() < 0.5, 10.0 ** (-6 * r()), pick(0.0, 1.0, 0.05, -1.0, 2.0)) if "m" in which else None)


DTYPES = {"f32": (torch.float32, "f32"), "bf16": (torch.bfloat16, "bf16"), "f32_of_bf16": (torch.float32, "bf16")}


@pytest.mark.parametrize("V", [1, 2, 7, 64, 257, 1003, 4099, 16389, 32000, 50257, 65536, 70001, 131072])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_draw(lib, dtype, V):
    dt, model = DTYPES[dtype]
    ctx, g = _ctx(lib, V, model), _gen(V)
    for i, kind in enumerate(("model", "flat", "steps", "masked", "wide")):
        for which in ("", "k", "p", "m", "tkpm", "tkp"):
            T = 7 if V < 40000 else 3
            x = _logits(g, T, V, kind).to(dt)
            _check(ctx, lib, x, torch.rand(T, generator=g, device="cuda"), **_rules(g, T, V, which))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [5, 1000, 9001, 66000])
def test_draw_borders(lib, dtype, V):
    """Random numbers at and beyond their ends, rows of one value, rows with one column or none to draw, infinities, columns that hold no number, zeros of both signs."""
    dt, model = DTYPES[dtype]
    ctx, g = _ctx(lib, V, model), _gen(3 + V)
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 7.0, -1.0, math.nan, 2.0 ** -24, 0.5], device="cuda")
    T = len(u)
    rows = [torch.zeros((T, V)), torch.full((T, V), -math.inf), torch.full((T, V), math.nan), torch.full((T, V), -3e38), torch.full((T, V), math.inf),
            torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0).expand(T, V)]
    one = torch.full((T, V), -math.inf)
    one[:, V // 2] = -100.0
    some = _logits(g, T, V).cpu()
    some[:, ::3] = math.nan
    some[:, 1::3] = -math.inf
    tops = _logits(g, T, V).cpu()
    tops[:, [1, V - 1]] = math.inf
    far = torch.full((T, V), -2000.0)       # the others are next to impossible
    far[:, V - 1] = 0.0
    for x in rows + [one, some, tops, far]:
        x = x.to(dt).cuda().contiguous()
        _check(ctx, lib, x, u)
        for which in ("k", "p", "m", "tkpm"):
            _check(ctx, lib, x, u, **_rules(g, T, V, which))
        _check(ctx, lib, x, u, top_k=torch.full((T,), 3, dtype=torch.int32, device="cuda"), top_p=torch.full((T,), 0.5, device="cuda"))


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_draw_strides_and_places(lib, dtype):
    """Rows at any distance from any element on; what lies between them is not read as theirs, results go where they are asked for."""
    dt, model = DTYPES[dtype]
    for V, pad, first in ((1003, 0, 1), (1003, 5, 0), (4100, 4, 3), (50257, 7, 2), (70003, 1, 5)):
        ctx, g = _ctx(lib, V, model), _gen(V + pad)
        T = 4
        whole = torch.full((T * (V + pad) + first + 3,), math.inf, dtype=dt, device="cuda")
        x = whole[first: first + T * (V + pad)].view(T, V + pad)[:, :V]
        x.copy_(_logits(g, T, V))
        out = [torch.full((T + 2,), -7, dtype=d, device="cuda") for d in (torch.int32, torch.float32, torch.int32)]
        got = _check(ctx, lib, x, torch.rand(T, generator=g, device="cuda"), **_rules(g, T, V, "kp"), tokens=out[0][1:-1], logprobs=out[1][1:-1], kept=out[2][1:-1])
        assert all((o[[0, -1]] == -7).all() and (o[1:-1] == r).all() for o, r in zip(out, got))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [5, 1000, 9001, 66000])
def test_draw_at_an_infinite_temperature(lib, dtype, V):
    """All columns but those at -infinity are as probable as the most probable one, also for a min_p of 1."""
    dt, model = DTYPES[dtype]
    ctx, g = _ctx(lib, V, model), _gen(V + 41)
    x = torch.cat([_logits(g, 1, V, kind) for kind in ("model", "flat", "masked", "wide", "model")])
    x[4, V - 1] = math.inf
    x = x.to(dt)
    T = len(x)
    hot = torch.full((T,), math.inf, device="cuda")
    for rules in ({}, dict(top_k=3), dict(top_k=1200), dict(top_p=0.5), dict(min_p=0.5), dict(min_p=1.0), dict(min_p=2.0), dict(top_k=40, min_p=1.0), dict(top_p=0.7, min_p=1.0)):
        rules = {k: torch.full((T,), v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in rules.items()}
        _check(ctx, lib, x, torch.rand(T, generator=g, device="cuda"), temperature=hot, **rules)


def test_draw_many_rows(lib):
    V, T = 300, 5000
    ctx, g = _ctx(lib, V), _gen(9)
    x = _logits(g, T, V)
    rules = _rules(g, T, V, "tkpm")
    first = _check(ctx, lib, x, torch.rand(T, generator=g, device="cuda"), rows=range(0, T, 97), **rules)
    assert ((first[0] >= 0) & (first[0] < V)).all()


def test_draws_follow_the_distribution(lib):
    """Evenly spaced random numbers draw every column as often as its probability says, but for one at each of its two ends."""
    V, T = 50, 8192
    ctx, g = _ctx(lib, V), _gen(1)
    x = torch.randn((1, V), generator=g, device="cuda")
    tokens, _, kept = ctx.twist_draw_raw(x.expand(T, V).contiguous(), (torch.arange(T, device="cuda") + 0.5) / T)
    n = torch.bincount(tokens.long(), minlength=V).double()
    assert (n - T * torch.softmax(x[0].double(), 0)).abs().max() <= 1.0 + 1e-6 and (kept == V).all()


def test_draw_refuses_what_does_not_fit(lib):
    V, T = 100, 4
    ctx = _ctx(lib, V, "bf16")
    x, u = torch.zeros((T, V), dtype=torch.bfloat16, device="cuda"), torch.zeros(T, device="cuda")
    i32 = torch.zeros(T, dtype=torch.int32, device="cuda")
    bad = [lambda: ctx.twist_draw_raw(x.half(), u), lambda: ctx.twist_draw_raw(x[:, :99], u), lambda: ctx.twist_draw_raw(x.cpu(), u), lambda: ctx.twist_draw_raw(x.t().contiguous().t(), u),
           lambda: ctx.twist_draw_raw(x, u[:3]), lambda: ctx.twist_draw_raw(x, u.double()), lambda: ctx.twist_draw_raw(x, u.cpu()), lambda: ctx.twist_draw_raw(x, None),
           lambda: ctx.twist_draw_raw(x, u, lib.DrawRules(top_p=u[:3].clone())), lambda: ctx.twist_draw_raw(x, u, tokens=i32[:3]), lambda: ctx.twist_draw_raw(x, u, tokens=u),
           lambda: ctx.twist_draw_raw(x, u, kept=torch.zeros(2 * T, dtype=torch.int32, device="cuda")[::2]), lambda: lib.DrawRules(top_k=u), lambda: lib.DrawRules(top_p=i32),
           lambda: lib.DrawRules(temperature=u, top_p=u[:2].clone()), lambda: ctx.twist_top_logits_raw(x, 0), lambda: ctx.twist_top_logits_raw(x, 1025),
           lambda: ctx.twist_top_logits_raw(x, 5, temperature=0.0), lambda: ctx.twist_top_logits_raw(x, 5, ids=torch.zeros((T, 6), dtype=torch.int32, device="cuda")),
           lambda: ctx.twist_top_logits_raw(x, 5, ids=torch.zeros((T, 6), dtype=torch.int32, device="cuda")[:, :5]),
           lambda: ctx.twist_top_logits_raw(x, 5, rest=i32)]
    for call in bad:
        with pytest.raises(lib.TwistError):
            call()


# ------------------------------------------------------------------------------------------------ the largest logits
def _check_top(ctx, x, k, tau=1.0, rows=None, **kw):
    T, V = x.shape
    ids, values, rest = ctx.twist_top_logits_raw(x, k, temperature=tau, **kw)
    xs, tau = x.double().cpu().numpy(), float(np.float32(tau))
    ids_, values_, rest_ = ids.cpu().numpy(), values.double().cpu().numpy(), rest.double().cpu().numpy()
    n = min(k, V)
    for t in range(T) if rows is None else rows:
        at, z = _order(xs[t])
        assert (ids_[t, :n] == at[:n]).all() and (values_[t, :n] == z[:n]).all(), t
        assert (ids_[t, n:] == -1).all() and (values_[t, n:] == -np.inf).all()
        m = z[n] if n < V else -np.inf
        if not np.isfinite(m):
            assert rest_[t] == m, (t, rest_[t], m)
            continue
        want = m / tau + math.log(np.exp((z[n:] - m) / tau).sum())
        off = U * (2 * math.log(V) + 4 + V / 256 + 16 + 2 * abs(m / tau) + 2 * abs(want - m / tau) + abs(want))
        assert abs(rest_[t] - want) <= off, (t, rest_[t], want, off)
    return ids, values, rest


@pytest.mark.parametrize("V", [1, 3, 65, 1003, 4099, 16389, 32000, 50257, 65536, 70001, 131072])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_top_logits(lib, dtype, V):
    dt, model = DTYPES[dtype]
    ctx, g = _ctx(lib, V, model), _gen(V + 1)
    for kind in ("model", "flat", "steps", "masked", "wide"):
        for k, tau in ((1, 1.0), (17, 2.0), (64, 0.5), (200, 1.0), (1000, 3.3), (1024, 1.0)):
            _check_top(ctx, _logits(g, 3, V, kind).to(dt), k, tau)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [5, 1000, 9001, 66000])
def test_top_logits_borders(lib, dtype, V):
    dt, model = DTYPES[dtype]
    ctx, g = _ctx(lib, V, model), _gen(5)
    some = _logits(g, 2, V).cpu()
    some[:, ::2] = math.nan
    tops = _logits(g, 2, V).cpu()
    tops[:, [0, V // 2, V - 1]] = math.inf
    zeros = torch.where(torch.arange(V) % 2 == 0, 0.0, -0.0).expand(2, V)
    far = torch.full((2, V), -3e38)
    far[:, V // 3] = 3e38
    for x in (torch.zeros((2, V)), torch.full((2, V), -math.inf), torch.full((2, V), math.nan), some, tops, zeros, far, torch.arange(2 * V).view(2, V).float()):
        for k in (1, 2, 40, 1024):
            _check_top(ctx, x.to(dt).cuda().contiguous(), k)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_top_logits_strides_and_places(lib, dtype):
    dt, model = DTYPES[dtype]
    for V, pad, first, k in ((1003, 0, 1, 30), (1003, 5, 0, 7), (4100, 4, 3, 100), (50257, 7, 2, 20), (70003, 1, 5, 20)):
        ctx, g = _ctx(lib, V, model), _gen(V + pad)
        T = 4
        whole = torch.full((T * (V + pad) + first + 3,), math.inf, dtype=dt, device="cuda")
        x = whole[first: first + T * (V + pad)].view(T, V + pad)[:, :V]
        x.copy_(_logits(g, T, V))
        ids, values = (torch.full((T, k + 3), -7, dtype=d, device="cuda") for d in (torch.int32, torch.float32))
        _check_top(ctx, x, k, ids=ids[:, 1: k + 1], values=values[:, 1: k + 1])
        assert all((o[:, 0] == -7).all() and (o[:, k + 1:] == -7).all() for o in (ids, values))


def test_top_logits_many_rows(lib):
    V, T = 1003, 3000
    ctx, g = _ctx(lib, V, "bf16"), _gen(2)
    _check_top(ctx, _logits(g, T, V).bfloat16(), 12, rows=range(0, T, 61))


@pytest.mark.parametrize("V", [1000, 9001, 70001])
def test_rest_at_temperatures_near_their_ends(lib, V):
    """Differences of logits that fp32 does not hold, at temperatures that make them small; and the smallest ones, at temperatures as small."""
    ctx, g = _ctx(lib, V), _gen(V + 51)
    far = torch.where(torch.rand((2, V), generator=g, device="cuda") < 0.5, -1.0, 1.0) * (3e38 + 3e37 * torch.rand((2, V), generator=g, device="cuda"))
    near = torch.randint(0, 5, (2, V), generator=g, device="cuda") * 2.0 ** -149
    for k in (1, 64, 300):
        for x, taus in ((far, (3e38, 1e38, 1e32, 1.0, 1e-3)), (near, (2.0 ** -149, 1e-44, 1e-40, 1e-30, 1.0)), (_logits(g, 2, V), (1e-28, 1e-20, 1e20, 1e31, 3e38))):
            for tau in taus:
                t = float(np.float32(tau))
                xs = x.double().cpu().numpy()
                ids, values, rest = ctx.twist_top_logits_raw(x, k, temperature=tau)
                for row in range(2):
                    at, z = _order(xs[row])
                    assert (ids[row].cpu().numpy() == at[:k]).all() and (values[row].double().cpu().numpy() == z[:k]).all()
                    want = z[k] / t + math.log(np.exp((z[k:] - z[k]) / t).sum())
                    if abs(want) > 3.4e38:
                        assert float(rest[row]) == math.copysign(math.inf, want)
                        continue
                    off = U * (2 * math.log(V) + 4 + V / 256 + 16 + 2 * abs(z[k] / t) + 2 * abs(want - z[k] / t) + abs(want))      # (as for other temperatures)
                    assert abs(float(rest[row]) - want) <= off, (k, tau, row, float(rest[row]), want, off)


@pytest.mark.parametrize("V", [1000, 9001, 70001])
def test_rest_of_infinite_logits(lib, V):
    """More columns at +infinity than the list has: so are the others together, at any temperature."""
    ctx, g = _ctx(lib, V), _gen(V + 61)
    x = torch.where(torch.rand((2, V), generator=g, device="cuda") < 0.5, math.inf, _logits(g, 2, V))
    for k in (1, 64, 300):
        for tau in (2.0 ** -149, 1e-20, 1.0, 3e38):
            ids, values, rest = ctx.twist_top_logits_raw(x, k, temperature=tau)
            for row in range(2):
                assert (ids[row].cpu().numpy() == _order(x[row].double().cpu().numpy())[0][:k]).all()
            assert (values == math.inf).all() and (rest == math.inf).all(), (k, tau)


# ------------------------------------------------------------------------------------------------ both, of many rows
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [5, 1000, 9001, 33000, 66000])
def test_rows_that_differ_by_next_to_nothing(lib, dtype, V):
    """Logits less than 1e-36 apart, down to the smallest steps of their type: bins of equal width between them would be more than fp32 has numbers for a unit."""
    dt, model = DTYPES[dtype]
    ctx, g = _ctx(lib, V, model), _gen(V + 31)
    step = 2.0 ** -149 if dt == torch.float32 else 2.0 ** -133
    noise = torch.randn((3, V), generator=g, device="cuda")
    few = torch.zeros((7, V), device="cuda")
    few[0, V // 3] = 1e-37
    few[1, V - 1] = -1e-37
    few[2] = torch.randint(0, 5, (V,), generator=g, device="cuda") * step
    few[3:6] = noise * torch.tensor([[1e-37], [5e-39], [1e-36]], device="cuda")
    few[6, 0], few[6, V // 2] = 7e-37, 3e-37
    for times in (1, 38):                                                 # (38: 266 rows, which other kernels take)
        n = len(few)
        x = few.to(dt).repeat(times, 1)
        u = torch.rand(n, generator=g, device="cuda")
        for rules in ({}, dict(top_k=3), dict(top_k=300), dict(top_k=1500), dict(top_p=0.5), dict(min_p=0.05), dict(temperature=1e-37, top_p=0.9), dict(temperature=1e-37, top_k=40, min_p=0.3)):
            rules = {k: torch.full((n * times,), v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in rules.items()}
            for got in _check(ctx, lib, x, u.repeat(times), rows=range(n), **rules):
                assert (got.view(times, n) == got[:n]).all()
        for k, tau in ((1, 1.0), (3, 1e-37), (64, 1.0), (200, 1e-37), (300, 1.0), (1024, 1.0)):
            ids, values, _ = _check_top(ctx, x, k, tau, rows=range(n))
            assert (ids.view(times, n, k) == ids[:n]).all() and (values.view(times, n, k) == values[:n]).all()


@pytest.mark.parametrize("V", [4097, 9001, 16384, 16387, 32000, 32768, 40001, 50257, 65536])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_rows_side_by_side(lib, dtype, V):
    """More rows than one for every CU, 264 of 22 kinds, which other kernels take than few rows: what they give for a kind is right and the same for all of its rows."""
    dt, model = DTYPES[dtype]
    ctx, g = _ctx(lib, V, model), _gen(V + 11)
    kinds = [_logits(g, 3, V, k) for k in ("model", "flat", "steps", "masked", "wide")]
    special = torch.zeros((7, V), device="cuda")
    special[0] = -math.inf
    special[1] = math.nan
    special[2, V - 1] = math.inf
    special[3] = -2000.0
    special[3, V // 2] = 0.0
    special[4, ::3] = math.nan
    special[5] = torch.arange(V, device="cuda") / 64
    n, times = 22, 12
    few = torch.cat(kinds + [special]).to(dt)
    whole = torch.zeros((n * times, V + 3), dtype=dt, device="cuda")
    x = whole[:, :V]
    x.copy_(few.repeat(times, 1))
    u = torch.rand(n, generator=g, device="cuda")
    for which in ("", "k", "p", "m", "tkpm"):
        rules = {k: v if v is None else v.repeat(times) for k, v in _rules(g, n, V, which).items()}
        for got in _check(ctx, lib, x, u.repeat(times), rows=range(n), **rules):
            assert (got.view(times, n) == got[:n]).all()
    for k in (1, 64, 300, 1024):
        ids, values, rest = _check_top(ctx, x, k, 0.7, rows=range(0, 4 * n, 3))
        for got in (ids, values):
            assert (got.view(times, n, k) == got[:n]).all()
        assert (rest.view(times // 4, 4 * n) == rest[: 4 * n]).all()   # a sum in 32 bits, grouped by aligned addresses, which a row has again 4 n rows on


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_largest_vocabulary(lib, dtype):
    dt, model = DTYPES[dtype]
    V, T = 2 ** 20 - 1, 2
    ctx, g = _ctx(lib, V, model), _gen(21)
    for kind in ("model", "flat"):
        x = _logits(g, T, V, kind).to(dt)
        for which in ("", "k", "p", "m"):
            _check(ctx, lib, x, torch.rand(T, generator=g, device="cuda"), **_rules(g, T, V, which))
        for k in (1, 200, 1024):
            _check_top(ctx, x, k)


def test_rows_beyond_32_bits(lib):
    """Rows so far apart that the last begin behind 2^32 elements."""
    V, T, ld = 1003, 5, 2 ** 30 + 1
    ctx, g = _ctx(lib, V, "bf16"), _gen(22)
    x = torch.empty((T - 1) * ld + V, dtype=torch.bfloat16, device="cuda").as_strided((T, V), (ld, 1))
    near = _logits(g, T, V).bfloat16()
    x.copy_(near)
    u = torch.rand(T, generator=g, device="cuda")
    for far, here in ((ctx.twist_draw_raw(x, u), ctx.twist_draw_raw(near, u)), (ctx.twist_top_logits_raw(x, 20), ctx.twist_top_logits_raw(near, 20))):
        assert torch.equal(far[0], here[0]) and (far[1] - here[1]).abs().max() == 0 and (far[2] - here[2]).abs().max() <= 1e-5   # (rest, grouped differently: twice 38 u and 8 u)
