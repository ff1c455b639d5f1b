"""Kernel-level parity of the steps of generating tokens (appending to a paged cache, attention over it, rules on logits), each against the formula in
64 bits on identical inputs, element by element.  u below is the rounding of the stored type (half a step: bf16 2^-8, fp32 2^-24)."""
import math
from collections import Counter

import numpy as np
import pytest
import torch

import synth_inputs as si

pytestmark = pytest.mark.gpu

BF, F32 = "bf16", "f32"
U = {BF: 2.0 ** -8, F32: 2.0 ** -24}
E24 = 2.0 ** -24
NAN, INF = float("nan"), float("inf")


def _ctx(lib, dtype, dh, rope=False, vocab=0, theta=10000.0, stream=None):
    cfg = si.ModelCfg(arch="llama", d_model=64, n_heads=1, d_head=dh, d_ff=8, vocab=vocab, rope=rope, rope_theta=theta, dtype=dtype)
    return lib.Context(lib.desc_from_cfg(cfg), stream)


def _dt(dtype):
    return torch.bfloat16 if dtype == BF else torch.float32


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype=F32, scale=1.0):
    return (scale * torch.randn(shape, generator=g, device="cuda")).to(_dt(dtype))


def _i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pools(g, n_pages, Hs, page, dh, dtype, extra=0):
    """Two pools whose pages lie `extra` elements further apart than they are long."""
    one = Hs * page * dh
    out = []
    for _ in range(2):
        flat = _randn(g, n_pages * (one + extra), dtype=dtype)
        out.append(flat.as_strided((n_pages, Hs, page, dh), (one + extra, page * dh, dh, 1)))
    return out


def _rounded(x, dtype):
    return x.to(_dt(dtype)).double()


# ------------------------------------------------------------------------------------------------ append
def _append_want(k, v, table, qkv, lens, seq, q_out, Hs, dh, rope, theta):
    """64-bit copies of (q_out, k, v) after the call, and the bound of each beside its rounding."""
    k, v, q_out = k.double().cpu(), v.double().cpu(), q_out.double().cpu()
    ek, eq = torch.zeros_like(k), torch.zeros_like(q_out)
    n_pages, _, page, _ = k.shape
    table, half = table.cpu(), dh // 2
    w = torch.tensor([theta ** (-2.0 * i / dh) for i in range(half)], dtype=torch.float64)
    for t, n in enumerate(lens.tolist()):
        s = t if seq is None else int(seq[t])
        if n < 1 or not 0 <= s < table.shape[0]:
            continue
        q, key, val = qkv[t].double().cpu().view(3, Hs, dh)
        size = []
        if rope:
            c, sn = torch.cos((n - 1) * w), torch.sin((n - 1) * w)
            turned = []
            for x in (q, key):
                a, b = x[:, :half], x[:, half:]
                turned.append(torch.cat([a * c - b * sn, b * c + a * sn], 1))
                size.append((a.abs() + b.abs()).repeat(1, 2))
            q, key = turned
        # the angle's turn is rounded to 2^-26 of a turn (2^-23.3 in radians), its sine and cosine to 2 ulp (2^-23), the two products and their
        # sum to 2^-23 of what they are made of: 2^-21 of |a| + |b| in all
        q_out[t] = q.reshape(-1)
        if rope:
            eq[t] = size[0].reshape(-1) * 2.0 ** -21
        i = (n - 1) // page
        at = int(table[s, i]) if i < table.shape[1] else -1
        if 0 <= at < n_pages:
            k[at, :, (n - 1) % page], v[at, :, (n - 1) % page] = key, val
            if rope:
                ek[at, :, (n - 1) % page] = size[1] * 2.0 ** -21
    return q_out, k, v, eq, ek


def _close(got, want, err, u):
    got, want = got.double().cpu(), want.cpu()
    bad = (got - want).abs() > u * want.abs() + err * (1 + u)
    assert not bad.any(), (int(bad.sum()), float((got - want).abs().max()))


def _check_append(lib, dtype, Hs, dh, rope, page, lens, seq=None, n_seqs=None, max_pages=4, extra=0, pad=0, theta=10000.0, holes=True, in_place=False, seed=0):
    g = _gen(seed + dh + Hs)
    ctx = _ctx(lib, dtype, dh, rope, theta=theta)
    T, HD = len(lens), Hs * dh
    n_seqs = n_seqs or T
    n_pages = n_seqs * max_pages + 1
    k, v = _pools(g, n_pages, Hs, page, dh, dtype, extra)
    table = torch.randperm(n_pages, generator=g, device="cuda")[: n_seqs * max_pages].to(torch.int32).view(n_seqs, max_pages)
    if holes:      # pages that a sequence does not have, by every kind of entry outside the pool
        for j, bad in enumerate((-1, n_pages, 2 ** 31 - 1, -2 ** 31)):
            if j + 1 < n_seqs:
                table[j + 1, 0] = bad
    buf = _randn(g, T, 3 * HD + pad, dtype=dtype)
    qkv = buf[:, : 3 * HD]
    q_out = qkv[:, :HD] if in_place else _randn(g, T, HD + pad, dtype=dtype)[:, :HD]
    lens_t = _i32(*lens)
    seq_t = None if seq is None else _i32(*seq)
    before = qkv.clone()
    wq, wk, wv, eq, ek = _append_want(k, v, table, before, lens_t, seq_t, q_out, Hs, dh, rope, theta)
    ctx.twist_cache_append_raw(lib.PagedCache(k, v, table), qkv, lens_t, seq=seq_t, q_out=q_out)
    torch.cuda.synchronize()
    u = U[dtype] if rope else 0.0
    _close(q_out, wq, eq, u)
    # what is not appended keeps its bits: its bound is 0
    changed = (ek > 0) if rope else torch.zeros_like(wk, dtype=torch.bool)
    _close(k, wk, ek, torch.where(changed, u, 0.0))
    assert torch.equal(v.double().cpu(), wv)
    assert torch.equal(qkv[:, HD:], before[:, HD:])
    if not in_place:
        assert torch.equal(qkv, before)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rope", [True, False])
@pytest.mark.parametrize("Hs,dh,page", [(1, 128, 16), (5, 64, 16), (3, 32, 1), (2, 256, 8), (7, 40, 32), (3, 80, 16), (5, 6, 4), (2, 20, 8), (16, 128, 64), (2, 2, 2)])
def test_append(lib, dtype, rope, Hs, dh, page):
    """Head widths that load 16 bytes at a time and ones that do not, sequences of one token, the last and first places of a page, unused rows, missing
    pages, positions beyond the table."""
    lens = [1, 2, page, page + 1, 2 * page, 3 * page, 4 * page, 0, -3, 4 * page + 1, 3]
    _check_append(lib, dtype, Hs, dh, rope, page, lens)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_prompts_and_single_tokens(lib, dtype):
    lens = list(range(1, 38)) + [5] + list(range(60, 65)) + [0, 0, 7, 7]
    seq = [2] * 37 + [0] + [1] * 5 + [0, 1, -1, 9]          # a prompt, one token, a few drafted ones, unused rows, sequences that are none
    _check_append(lib, dtype, 4, 64, True, 16, lens, seq, n_seqs=3, holes=False)
    _check_append(lib, dtype, 4, 64, True, 16, lens, seq, n_seqs=3, holes=False, in_place=True)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("extra,pad", [(8, 8), (3, 5), (0, 1), (16, 0), (4, 4)])
def test_append_strides(lib, dtype, extra, pad):
    """Pages and rows that are padded, by whole 16-byte pieces and not."""
    _check_append(lib, dtype, 3, 64, True, 16, [1, 16, 17, 30, 64], extra=extra, pad=pad, holes=False)
    _check_append(lib, dtype, 3, 64, False, 16, [1, 16, 17, 30, 64], extra=extra, pad=pad, holes=False, in_place=True)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_append_at_far_positions(lib, dtype):
    """An angle of a million radians: 32 bits of it are off by 0.03."""
    ctx, g = _ctx(lib, dtype, 64, True), _gen(3)
    k, v = _pools(g, 3, 2, 4096, 64, dtype)
    table = torch.full((2, 300), -1, dtype=torch.int32, device="cuda")
    table[0, 244], table[1, 299] = 2, 1
    lens = _i32(10 ** 6 + 1, 300 * 4096)
    qkv, q_out = _randn(g, 2, 3 * 128, dtype=dtype), torch.zeros((2, 128), dtype=_dt(dtype), device="cuda")
    wq, wk, wv, eq, ek = _append_want(k, v, table, qkv, lens, None, q_out, 2, 64, True, 10000.0)
    ctx.twist_cache_append_raw(lib.PagedCache(k, v, table), qkv, lens, q_out=q_out)
    torch.cuda.synchronize()
    _close(q_out, wq, eq, U[dtype])
    _close(k, wk, ek, torch.where(ek > 0, U[dtype], 0.0))
    assert torch.equal(v.double().cpu(), wv)


def test_append_of_many_rows(lib):
    """Enough rows for every form of the kernel, and without queries."""
    g = _gen(9)
    for T, Hs, dh in ((700, 12, 64), (3000, 3, 128), (129, 32, 128)):
        ctx = _ctx(lib, BF, dh, True)
        page, n_seqs = 16, 3
        max_pages = -(-T // page)
        k, v = _pools(g, n_seqs * max_pages, Hs, page, dh, BF)
        table = torch.randperm(n_seqs * max_pages, generator=g, device="cuda").to(torch.int32).view(n_seqs, max_pages)
        seq = (torch.arange(T, device="cuda") % n_seqs).to(torch.int32)
        lens = (torch.arange(T, device="cuda") // n_seqs + 1).to(torch.int32)
        qkv = _randn(g, T, 3 * Hs * dh, dtype=BF)
        q_out = torch.zeros((T, Hs * dh), dtype=torch.bfloat16, device="cuda")
        k0, v0 = k.clone(), v.clone()
        wq, wk, wv, eq, ek = _append_want(k, v, table, qkv, lens, seq, q_out, Hs, dh, True, 10000.0)
        ctx.twist_cache_append_raw(lib.PagedCache(k, v, table), qkv, lens, seq=seq, q_out=q_out)
        ctx.twist_cache_append_raw(lib.PagedCache(k0, v0, table), qkv, lens, seq=seq)
        torch.cuda.synchronize()
        _close(q_out, wq, eq, U[BF])
        _close(k, wk, ek, torch.where(ek > 0, U[BF], 0.0))
        assert torch.equal(v.double().cpu(), wv) and torch.equal(k, k0) and torch.equal(v, v0)


# ------------------------------------------------------------------------------------------------ attention
def _attention_want(k, v, table, q, lens, seq, max_len, Hs, dh):
    """(o, lse, bound of o beside its rounding, bound of lse), 64 bits; rows that are left alone are NaN."""
    # rows with a list of sequences, bf16: weights in two bf16 terms, the first cut off (what is left is below 2^-7 of the weight), the second rounded (2^-9)
    terms = 2.0 ** -16 if seq is not None and k.dtype == torch.bfloat16 else 0.0
    n_pages, _, page, _ = k.shape
    T = q.shape[0]
    o = torch.full((T, Hs * dh), NAN, dtype=torch.float64)
    lse = torch.full((T, Hs), NAN, dtype=torch.float64)
    eo, el = torch.zeros_like(o), torch.zeros_like(lse)
    table = table.cpu()
    for t, n in enumerate(lens.tolist()):
        s = t if seq is None else int(seq[t])
        if n < 0 or not 0 <= s < table.shape[0]:
            continue
        n = min(n, max_len, table.shape[1] * page)
        pos = [p for p in range(n) if 0 <= int(table[s, p // page]) < n_pages]
        if not pos:
            o[t], lse[t] = 0.0, -INF
            continue
        at = torch.tensor([int(table[s, p // page]) for p in pos], device=k.device)
        slot = torch.tensor([p % page for p in pos], device=k.device)
        kk, vv = k[at, :, slot].double().cpu(), v[at, :, slot].double().cpu()          # [n, Hs, dh]
        qq = q[t].double().cpu().view(1, Hs, dh)
        sc = (kk * qq).sum(-1) / math.sqrt(dh)
        p = torch.softmax(sc, 0)
        o[t] = (p[..., None] * vv).sum(0).reshape(-1)
        lse[t] = torch.logsumexp(sc, 0)
        # a score: dh products summed in any order, scaled, brought to base 2 and its exponential taken (2^-23): dh + 4 roundings of the sum of
        # magnitudes; a sum over n keys: n + 8 roundings, of the softmax's sum and of the output's alike
        mag = (kk * qq).abs().sum(-1) / math.sqrt(dh)
        ds = (dh + 4) * E24 * mag.amax(0) + 2.0 ** -22                                  # [Hs]
        rel = 2 * ds + 2 * (len(pos) + 8) * E24 + terms
        eo[t] = (rel[:, None] * (p[..., None] * vv.abs()).sum(0)).reshape(-1)
        el[t] = ds + (len(pos) + 8) * E24 + lse[t].abs() * 2.0 ** -23
    return o, lse, eo, el


def _check_attention(lib, dtype, Hs, dh, page, lens, seq=None, n_seqs=None, max_len=None, extra=0, pad=0, holes=(), q_scale=1.5, seed=0, max_pages=None, poison=True,
                     ctx=None):
    g = _gen(seed + dh + Hs)
    ctx = ctx or _ctx(lib, dtype, dh)
    T, HD = len(lens), Hs * dh
    n_seqs = n_seqs or T
    top = max(max(lens), 1)
    max_len = top if max_len is None else max_len
    max_pages = max_pages or -(-top // page)
    n_pages = n_seqs * max_pages + 1
    k, v = _pools(g, n_pages, Hs, page, dh, dtype, extra)
    table = torch.randperm(n_pages, generator=g, device="cuda")[: n_seqs * max_pages].to(torch.int32).view(n_seqs, max_pages).clone()
    # nothing behind a sequence's end is used: NaN and infinities there, entries outside the pool where it has no more pages
    if poison:
        for s in range(n_seqs):
            rows = [t for t in range(T) if (t if seq is None else seq[t]) == s]
            end = max([min(lens[t], max_len) for t in rows] + [0])
            for i in range(max_pages):
                lo = max(0, min(page, end - i * page))
                if lo < page:
                    k[int(table[s, i]), :, lo:], v[int(table[s, i]), :, lo:] = NAN, INF if s % 2 else NAN
                if lo == 0:
                    table[s, i] = (-1, n_pages, 2 ** 31 - 1, -2 ** 31)[i % 4]
    for s, i in holes:
        at = int(table[s, i])
        if 0 <= at < n_pages:
            k[at], v[at] = NAN, NAN
        table[s, i] = -1
    q = _randn(g, T, HD + pad, dtype=dtype, scale=q_scale)[:, :HD]
    out = torch.full((T, HD + pad), 7.0, dtype=_dt(dtype), device="cuda")[:, :HD]
    lse = torch.full((T, Hs), 7.0, dtype=torch.float32, device="cuda")
    lens_t, seq_t = _i32(*lens), None if seq is None else _i32(*seq)
    ctx.twist_cache_attention_raw(lib.PagedCache(k, v, table), q, lens_t, max_len, seq=seq_t, out=out, lse=lse)
    torch.cuda.synchronize()
    wo, wl, eo, el = _attention_want(k, v, table, q, lens_t, seq_t, max_len, Hs, dh)
    left = torch.isnan(wl[:, 0])
    assert (out[left.cuda()] == 7).all() and (lse[left.cuda()] == 7).all()
    on = ~left
    _close(out.cpu()[on], wo[on], eo[on], U[dtype])
    got = lse.double().cpu()[on]
    empty = wl[on] == -INF
    assert (got[empty] == -INF).all()
    assert ((got - wl[on]).abs()[~empty] <= el[on][~empty]).all(), float((got - wl[on]).abs()[~empty].max())
    return out, lse


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hs,dh,page", [(1, 128, 16), (12, 64, 16), (3, 32, 1), (2, 256, 8), (7, 40, 32), (3, 80, 16), (5, 6, 4), (2, 20, 8), (4, 128, 128), (2, 1, 2), (1, 96, 256)])
def test_attention_lengths(lib, dtype, Hs, dh, page):
    lens = [1, 2, page, page + 1, 63, 64, 65, 127, 200, 256, 257, 300, 0, -1]
    _check_attention(lib, dtype, Hs, dh, page, lens)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hs,dh,page,T,top", [(2, 64, 16, 1, 3000), (1, 128, 64, 1, 5001), (3, 32, 16, 2, 2500), (2, 128, 16, 3, 1999), (1, 40, 8, 2, 1500), (1, 256, 16, 1, 2049),
                                               (1, 7, 16, 1, 1300)])
def test_attention_over_long_sequences_of_few_rows(lib, dtype, Hs, dh, page, T, top):
    """The length is what there is to share out; parts that no token reaches in the shorter rows."""
    _check_attention(lib, dtype, Hs, dh, page, [max(1, top // (3 * t + 1)) for t in range(T)], max_pages=-(-top // page) + 2)
    _check_attention(lib, dtype, Hs, dh, page, [top] + [0] * (T - 1), max_len=2 * top, max_pages=-(-top // page))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hs,dh,page", [(2, 128, 16), (3, 64, 16), (2, 32, 8), (1, 256, 16), (3, 40, 32), (2, 80, 16), (1, 96, 64), (2, 20, 8), (1, 8, 1), (1, 160, 16), (1, 192, 16), (1, 224, 16)])
def test_attention_of_rows_that_share_sequences(lib, dtype, Hs, dh, page):
    """Runs of rows of one sequence that start and end anywhere, in any order of lengths, beside rows of their own and unused ones; NaN behind each sequence."""
    lens = [97, 98, 99, 100, 1, 2, 3, 40, 41, 0, 50, 50, -1]
    seq = [0, 0, 0, 0, 2, 2, 2, 1, 1, 1, 7, -1, 0]
    _check_attention(lib, dtype, Hs, dh, page, lens, seq, n_seqs=3)
    _check_attention(lib, dtype, Hs, dh, page, list(range(1, 71)), [0] * 70, n_seqs=1)       # a whole prompt at once
    _check_attention(lib, dtype, Hs, dh, page, list(range(230, 195, -1)) + [-1, 0, 3], [1] * 38, n_seqs=2)
    _check_attention(lib, dtype, Hs, dh, page, [33, 34], [0, 0], n_seqs=1)                   # no more rows than a group has
    _check_attention(lib, dtype, Hs, dh, page, [20, 33, 4], [0, -1, 0], n_seqs=1)
    _check_attention(lib, dtype, Hs, dh, page, [1, 64, 65, 200, 0, 31, 32, 33, 16, 17, 300], list(range(11)), n_seqs=11)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hs,dh", [(1, 128), (2, 64), (1, 40)])
def test_attention_of_drafts_over_long_sequences(lib, dtype, Hs, dh):
    """Rows of one sequence whose last parts only some of them reach, missing pages among them."""
    _check_attention(lib, dtype, Hs, dh, 16, [4500, 4501, 4502, 4503, 4096, 4097, 1], [0] * 7, n_seqs=1)
    _check_attention(lib, dtype, Hs, dh, 16, [4500, 4501, 60, 2500, 2501], [1, 1, 1, 0, 0], n_seqs=2, holes=[(1, 3), (1, 200), (0, 0)] + [(1, i) for i in range(64, 128)])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_of_a_long_prompt(lib, dtype):
    """2500 rows of two sequences, one after another and mixed, against causal attention in 64 bits; the bound of every row as for single ones."""
    n, Hs, dh, page = 1250, 2, 64, 16
    ctx, g = _ctx(lib, dtype, dh), _gen(11)
    pages = -(-n // page)
    k, v = _pools(g, 2 * pages, Hs, page, dh, dtype)
    table = torch.randperm(2 * pages, generator=g, device="cuda").to(torch.int32).view(2, pages)
    q = _randn(g, 2 * n, Hs * dh, dtype=dtype)
    flat = lambda p, s: p[table[s].long()].permute(1, 0, 2, 3).reshape(Hs, -1, dh)[:, :n].double()  # noqa: E731
    for order in (torch.arange(2 * n, device="cuda"), torch.randperm(2 * n, generator=g, device="cuda")):
        seq, lens = (order // n).to(torch.int32), (order % n + 1).to(torch.int32)
        o, lse = ctx.twist_cache_attention_raw(lib.PagedCache(k, v, table), q, lens, n, seq=seq)
        torch.cuda.synchronize()
        for s in range(2):
            rows = torch.nonzero(seq == s)[:, 0]
            rows = rows[torch.argsort(lens[rows])]
            kk, vv, qq = flat(k, s), flat(v, s), q[rows].double().view(n, Hs, dh).transpose(0, 1)
            sc = torch.matmul(qq, kk.transpose(1, 2).contiguous()) / math.sqrt(dh)
            hidden = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
            p = torch.softmax(sc.masked_fill(hidden, -INF), -1)
            want = torch.matmul(p, vv)
            mag = torch.matmul(qq.abs(), kk.abs().transpose(1, 2).contiguous()).masked_fill(hidden, 0).amax(-1) / math.sqrt(dh)
            rel = 2 * ((dh + 4) * E24 * mag + 2.0 ** -22) + 2 * (n + 8) * E24 + (2.0 ** -16 if dtype == BF else 0.0)
            err = rel[..., None] * torch.matmul(p, vv.abs())
            got = o[rows].double().view(n, Hs, dh).transpose(0, 1)
            assert ((got - want).abs() <= U[dtype] * want.abs() + err * (1 + U[dtype])).all()
            wl = torch.logsumexp(sc.masked_fill(hidden, -INF), -1)
            assert ((lse[rows].double().t() - wl).abs() <= (dh + 4) * E24 * mag + 2.0 ** -22 + (n + 8) * E24 + wl.abs() * 2.0 ** -23).all()


def _tiled(lens, seq, Hs, dh, max_len):
    """The rows, and as many unused ones behind them as make a call large enough for tiles of 16 rows (2^25 products of a score, 256 tokens)."""
    more = max(0, -(-2 ** 25 // (Hs * dh * max_len)) - len(lens))
    return lens + [-1] * more, seq + [(-1, 0, 99)[i // 5 % 3] for i in range(more)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hs,dh,page", [(2, 128, 16), (3, 64, 16), (2, 32, 8), (1, 256, 16), (3, 40, 32), (2, 80, 16), (1, 96, 64), (2, 24, 8), (4, 8, 1), (1, 160, 16), (1, 192, 16), (1, 224, 16),
                                        (9, 16, 4), (2, 112, 128)])
def test_attention_in_tiles_of_rows(lib, dtype, Hs, dh, page):
    """Runs of rows of one sequence that start and end anywhere, in any order of lengths, beside rows of their own and unused ones; NaN behind each sequence."""
    check = lambda lens, seq, n_seqs, **kw: _check_attention(lib, dtype, Hs, dh, page, *_tiled(lens, seq, Hs, dh, 300), n_seqs=n_seqs, max_len=300, max_pages=-(-300 // page), **kw)  # noqa: E731
    check([97, 98, 99, 100, 1, 2, 3, 40, 41, 0, 50, 50, -1], [0, 0, 0, 0, 2, 2, 2, 1, 1, 1, 7, -1, 0], 3)
    check(list(range(1, 71)), [0] * 70, 1)                                                   # a whole prompt at once
    check(list(range(230, 195, -1)) + [-1, 0, 3, 299, 300], [1] * 40, 2)
    check([20, 33, 4, 290], [0, -1, 0, 0], 1, holes=[(0, 0), (0, 200 // page)])
    check([1, 64, 65, 200, 0, 31, 32, 33, 16, 17, 300], list(range(11)), 11)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hs,dh,page", [(2, 128, 16), (3, 64, 16), (1, 40, 32), (2, 80, 1), (1, 96, 64), (2, 120, 16), (1, 36, 8), (4, 72, 512)])
def test_attention_in_pairs_of_tiles(lib, dtype, Hs, dh, page):
    """Prompts: more than 32 rows a sequence and room for 768 tokens; runs that start and end anywhere, rows that end long before others of their tiles."""
    check = lambda lens, seq, n_seqs, **kw: _check_attention(lib, dtype, Hs, dh, page, *_tiled(lens, seq, Hs, dh, 800), n_seqs=n_seqs, max_len=800, max_pages=-(-800 // page), **kw)  # noqa: E731
    check(list(range(1, 71)) + [790, 5, 0, -1, 300], [0] * 75, 1)
    check(list(range(60, 0, -1)) + list(range(500, 520)) + [800], [1] * 60 + [0] * 21, 2)
    check([30, 31] + [700] * 17 + list(range(300, 340)), [0] * 2 + [2] * 17 + [1] * 40, 3, holes=[(2, 0), (1, 300 // page), (0, 0)])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Hs,dh,top", [(1, 128, 5000), (2, 64, 4503), (1, 40, 9000), (1, 256, 3001)])
def test_attention_in_tiles_over_long_sequences(lib, dtype, Hs, dh, top):
    """Sequences cut into parts, the last of which only some rows of a tile reach, missing pages among them."""
    lens, seq = [top - 3, top - 2, top - 1, top, 2048, 2049, 1, 0, -1, 700, 2500, 2501], [0] * 9 + [1] * 3
    check = lambda **kw: _check_attention(lib, dtype, Hs, dh, 16, *_tiled(lens, seq, Hs, dh, top), n_seqs=2, max_len=top, **kw)  # noqa: E731
    check()
    check(holes=[(0, 3), (1, 0), (1, 156)] + [(0, i) for i in range(64, 160)])


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("room", [320, 800])
def test_attention_in_tiles_of_values_that_are_no_numbers(lib, dtype, room):
    """An infinity reaches the rows that see it and no others, also where their scores leave nothing of a term of its weight."""
    ctx, g, dh = _ctx(lib, dtype, 64), _gen(8), 64
    k, v = _pools(g, room // 16, 1, 16, dh, dtype)
    table = torch.arange(room // 16, dtype=torch.int32, device="cuda").view(1, -1)
    cache = lib.PagedCache(k, v, table)
    lens, seq = _tiled([40, 41, 100, 320], [0, 0, 0, 0], 1, dh, room)
    q = torch.zeros((len(lens), dh), dtype=_dt(dtype), device="cuda")
    lens, seq = _i32(*lens), _i32(*seq)
    base = ctx.twist_cache_attention_raw(cache, q, lens, room, seq=seq)[0][:4].clone()
    v[2, 0, 8, 5] = INF                                    # token 40: the last of row 1, none of row 0
    v[6, 0, 2, 7] = -INF                                   # token 98
    v[16, 0, 5, 9] = NAN                                   # token 261: row 3 only
    o = ctx.twist_cache_attention_raw(cache, q, lens, room, seq=seq)[0][:4]
    torch.cuda.synchronize()
    assert torch.equal(o[0], base[0])
    assert (o[1:, 5] == INF).all() and torch.isfinite(o[1, 7]) and (o[2:, 7] == -INF).all()
    assert torch.isfinite(o[:3, 9]).all() and torch.isnan(o[3, 9])
    rest = [e for e in range(dh) if e not in (5, 7, 9)]
    # (such tokens go another way through the kernel: equal up to the 2^-16 of the weights' bf16 terms, or 320 + 8 roundings, and one rounding of the output)
    top = v[torch.isfinite(v)].float().abs().max()
    assert ((o - base).float().abs()[:, rest] <= 2 * U[dtype] * base.float().abs()[:, rest] + (2.0 ** -15 if dtype == BF else 328 * E24) * top).all()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_of_values_that_are_no_numbers(lib, dtype):
    """An infinity reaches the rows that see it and no others, also where their scores leave nothing of a term of its weight."""
    ctx, g, dh = _ctx(lib, dtype, 64), _gen(8), 64
    k, v = _pools(g, 8, 1, 16, dh, dtype)
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(1, -1)
    cache = lib.PagedCache(k, v, table)
    q = torch.zeros((4, dh), dtype=_dt(dtype), device="cuda")
    lens, seq = _i32(40, 41, 100, 128), _i32(0, 0, 0, 0)
    base, _ = ctx.twist_cache_attention_raw(cache, q, lens, 128, seq=seq)
    v[2, 0, 8, 5] = INF                                    # token 40: the last of row 1, none of row 0
    v[6, 0, 2, 7] = -INF                                   # token 98
    v[6, 0, 5, 9] = NAN                                    # token 101: row 3 only
    o, lse = ctx.twist_cache_attention_raw(cache, q, lens, 128, seq=seq)
    torch.cuda.synchronize()
    assert torch.equal(o[0], base[0])
    assert (o[1:, 5] == INF).all() and torch.isfinite(o[1, 7]) and (o[2:, 7] == -INF).all()
    assert torch.isfinite(o[:3, 9]).all() and torch.isnan(o[3, 9])
    rest = [e for e in range(dh) if e not in (5, 7, 9)]
    # (such tokens go another way through the kernel: equal up to the 2^-16 of the weights' bf16 terms, or 128 + 8 roundings, and one rounding of the output)
    assert ((o - base).float().abs()[:, rest] <= 2 * U[dtype] * base.float().abs()[:, rest] + (2.0 ** -15 if dtype == BF else 136 * E24 * v[torch.isfinite(v)].abs().max())).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("extra,pad", [(8, 8), (3, 5), (0, 1), (16, 0), (4, 4)])
def test_attention_strides(lib, dtype, extra, pad):
    _check_attention(lib, dtype, 3, 64, 16, [1, 17, 100, 250], extra=extra, pad=pad)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attention_without_pages(lib, dtype):
    """Pages missing in the middle, at the start, and all of them; a bound below the lengths, one beyond the table."""
    _check_attention(lib, dtype, 2, 64, 16, [100, 100, 100, 64, 30], holes=[(0, 1), (1, 0), (2, 6), (2, 0), (3, 0), (3, 1), (3, 2), (3, 3), (4, 0)])
    _check_attention(lib, dtype, 2, 64, 16, [100, 20, 90, 33], max_len=50)
    _check_attention(lib, dtype, 2, 64, 16, [100, 20, 200, 33], max_len=10 ** 6, max_pages=5)
    _check_attention(lib, dtype, 1, 128, 16, [4000], holes=[(0, i) for i in range(3, 200)])      # whole parts of a split sequence without a page
    _check_attention(lib, dtype, 1, 128, 16, [4000], holes=[(0, i) for i in range(0, 250)])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_pages_that_sequences_share(lib, dtype):
    """A common beginning of three sequences, read by all; one place written by two rows holds, value by value, one of theirs."""
    Hs, dh, page = 3, 64, 16
    ctx, g = _ctx(lib, dtype, dh), _gen(12)
    k, v = _pools(g, 8, Hs, page, dh, dtype)
    table = torch.tensor([[5, 2, 7, 0], [5, 2, 1, -1], [5, 5, 5, 3]], dtype=torch.int32, device="cuda")
    cache = lib.PagedCache(k, v, table)
    qkv, lens = _randn(g, 3, 3 * Hs * dh, dtype=dtype), _i32(50, 40, 64)
    ctx.twist_cache_append_raw(cache, qkv, lens)
    for seq in (None, _i32(2, 0, 0)):
        o, lse = ctx.twist_cache_attention_raw(cache, qkv[:, : Hs * dh], lens, 64, seq=seq)
        torch.cuda.synchronize()
        wo, wl, eo, el = _attention_want(k, v, table, qkv[:, : Hs * dh], lens, seq, 64, Hs, dh)
        _close(o, wo, eo, U[dtype])
        assert ((lse.double().cpu() - wl).abs() <= el).all()
    before = k.clone(), v.clone()
    ctx.twist_cache_append_raw(cache, qkv, _i32(4, 4, 36))              # places 3 of page 5, three times
    torch.cuda.synchronize()
    for i, (pool, old) in enumerate(zip((k, v), before), 1):
        theirs = qkv[:, i * Hs * dh : (i + 1) * Hs * dh].view(3, Hs, dh)
        assert (pool[5, :, 3] == theirs).any(0).all()
        old[5, :, 3] = pool[5, :, 3]
        assert torch.equal(pool, old)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("dh,n", [(64, 50), (64, 2000), (20, 50)])
def test_attention_of_extreme_scores(lib, dtype, dh, n):
    """One key far above the others, far below them, scores of -infinity beside finite ones; an infinite or undefined one gives no number."""
    _check_attention(lib, dtype, 2, dh, 16, [n], q_scale=30.0)
    ctx, g = _ctx(lib, dtype, dh), _gen(1)
    pages = -(-n // 16)
    k, v = _pools(g, pages, 2, 16, dh, dtype)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
    q = torch.zeros((1, 2 * dh), dtype=_dt(dtype), device="cuda")
    q[0, 0] = 1.0
    cache, lens = lib.PagedCache(k, v, table), _i32(n)
    k[0, 0, 3, 0] = -INF                       # head 0: a weight of nothing
    k[:, 1, :, :] = 0.0
    o, lse = ctx.twist_cache_attention_raw(cache, q, lens, n)
    rest = torch.cat([k[:, 0].reshape(-1, dh)[:n][:3], k[:, 0].reshape(-1, dh)[:n][4:]]).double()
    vals = torch.cat([v[:, 0].reshape(-1, dh)[:n][:3], v[:, 0].reshape(-1, dh)[:n][4:]]).double()
    p = torch.softmax(rest[:, 0] / math.sqrt(dh), 0)
    bound = (16 + n) * 2.0 ** -22 * (p[:, None] * vals.abs()).sum(0)
    _close(o[0, :dh], (p[:, None] * vals).sum(0).cpu(), bound.cpu(), U[dtype])
    k[:, 0, :, 0] = -INF                       # nothing but weights of nothing: 0 / 0, as a softmax gives
    o, lse = ctx.twist_cache_attention_raw(cache, q, lens, n)
    assert torch.isnan(o[0, :dh]).all() and torch.isfinite(o[0, dh:]).all() and lse[0, 0] == -INF
    for bad in (INF, NAN):
        k[:, 0, :, 0] = 0.5
        k[0, 0, 5, 0] = bad
        o, lse = ctx.twist_cache_attention_raw(cache, q, lens, n)
        assert torch.isnan(o[0, :dh]).all() and torch.isfinite(o[0, dh:]).all() and torch.isfinite(lse[0, 1])
    k[0, 0, 5, 0] = 0.5
    v[0, 0, 2, 1] = INF
    o, lse = ctx.twist_cache_attention_raw(cache, q, lens, n)
    assert o[0, 1] == INF and torch.isfinite(o[0, 2:]).all() and torch.isfinite(o[0, 0]) and torch.isfinite(lse).all()


def test_cache_beyond_32_bits(lib):
    """Pages whose element offsets pass 2^31 and byte offsets 2^33, read and written."""
    dh, Hs, page, stride = 64, 2, 16, 2 ** 30 + 8
    g = _gen(5)
    flat = [torch.zeros(4 * stride + Hs * page * dh, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    k, v = (f.as_strided((5, Hs, page, dh), (stride, page * dh, dh, 1)) for f in flat)
    for p in (k, v):
        p.copy_(_randn(g, 5, Hs, page, dh, dtype=BF))
    ctx = _ctx(lib, BF, dh)
    table = _i32(4, 1, 3, 0, 2).view(1, 5)
    cache = lib.PagedCache(k, v, table)
    qkv = _randn(g, 1, 3 * Hs * dh, dtype=BF)
    lens = _i32(10)
    ctx.twist_cache_append_raw(cache, qkv, lens)
    torch.cuda.synchronize()
    assert torch.equal(k[4, :, 9], qkv[0, Hs * dh:2 * Hs * dh].view(Hs, dh)) and torch.equal(v[4, :, 9], qkv[0, 2 * Hs * dh:].view(Hs, dh))
    lens, q = _i32(77), _randn(g, 1, Hs * dh, dtype=BF)
    o, lse = ctx.twist_cache_attention_raw(cache, q, lens, 80)
    torch.cuda.synchronize()
    wo, wl, eo, el = _attention_want(k, v, table, q, lens, None, 80, Hs, dh)
    _close(o, wo, eo, U[BF])
    assert ((lse.double().cpu() - wl).abs() <= el).all()


def test_attention_of_parts_that_begin_inside_a_page(lib):
    """A million tokens of a head of one number: the longest parts that there are, none a whole number of pages."""
    Hs, page, n = 128, 256, 1048448
    ctx, g = _ctx(lib, BF, 1), _gen(6)
    pages = -(-n // page)
    k, v = _pools(g, pages, Hs, page, 1, BF)
    table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(1, -1)
    q = _randn(g, 1, Hs, dtype=BF)
    o, lse = ctx.twist_cache_attention_raw(lib.PagedCache(k, v, table), q, _i32(n), n)
    torch.cuda.synchronize()
    for h in range(Hs):
        kk, vv = (p[table[0].long(), h].reshape(-1)[:n].double() for p in (k, v))
        sc = kk * q[0, h].double()
        p = torch.softmax(sc, 0)
        want, wl = (p * vv).sum(), torch.logsumexp(sc, 0)
        # a lane sums 2^20 / (2 parts, 16 waves, 64 lanes) = 512 tokens at most, the joins add 25
        ds = 5 * E24 * sc.abs().max() + 2.0 ** -22
        err = (2 * ds + 2 * 537 * E24) * (p * vv.abs()).sum()
        assert (o[0, h].double() - want).abs() <= U[BF] * want.abs() + err * (1 + U[BF]), h
        assert (lse[0, h].double() - wl).abs() <= ds + 537 * E24 + wl.abs() * 2.0 ** -23, h


# ------------------------------------------------------------------------------------------------ logits
def _logits_want(x, r, V):
    """(result, bound) in 64 bits, column by column from the definition."""
    x = x.double().cpu().clone()
    mag = x.abs()
    at = lambda name, t, default=None: default if r[name] is None else r[name][t].double().item() if r[name].dim() == 1 else r[name][t].cpu()  # noqa: E731
    for t in range(x.shape[0]):
        hist = [] if r["history"] is None else r["history"][t].tolist()
        hist = hist[: max(0, int(at("n_history", t, len(hist))))]
        n_prompt = int(at("n_prompt", t, 0))
        rep, freq, pres = at("repetition", t), at("frequency", t, 0.0), at("presence", t, 0.0)
        times = Counter(hist[max(0, n_prompt):])
        for c in {h for h in hist if 0 <= h < V}:
            n = times[c]
            if rep is not None:
                x[t, c] = x[t, c] / rep if x[t, c] > 0 else x[t, c] * rep
                mag[t, c] = max(mag[t, c], x[t, c].abs())
            if n:
                x[t, c] = x[t, c] - freq * n - pres
                mag[t, c] += abs(freq) * n + abs(pres)
        ids = [] if r["bias_ids"] is None else r["bias_ids"][t].tolist()
        last = {c: i for i, c in enumerate(ids[: max(0, int(at("n_bias", t, len(ids))))]) if 0 <= c < V}
        values = [] if r["bias_values"] is None else r["bias_values"][t].double().tolist()
        for c, i in last.items():
            x[t, c] += values[i]
            mag[t, c] += abs(values[i])
        if r["allowed"] is not None:
            w = r["allowed"][t].cpu().numpy().view(np.uint32)
            bit = torch.tensor(np.unpackbits(w.view(np.uint8), bitorder="little")[:V].astype(bool))
            x[t, ~bit] = -INF
    return x, 6 * E24 * mag


def _rules(g, T, V, hist=0, nb=0, allow=1.0, penalties=True, span=None, prompt=True):
    r = dict.fromkeys(("history", "n_history", "n_prompt", "repetition", "frequency", "presence", "bias_ids", "bias_values", "n_bias", "allowed"))
    ints = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda", dtype=torch.int32)  # noqa: E731
    if hist:
        r["history"] = ints(-2, span or V + 2, T, hist)                       # ids outside the vocabulary among them
        r["n_history"] = ints(-1, hist + 3, T)
        r["n_prompt"] = ints(-1, hist + 2, T) if prompt else None
        if penalties:
            r["repetition"] = 0.7 + torch.rand(T, generator=g, device="cuda")
            r["frequency"] = torch.rand(T, generator=g, device="cuda") - 0.3
            r["presence"] = torch.rand(T, generator=g, device="cuda")
    if nb:
        r["bias_ids"] = ints(-2, min(V + 2, 3 * nb), T, nb)                   # the same id twice among them
        r["bias_values"] = 3 * torch.randn((T, nb), generator=g, device="cuda")
        r["n_bias"] = ints(-1, nb + 3, T)
    if allow < 1:
        words = (V + 31) // 32 + 1
        on = torch.rand((T, words, 32), generator=g, device="cuda") < allow
        bits = (on.long() << torch.arange(32, device="cuda")).sum(-1)
        r["allowed"] = torch.where(bits >= 2 ** 31, bits - 2 ** 32, bits).to(torch.int32)
        r["allowed"][T // 2] = 0                                              # a row that nothing is allowed in
    return r


def _check_logits(lib, dtype, T, V, seed=0, pad=0, opad=0, **kw):
    g = _gen(seed + V)
    ctx = _ctx(lib, dtype, 64, vocab=V)
    x = _randn(g, T, V + pad, dtype=dtype, scale=3.0)[:, :V]
    r = _rules(g, T, V, **kw)
    out = torch.full((T, V + opad), 7.0, device="cuda")
    want, bound = _logits_want(x, r, V)
    before = x.clone()
    ctx.twist_logits_raw(x, lib.LogitRules(**r), out[:, :V])
    torch.cuda.synchronize()
    got = out[:, :V].double().cpu()
    assert torch.equal(torch.isinf(got), torch.isinf(want)) and torch.equal(x, before) and (out[:, V:] == 7).all()
    on = ~torch.isinf(want)
    assert ((got - want).abs()[on] <= bound[on]).all(), float((got - want).abs()[on].max())


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T,V", [(1, 1), (3, 31), (2, 33), (1, 4096), (2, 4097), (3, 8190), (2, 50257), (5, 1003)])
def test_logits_rules(lib, dtype, T, V):
    _check_logits(lib, dtype, T, V, hist=200, nb=40, allow=0.4)
    _check_logits(lib, dtype, T, V, hist=300, span=7)                  # few tokens very often
    _check_logits(lib, dtype, T, V, seed=1)                            # no rule at all: a copy in fp32


@pytest.mark.parametrize("dtype", [BF, F32])
def test_logits_single_rules_and_strides(lib, dtype):
    for pad, opad in ((0, 0), (7, 0), (5, 3), (8, 8), (6, 6), (3, 7)):
        _check_logits(lib, dtype, 3, 5000, pad=pad, opad=opad, hist=50, nb=1, allow=0.9)
        _check_logits(lib, dtype, 3, 5003, pad=pad, opad=opad, nb=300)
        _check_logits(lib, dtype, 3, 5005, pad=pad, opad=opad, allow=0.5)
    _check_logits(lib, dtype, 4, 700, hist=1, prompt=False)
    _check_logits(lib, dtype, 4, 700, hist=5000, span=700)
    _check_logits(lib, dtype, 4, 700, hist=60, penalties=False)
    _check_logits(lib, dtype, 2, 9001, hist=70000, nb=600)             # lists that are longer than 16 bits count
    _check_logits(lib, dtype, 1, 9001, hist=20, nb=40000, allow=0.5)


def test_logits_in_place_and_of_no_number(lib):
    V = 3001
    ctx, g = _ctx(lib, F32, 64, vocab=V), _gen(4)
    x = _randn(g, 2, V)
    x[0, 5], x[0, 6], x[1, 7], x[1, 8] = NAN, INF, -INF, NAN
    r = _rules(g, 2, V, hist=100, allow=0.999)
    r["allowed"][:] = -1
    r["allowed"][1, 0] = ~(1 << 8)                                     # a NaN that the mask takes out
    r["history"][:] = 4 + torch.arange(100, device="cuda", dtype=torch.int32) % 6
    r["n_history"][:], r["n_prompt"][:] = 100, 50
    rules = lib.LogitRules(**r)
    out = ctx.twist_logits_raw(x, rules)
    same = ctx.twist_logits_raw(x, rules, out=x)
    torch.cuda.synchronize()
    assert same is x and torch.equal(torch.nan_to_num(x, nan=123.0), torch.nan_to_num(out, nan=123.0))
    assert torch.isnan(out[0, 5]) and out[0, 6] == INF and out[1, 7] == -INF and out[1, 8] == -INF
    assert int(torch.isnan(out).sum()) == 1 and int(torch.isinf(out).sum()) == 3
