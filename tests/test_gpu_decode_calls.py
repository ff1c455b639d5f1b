"""Calls of token generation as a caller may make them, beside the kernels' own cases: buffers with gaps, prompts near the limits of a launch, batches of
sequences with a few rows each, prompts in large tables, logits at any place, tables in others."""
import numpy as np
import pytest
import torch

import synth_inputs as si
import test_gpu_decode as decode
from helpers import rel_fro_of_numbers, to_numpy, within
from test_gpu_generate import Deployed, _bound

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def numbers_only(monkeypatch):
    monkeypatch.setattr(decode, "_close", within)


def test_decode_refuses_storage_with_gaps(lib):
    """Strided views that pass every size check: nothing is written behind or between their elements."""
    d = Deployed(lib, "gpt_bf16", 2, 64)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    n = d.ctx.twist_decode_workspace_bytes(d.sub, d.pages, 2, 64)
    ws, big = (torch.full((2 * b,), 0xaa, dtype=torch.uint8, device="cuda") for b in (n, d.cache.numel()))
    for cache, work in ((d.cache, ws[::2]), (d.cache, ws.view(-1, 512)[:, :256]), (big[::2], ws), (big.view(-1, 512)[:, :256], ws)):
        with pytest.raises(lib.TwistError):
            d.ctx.twist_subnet_decode(d.sub, i32([1, 2]), i32([1, 1]), 64, d.pages, cache, work)
    torch.cuda.synchronize()
    assert (ws == 0xaa).all() and (big == 0xaa).all() and (d.cache == 0xff).all()


def test_a_prompt_of_more_rows_and_parts_than_workgroups_of_a_launch(lib):
    """4096 rows of 104 heads over ten parts (pages of a token): tiles, where a workgroup a row would be 2^22 of them and more."""
    T, Hs, dh, top = 4096, 104, 8, 20470
    ctx, g = decode._ctx(lib, decode.BF, dh), decode._gen(21)
    k, v = decode._pools(g, top, Hs, 1, dh, decode.BF)
    table = torch.randperm(top, generator=g, device="cuda").to(torch.int32).view(1, -1)
    q = decode._randn(g, T, Hs * dh, dtype=decode.BF)
    lens = (torch.arange(T, device="cuda") + top - T + 1).to(torch.int32)
    seq = torch.zeros(T, dtype=torch.int32, device="cuda")
    cache = lib.PagedCache(k, v, table)
    assert T * Hs * -(-top // 2047) >= 2 ** 22 and ctx.twist_cache_attention_floats(cache, T, top) == T * Hs * 10 * (dh + 2)
    o, lse = ctx.twist_cache_attention_raw(cache, q, lens, top, seq=seq)
    torch.cuda.synchronize()
    rows = torch.tensor([0, 1500, 4095], device="cuda")
    wo, wl, eo, el = decode._attention_want(k, v, table, q[rows], lens[rows], seq[rows], top, Hs, dh)
    within(o[rows], wo, eo, decode.U[decode.BF])
    assert ((lse[rows].double().cpu() - wl).abs() <= el).all()
    assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()


def _batch(S, r, top, order):
    """Lengths and sequences of S times r rows, one length of each sequence near the top, and what a batch holds beside them."""
    ends = [max(r, top - (top * s) // S) for s in range(S)]
    rows = [(ends[s] - r + 1 + i, s) for s in range(S) for i in range(r)]
    if order == "mixed":                                               # no two neighbours of one sequence: a tile holds 16 groups
        rows = [rows[s * r + i] for i in range(r) for s in range(S)]
    elif order == "ragged":                                            # runs of 1 to 2 r - 1 rows across the tiles, unused rows between them
        rows = [x for i, x in enumerate(rows) if i % (2 * r) or i % 5]
        for at in (3, 17, 40):
            rows[at:at] = [(0, rows[at][1]), (-1, rows[at][1]), (5, -1), (7, S)]
    return [n for n, _ in rows], [s for _, s in rows]


@pytest.mark.parametrize("order", ["runs", "mixed", "ragged"])
@pytest.mark.parametrize("Hs,dh,S,r,top", [(8, 128, 40, 2, 600), (8, 96, 40, 3, 500), (12, 64, 32, 5, 310), (16, 40, 40, 4, 300), (16, 80, 24, 4, 280), (16, 32, 30, 6, 300),  # workgroups of 4 waves
                                           (8, 128, 24, 8, 250), (4, 64, 20, 7, 1000), (3, 40, 40, 4, 1800), (2, 96, 30, 12, 500), (1, 32, 36, 15, 2000), (4, 256, 20, 3, 600)])
def test_attention_of_a_few_rows_of_many_sequences(lib, Hs, dh, S, r, top, order):
    """bf16 tiles that several workgroups share, each taking every second to eighth group of their rows."""
    lens, seq = _batch(S, r, top, order)
    decode._check_attention(lib, decode.BF, Hs, dh, 16, lens, seq, n_seqs=S, max_len=top, max_pages=-(-top // 16), holes=[(1, 0), (2, 3), (S - 1, 1)])


@pytest.mark.parametrize("order", ["runs", "mixed", "ragged"])
@pytest.mark.parametrize("Hs,dh,S,r,top", [(8, 128, 20, 4, 520), (12, 64, 24, 3, 700), (12, 40, 24, 8, 400), (8, 80, 20, 6, 700), (4, 32, 40, 12, 800), (4, 256, 12, 5, 600)])
def test_fp32_attention_of_a_few_rows_of_many_sequences(lib, Hs, dh, S, r, top, order):
    lens, seq = _batch(S, r, top, order)
    decode._check_attention(lib, decode.F32, Hs, dh, 16, lens, seq, n_seqs=S, max_len=top, max_pages=-(-top // 16), holes=[(1, 0), (2, 3), (S - 1, 1)])


@pytest.mark.parametrize("dtype,dh", [(decode.BF, 128), (decode.F32, 64)])
def test_attention_of_a_few_rows_of_many_long_sequences(lib, dtype, dh):
    """The same where sequences are cut into parts, the last of which few of them reach."""
    S, r, top = 40, 3, 4300
    lens, seq = _batch(S, r, top, "runs")
    lens = [n if s in (0, 1, 2, 20) else min(n, 90 + n % 7) for n, s in zip(lens, seq)]
    decode._check_attention(lib, dtype, 4, dh, 64, lens, seq, n_seqs=S, max_len=top, max_pages=-(-top // 64), holes=[(1, 0), (0, 40)] + [(2, i) for i in range(16, 40)])


@pytest.mark.parametrize("dtype", [decode.BF, decode.F32])
@pytest.mark.parametrize("n_seqs", [1, 8, 40, 200, 600])
def test_a_prompt_in_a_table_of_any_size(lib, dtype, n_seqs):
    """Kernels are chosen by the table's rows: one prompt of 400 rows through each form of them, and through its own row of the table alone."""
    Hs, dh, T, top, page = 4, 64, 400, 800, 16
    ctx, g = decode._ctx(lib, dtype, dh), decode._gen(31)
    n_pages = top // page + 5
    k, v = decode._pools(g, n_pages, Hs, page, dh, dtype)
    at = n_seqs // 2
    table = torch.full((n_seqs, top // page), -1, dtype=torch.int32, device="cuda")
    table[at] = torch.randperm(n_pages, generator=g, device="cuda")[: top // page].to(torch.int32)
    q = decode._randn(g, T, Hs * dh, dtype=dtype, scale=1.5)
    lens = (torch.arange(T, device="cuda") + top - T + 1).to(torch.int32)
    seq = torch.full((T,), at, dtype=torch.int32, device="cuda")
    rows = torch.arange(0, T, 37, device="cuda")
    for pages, which in ((table, seq), (table[at:at + 1], torch.zeros_like(seq))):
        o, lse = ctx.twist_cache_attention_raw(lib.PagedCache(k, v, pages), q, lens, top, seq=which)
        torch.cuda.synchronize()
        wo, wl, eo, el = decode._attention_want(k, v, pages, q[rows], lens[rows], which[rows], top, Hs, dh)
        within(o[rows], wo, eo, decode.U[dtype])
        assert ((lse[rows].double().cpu() - wl).abs() <= el).all()
        assert torch.isfinite(o.float()).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("name", ["llama_f32_um", "llama_bf16", "gpt_bf16"])
def test_a_prompt_through_its_own_row_of_the_table(lib, name):
    """A prompt of one of 40 sequences through a table of that row alone, then tokens through the whole table: one cache, the oracle's logits."""
    d = Deployed(lib, name, 40, 64)
    ids = si.tokens_uniform(d.cfg.vocab, 1, 64, 5)[0][:52]
    s, n = 23, 48
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    own = lib.Pages(d.table[s:s + 1], d.pages.n_pages, d.page)
    assert d.ctx.twist_cache_bytes(d.sub, own) == d.cache.numel()
    ws = torch.full((d.ctx.twist_decode_workspace_bytes(d.sub, own, n, 64),), 0xff, dtype=torch.uint8, device="cuda")
    got = list(to_numpy(d.ctx.twist_subnet_decode(d.sub, i32(ids[:n].tolist()), i32(list(range(1, n + 1))), 64, own, d.cache, ws, seq=i32([0] * n))))
    for p in range(n, len(ids)):
        got.append(to_numpy(d.step([3, int(ids[p])], [1, p + 1], [7, s], 64))[1])
    assert rel_fro_of_numbers(np.stack(got), d.want(ids)) <= _bound(d.cfg)


@pytest.mark.parametrize("name", ["gpt_bf16", "llama_f32_um", "ragged_f32", "llama_bf16_um"])
@pytest.mark.parametrize("T", [3, 40])
def test_logits_at_any_place(lib, name, T):
    """Rows of logits of any stride, from any element on: the same numbers up to rounding, nothing beside them."""
    d = Deployed(lib, name, T, 16)
    V, dt = d.cfg.vocab, d.ctx.torch_dtype
    step = lambda out: d.step([t % V for t in range(T)], [1] * T, max_len=16, logits=out)  # noqa: E731
    base = step(None).clone()
    assert torch.isfinite(base.float()).all()
    for ldl, at in ((V, 0), (V + 1, 1), (V + 5, 3), (V + 8 - V % 8, 2)):
        buf = torch.full((T * ldl + 8,), 7.0, dtype=dt, device="cuda")
        out = buf.as_strided((T, V), (ldl, 1), at)
        step(out)
        torch.cuda.synchronize()
        assert rel_fro_of_numbers(to_numpy(out), to_numpy(base)) <= _bound(d.cfg)
        out.fill_(7.0)
        assert (buf == 7).all()


@pytest.mark.parametrize("dtype", [decode.BF, decode.F32])
def test_tables_that_are_part_of_others(lib, dtype):
    """A table whose rows lie further apart than they are long, or that begins inside one: what lies between is not the sequence's."""
    Hs, dh, page, S = 3, 64, 16, 5
    ctx, g = decode._ctx(lib, dtype, dh, rope=True), decode._gen(17)
    k, v = decode._pools(g, 64, Hs, page, dh, dtype)
    whole = torch.randint(0, 64, (S + 2, 12), generator=g, device="cuda", dtype=torch.int32)
    whole[1:6, 2:10] = torch.randperm(64, generator=g, device="cuda")[:40].view(5, 8).to(torch.int32)
    part = whole[1:6, 2:10]
    qkv, lens = decode._randn(g, S, 3 * Hs * dh, dtype=dtype), decode._i32(1, 17, 100, 128, 129)       # the last: beyond its eight pages
    q = torch.zeros((S, Hs * dh), dtype=k.dtype, device="cuda")
    wq, wk, wv, eq, ek = decode._append_want(k, v, part, qkv, lens, None, q, Hs, dh, True, 10000.0)
    cache = lib.PagedCache(k, v, part)
    ctx.twist_cache_append_raw(cache, qkv, lens, q_out=q)
    torch.cuda.synchronize()
    within(q, wq, eq, decode.U[dtype])
    within(k, wk, ek, torch.where(ek > 0, decode.U[dtype], 0.0))
    assert torch.equal(v.double().cpu(), wv)
    for seq in (None, decode._i32(4, 4, 3, 2, 2)):
        o, lse = ctx.twist_cache_attention_raw(cache, q, lens, 200, seq=seq)
        torch.cuda.synchronize()
        wo, wl, eo, el = decode._attention_want(k, v, part, q, lens, seq, 200, Hs, dh)
        within(o, wo, eo, decode.U[dtype])
        assert ((lse.double().cpu() - wl).abs() <= el).all()
