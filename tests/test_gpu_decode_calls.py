"""Calls of token generation as a caller may make them, beside the kernels' own cases: buffers with gaps, prompts near the limits of a launch."""
import pytest
import torch

import test_gpu_decode as decode
from helpers import within
from test_gpu_generate import Deployed

pytestmark = pytest.mark.gpu


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
