"""Calls of token generation as a caller may make them, beside the kernels' own cases: buffers with gaps."""
import pytest
import torch

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
