"""What the binding of token generation refuses by itself (no GPU needed)."""
import pytest
import torch


@pytest.mark.parametrize("what", ["cache", "workspace"])
def test_storage_is_one_run_of_memory(what):
    """The library writes every byte behind the address: of a buffer with gaps these are another's."""
    import paper_2511_03983_amd as tw
    storage, at = tw.binding._storage, torch.zeros(64, dtype=torch.uint8)      # (GPU -1: the CPU)
    assert storage(at, what, -1) == (at.data_ptr(), 64)
    assert storage(torch.zeros((4, 8), dtype=torch.bfloat16), what, -1)[1] == 64
    for bad in (at[::2], at.view(8, 8)[:, :4], at.view(8, 8).t(), at[:1].expand(64)):
        with pytest.raises(tw.TwistError, match=what):
            storage(bad, what, -1)
    with pytest.raises(tw.TwistError, match=what):
        storage(at, what, 0)
