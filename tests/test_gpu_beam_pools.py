"""The reordering of states (tcl_beam_reorder) at the limits of one launch."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_the_largest_states_in_many_pools():
    """64 pools of states of 2^31 bytes, 2^24 pieces in all, are more than one launch takes. (One pool's memory stands for all: the
    same copy 64 times.)"""
    from paper_2604_12891_amd import binding as tb
    print("reorder: 64 pools of 2 x 2^31 bytes", flush=True)
    pool = torch.empty(2, 1 << 31, dtype=torch.uint8, device="cuda")
    words = pool.view(torch.int64).view(-1)
    torch.arange(words.numel(), out=words)
    other = torch.zeros(2, 5, device="cuda")
    other[1] = 3.0
    slots = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    new = tb.beam_reorder(torch.tensor([[0, 0]], dtype=torch.int32, device="cuda"), slots, [pool] * 64 + [other])
    assert new.tolist() == [[1, 0]]
    assert torch.equal(pool[0], pool[1]) and words[0].item() == words.numel() // 2 and (other == 3.0).all()
    # nothing to move
    words[0] = 7
    new = tb.beam_reorder(torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"), slots, [other] + [pool] * 64)
    assert new.tolist() == [[0, 1]] and words[0].item() == 7 and words[words.numel() // 2].item() == words.numel() // 2
