"""Calls of the sequence and logit operators that their documentation allows and that are easily
forgotten."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _tb():
    from paper_2604_12891_amd import binding as tb
    return tb


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1, 3, 700])
def test_segments_of_an_empty_array(n, dtype):
    """No task has a candidate: an array without entries (whose address is NULL), all segments empty."""
    tb, K = _tb(), 5
    x = torch.empty(0, dtype=dtype, device="cuda")
    offs = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    r = tb.logprobs(x, torch.zeros(n, dtype=torch.int32, device="cuda"), K, seg_offsets=offs)
    assert torch.isnan(r["logp"]).all() and not r["entropy"].any()
    assert (r["top"] == -1).all() and (r["top_logp"] == -float("inf")).all()
    top, val = r["top"], torch.zeros(n, K, device="cuda")
    for grad in (True, False):
        d = tb.distill_topk(x, top, val, seg_offsets=offs, grad=grad)
        assert d["loss"].shape == (n,) and not d["loss"].any()
        assert d["grad"].shape == (0,) if grad else d["grad"] is None
    # the same with entries that belong to none of them
    x = torch.randn(9, device="cuda").to(dtype)
    d = tb.distill_topk(x, top, val, seg_offsets=offs + 4, max_len=1, grad=False)
    assert not d["loss"].any()
    assert torch.equal(tb.logprobs(x, K=K, seg_offsets=offs + 4, max_len=1)["top"], r["top"])
