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


@pytest.mark.parametrize("n,V", [(3, 900), (2, 70001), (600, 150)])
def test_what_the_student_masks(n, V):
    """A student's mask where the teacher has a probability: an infinite loss, unless that is below
    fp32's smallest normal number; finite gradients either way. Rows without a teacher are zeros whatever the
    student's logits are; NaN and +inf show in all others."""
    tb, inf, nan = _tb(), float("inf"), float("nan")
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.zeros(n, V, device="cuda", dtype=dtype)
        x[:, 7] = -inf
        top = torch.tensor([[3, 7]], dtype=torch.int32, device="cuda").repeat(n, 1)

        def loss(*teacher, x=x, top=top):
            r = tb.distill_topk(x, top, torch.tensor([teacher], device="cuda").repeat(n, 1))
            return r["loss"].double().cpu().numpy(), r["grad"]

        for low, want in ((-80.0, inf), (-100.0, np.log(V - 1)), (-inf, np.log(V - 1))):
            got, grad = loss(0.0, low)
            # log of a sum of ones: a few roundings of log V < 16
            assert (got == want).all() if want == inf else (np.abs(got - want) < 16 * 8 * 2.0 ** -24).all(), (low, got)
            assert torch.isfinite(grad).all()
        for v in (nan, inf):
            bad = x.clone()
            bad[0, 1] = v
            got, grad = loss(0.0, -1.0, x=bad)
            assert np.isnan(got[0]) and (got[1:] == inf).all()
            assert torch.isnan(grad[0]).any() and torch.isfinite(grad[1:]).all()
            got, grad = loss(0.0, v)
            assert np.isnan(got).all()
            got, grad = loss(0.0, -1.0, x=bad, top=torch.full_like(top, -1))  # no teacher
            assert not got.any() and not grad.any()


def test_the_readme_example():
    """What README.md shows, on small tensors."""
    tcl = _tb()
    T, n, E, N, V, K = 12, 3, 16, 16, 40, 5
    r = lambda *s: torch.randn(*s, device="cuda")
    x, x1, w, b, dt, dt1, z, z1 = r(T, E), r(n, E), r(E, 4), r(E), r(T, E), r(n, E), r(T, E), r(n, E)
    A_log, B, C, B1, C1, D, b_dt, dy = r(E, N), r(T, N), r(T, N), r(n, N), r(n, N), r(E), r(E), r(T, E)
    offs, longest = torch.tensor([0, 5, 5, 12], dtype=torch.int32, device="cuda"), 7
    conv_state, state = torch.empty(n, 3, E, device="cuda"), torch.empty(n, E, N, device="cuda")
    teacher_logits, logits, tokens = r(T, V), r(T, V), torch.zeros(T, dtype=torch.int32, device="cuda")
    u = tcl.ssm_conv(x, w, b, offs=offs, state_out=conv_state)
    y = tcl.ssm_scan(u, dt, A_log, B, C, D=D, z=z, b_dt=b_dt, offs=offs, L=longest, state_out=state)
    u1 = tcl.ssm_conv(x1, w, b, state=conv_state, state_out=conv_state)
    y1 = tcl.ssm_scan(u1, dt1, A_log, B1, C1, D=D, z=z1, b_dt=b_dt, state=state, state_out=state)
    t = tcl.logprobs(teacher_logits, tokens, K=K)
    d = tcl.distill_topk(logits, t["top"], t["top_logp"])
    g = tcl.ssm_scan_backward(u, dt, A_log, B, C, dy, D=D, z=z, b_dt=b_dt, offs=offs, L=longest)
    assert y.shape == (T, E) and y1.shape == (n, E) and d["grad"].shape == (T, V) and g["du"].shape == (T, E)
    for v in (u, y, u1, y1, conv_state, state, d["loss"], d["grad"], g["du"], g["dA_log"]):
        assert torch.isfinite(v).all()
