"""The gated delta rule where many value heads share a key head, on few chunks and on many, against the fp64 oracle
(oracle/layer.py).

Tolerance: that of test_gpu_delta.py on fp32 arithmetic, and of a bf16 result the norm of one rounding, taken of the oracle's
result itself: roundings of numbers that differ by fp32's errors have the same norm but for the sample's spread, which over 512
results or more (a relative deviation of at most 0.9 of a squared rounding's mean each) stays below 5 x 0.9 / sqrt(512) / 2 = 10%."""
import numpy as np
import pytest
import torch

from oracle import layer as ol
from tests.test_gpu_delta import DT, GRADS, _case, _gpu, head_errors, tolerance

pytestmark = pytest.mark.gpu


def _near(name, got, ref, tol, dtype):
    got = got.double().cpu().numpy()
    assert got.shape == ref.shape and np.isfinite(got).all(), name
    if dtype == "bf16":
        tol = tol + 1.1 * head_errors(torch.from_numpy(ref).bfloat16().double().numpy(), ref)
    e = head_errors(got, ref)
    assert (e <= tol).all(), (name, (e / tol).max(), e.max())


# few chunks: the value heads spread over workgroups; 256 chunks and more of a key head: one for all of them
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,Hk,H,Dk,Dv", [([130, 70], 1, 8, 64, 64), ([200], 1, 16, 128, 40), ([90, 65, 300], 2, 10, 24, 128),
                                             ([4200, 4101, 4099, 4300], 1, 5, 16, 8), ([2100] * 4, 2, 8, 8, 16)])
def test_value_heads_of_a_key_head(lens, Hk, H, Dk, Dv, dtype):
    print(f"delta heads {len(lens)} x {lens[0]} Hk={Hk} H={H} Dk={Dk} Dv={Dv} {dtype}", flush=True)
    from paper_2604_12891_amd import binding as tb
    T, n, rng = sum(lens), len(lens), np.random.default_rng(H)
    a = _case(lens, Hk, H, Dk, Dv, dtype, H + Dk)
    x, offs = _gpu(a, dtype, False, spare=0), torch.from_numpy(a["offs"]).cuda()
    S = torch.from_numpy(a["state"]).float().cuda()
    end = torch.empty_like(S)
    o = tb.delta_rule(**x, offs=offs, state=S, state_out=end)
    r, tol = ol.delta_rule(**a), tolerance(Dk, lens)
    _near("o", o, r["o"], tol, dtype)
    _near("end", end, r["end"], tol, "f32")
    do = torch.from_numpy(rng.standard_normal((T, H, Dv))).to(DT[dtype])
    dend = rng.standard_normal((n, H, Dk, Dv)).astype(np.float32)
    g = tb.delta_rule_backward(**x, do=do.cuda(), offs=offs, state=S, state_grad=torch.from_numpy(dend).cuda())
    r = ol.delta_rule_backward(do=do.double().numpy(), dend=dend, **a)
    for name in GRADS:
        _near(name, g[name], r[name], tol, dtype if name in ("dq", "dk", "dv") else "f32")
