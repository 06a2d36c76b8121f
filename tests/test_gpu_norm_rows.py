"""Layer norm's rows: NaN and infinities stay in their row, and many bf16 rows (tcl_layer_norm*)."""
import numpy as np
import pytest
import torch

from oracle import layer as ol
from tests.test_gpu_norm import DT, HALF, _near

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def _tb():
    from paper_2604_12891_amd import binding as tb
    return tb


# 16, 32, 64 lanes a row, two vectors a lane, workgroups of one, two and four vectors a thread
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [40, 100, 250, 500, 1500, 5000, 9001])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_what_is_no_number_stays_in_its_row(C, bad, dtype):
    tb, rows, hit = _tb(), 70, (0, 33, 69)
    torch.manual_seed(C)
    x, dy = (torch.randn(rows, C, device="cuda").to(DT[dtype]) for _ in range(2))
    w, b = torch.randn(C, device="cuda"), torch.randn(C, device="cuda")
    keep = torch.tensor([r for r in range(rows) if r not in hit], device="cuda")
    y, g = tb.layer_norm(x, w, b), tb.layer_norm_backward(x, w, dy)
    z = x.clone()
    for r, c in zip(hit, (0, C // 2, C - 1)):
        z[r, c] = bad
    y2, g2 = tb.layer_norm(z, w, b), tb.layer_norm_backward(z, w, dy)
    for got, want in ((y2, y), (g2["dx"], g["dx"])):
        assert torch.equal(got[keep], want[keep])
        assert got[list(hit)].isnan().all()  # the row's mean is none, and all its results with it
    assert g2["dw"].isnan().all() and torch.equal(g2["db"], g["db"])
    # in dy: of its row's dx all, of the sums its column's
    d = dy.clone()
    d[33, C // 2] = bad
    g2 = tb.layer_norm_backward(x, w, d)
    rest = torch.arange(C, device="cuda") != C // 2
    others = torch.arange(rows, device="cuda") != 33
    assert torch.equal(g2["dx"][others], g["dx"][others]) and not g2["dx"][33].isfinite().any()
    for k in ("dw", "db"):
        assert torch.equal(g2[k][rest], g[k][rest]) and not g2[k][C // 2].isfinite()


@pytest.mark.parametrize("rows,C", [(5000, 40), (9000, 256), (2100, 2056), (1300, 5120), (1100, 9001)])
def test_many_bf16_rows(rows, C):
    """More rows than workgroups; the same bits every time."""
    print(f"norm rows={rows} C={C} bf16", flush=True)
    rng = np.random.default_rng(C)
    x, dy = (torch.from_numpy(rng.standard_normal((rows, C)).astype(np.float32)).bfloat16() for _ in range(2))
    w = rng.standard_normal(C).astype(np.float32)
    X, DY, W = x.cuda(), dy.cuda(), torch.from_numpy(w).cuda()
    x, dy = x.double().numpy(), dy.double().numpy()
    r = ol.layer_norm(x, w)
    _near("y", _tb().layer_norm(X, W), r["y"], r["bound"], HALF["bf16"])
    g, r = _tb().layer_norm_backward(X, W, DY), ol.layer_norm_backward(x, w, dy)
    _near("dx", g["dx"], r["dx"], r["bound"]["dx"], HALF["bf16"])
    for name in ("dw", "db"):
        _near(name, g[name], r[name], r["bound"][name], HALF["f32"])
    again = _tb().layer_norm_backward(X, W, DY)
    assert all(torch.equal(g[k], again[k]) for k in g)
