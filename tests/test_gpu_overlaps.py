"""Results right beside what their call reads are none that overlap."""
import numpy as np
import pytest
import torch

from oracle import search as osr

pytestmark = pytest.mark.gpu


def test_selection_beside_its_scores():
    """Scores, ended beams, parents, tokens and new scores one behind the other in one buffer."""
    from paper_2604_12891_amd import binding as tb
    G, W, V, K = 5, 3, 400, 6
    rng = np.random.default_rng(0)
    x = rng.standard_normal((G * W, V)).astype(np.float32)
    score = -rng.random((G, W)).astype(np.float32)
    ended = np.full((G, W), -1, np.int32)
    ended[1, 2] = 9
    buf = torch.empty(2 * G * W + 3 * G * K, dtype=torch.int32, device="cuda")
    parts = torch.split(buf, [G * K, G * W, G * K, G * W, G * K])
    parts[1].view(torch.float32).copy_(torch.from_numpy(score.reshape(-1)))
    parts[3].copy_(torch.from_numpy(ended.reshape(-1)))
    X, ws = torch.from_numpy(x).cuda(), tb.beam_select_workspace(G, W, V, K)
    p = [t.data_ptr() for t in parts]
    tb.check(tb.lib().tcl_beam_select(0, G, W, V, X.data_ptr(), V, 1.0, p[1], p[3], K, p[0], p[2], p[4], ws.data_ptr(),
                                      ws.numel(), torch.cuda.current_stream().cuda_stream))
    ref = osr.beam_select(x, score, K, ended)
    assert np.array_equal(parts[0].view(G, K).cpu().numpy(), ref["parent"])
    assert np.array_equal(parts[2].view(G, K).cpu().numpy(), ref["token"])
    assert np.array_equal(parts[1].view(torch.float32).cpu().numpy(), score.reshape(-1))


@pytest.mark.parametrize("kind", ["columns", "columns of the next row", "rows between", "strides", "one row", "behind"])
def test_norm_beside_its_rows(kind):
    """Rows and results in one buffer: columns beside each other, rows between each other's, two strides."""
    from paper_2604_12891_amd import binding as tb
    rows, C = 37, 40
    flat = torch.randn(40000, device="cuda")
    x0, ldx, y0, ldy = {"columns": (0, 100, 40, 100), "columns of the next row": (50, 90, 90, 90), "rows between": (0, 160, 80, 160),
                        "strides": (0, 100, 50, 200), "one row": (10, 999, 50, 40), "behind": (0, 50, 36 * 50 + 40, 41)}[kind]
    if kind == "one row":
        rows = 1
    x, y = (torch.as_strided(flat, (rows, C), (ld, 1), at) for at, ld in ((x0, ldx), (y0, ldy)))
    before, want = x.clone(), tb.layer_norm(x.clone())
    tb.layer_norm(x, out=y)
    assert torch.equal(y, want) and torch.equal(x, before)
    dy = torch.randn(rows, C, device="cuda")
    want = tb.layer_norm_backward(x, None, dy)
    got = tb.layer_norm_backward(x, None, dy, out=dict(dx=y))
    assert all(torch.equal(got[k], want[k]) for k in want) and torch.equal(x, before)


def test_norm_in_place_is_refused():
    from paper_2604_12891_amd import binding as tb
    x = torch.randn(5, 40, device="cuda")
    with pytest.raises(tb.TclError):
        tb.layer_norm(x, out=x)
    with pytest.raises(tb.TclError):
        tb.layer_norm_backward(x, None, x, out=dict(dx=x))
