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
