"""Beam selection (tcl_beam_select) among rows whose scores hardly differ: rows of the same logits give equal scores wherever
they start in memory and however they are read, so that the lower row comes first."""
import numpy as np
import pytest
import torch

from oracle import search as osr

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _select(*args, **kw):
    from paper_2604_12891_amd import binding as tb
    return tb.beam_select(*args, **kw)


# rows whole on one workgroup, in parts, on a wavefront; every start in a 16-byte vector, by odd widths
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G,W,V,K", [(20, 8, 4001, 16), (20, 8, 16001, 16), (6, 8, 50001, 16), (1, 16, 131073, 20), (520, 4, 2503, 8),
                                     (40, 4, 77, 8)])
def test_rows_of_the_same_logits(G, W, V, K, dtype):
    print(f"same rows G={G} W={W} V={V} K={K} {dtype}", flush=True)
    rng = np.random.default_rng(V)
    x = torch.from_numpy(2.5 * rng.standard_normal((G, 1, V))).to(DT[dtype]).expand(G, W, V).reshape(G * W, V)
    score = np.repeat(-10 * rng.random((G, 1)), W, 1).astype(np.float32)
    buf = torch.zeros(G * W * V + 1, dtype=DT[dtype], device="cuda")
    X = buf[1:].view(G * W, V)
    X.copy_(x)
    r = _select(X, torch.from_numpy(score).cuda(), K, temperature=0.7)
    ref = osr.beam_select(x.double().numpy(), score, K, temperature=0.7)
    assert np.array_equal(r["parent"].cpu().numpy(), ref["parent"])
    assert np.array_equal(r["token"].cpu().numpy(), ref["token"])
    r = r["score"].cpu().numpy().reshape(G, -1)
    assert (r[:, :W] == r[:, :1]).all()  # (the best token of every beam)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G,W,V", [(10, 4, 4001), (4, 4, 50001)])
def test_scores_a_step_apart(G, W, V, dtype):
    """Rows of the same logits in another order, whose sums differ by their roundings alone: beams 2^-18 apart, nine times what
    a score of so many logits may be off (4e-7), come in the order of their own scores."""
    rng = np.random.default_rng(V)
    x = np.repeat(2.5 * rng.standard_normal((G, 1, V)), W, 1)
    x[:, :, 7] = 14.0  # every beam's best token, far in front of its others
    best = np.empty((G, W), np.int64)
    for g in range(G):
        for w in range(W):
            x[g, w] = rng.permutation(x[g, w])
            best[g, w] = x[g, w].argmax()
    score = (2.0 ** -18 * rng.permuted(np.tile(np.arange(W), (G, 1)), axis=1)).astype(np.float32) - np.float32(1.0)
    r = _select(torch.from_numpy(x).to(DT[dtype]).reshape(G * W, V).cuda(), torch.from_numpy(score).cuda(), W)
    want = np.argsort(-score, axis=1)
    assert np.array_equal(r["parent"].cpu().numpy(), want + W * np.arange(G)[:, None])
    assert np.array_equal(r["token"].cpu().numpy(), np.take_along_axis(best, want, 1))
