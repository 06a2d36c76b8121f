"""Sizes at which the sequence and logit operators run in another way than at those of
test_gpu_sequence.py and test_gpu_logits.py, against the same oracles."""
import numpy as np
import pytest
import torch

from oracle import sequence as osq
from tests.test_gpu_sequence import DT, HALF, _cuda, _near, _np, _offs, _round, _tb

pytestmark = pytest.mark.gpu
EPS = osq.EPS


@pytest.mark.parametrize("n", [1, 900, 1023])
def test_parameter_gradients_of_one_long_sequence_among_empty_ones(n):
    """Convolution gradients of 60,000 equal tokens: dw and db are 60,000 times one term, whatever the other
    sequences are. A running fp32 sum of that many is off by some 5e-4; sums of at most 512
    terms each (eight even shares of 59 tokens), and of 1,152 such parts in sixteens, are off by
    512 + 72 + 16 roundings at most. The term itself, du SiLU'(x w + b) x with x w + b in (0, 1), is off
    by EPS_ACT (1 + 1) sigmoid / SiLU' < 6.4e-6 and ten roundings."""
    T, E = 60_000, 64
    print(f"conv gradients of one long sequence, n={n}", flush=True)
    rng = np.random.default_rng(n)
    x, du, w, b = (0.25 + 0.5 * rng.random(E).astype(np.float32) for _ in range(4))
    b = 0.4 * b
    offs = np.zeros(n + 1, np.int32)
    offs[n // 2 + 1:] = T
    X, DU = (_cuda(np.tile(v, (T, 1))) for v in (x, du))
    g = _tb().ssm_conv_backward(X, _cuda(w[:, None]), _cuda(b), DU, _cuda(offs, torch.int32))
    x, du, w, b = (v.astype(np.float64) for v in (x, du, w, b))
    s = osq.sigmoid(b + w * x)
    t = du * s * (1 + (b + w * x) * (1 - s))
    rel = 6.4e-6 + (512 + 72 + 16 + 10) * EPS
    assert (np.abs(_np(g["db"]) / (T * t) - 1) <= rel).all()
    assert (np.abs(_np(g["dw"])[:, 0] / (T * t * x) - 1) <= rel).all()
    assert (np.abs(_np(g["dx"]) / (t * w) - 1) <= 6.4e-6 + 10 * EPS).all()
