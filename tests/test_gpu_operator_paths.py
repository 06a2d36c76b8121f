"""Sizes at which the sequence and logit operators run in another way than at those of
test_gpu_sequence.py and test_gpu_logits.py, against the same oracles."""
import numpy as np
import pytest
import torch

from oracle import logits as ol
from oracle import sequence as osq
from tests.test_gpu_logits import _check_logprobs, _logits
from tests.test_gpu_sequence import (DT, HALF, NAN, _check_scan_grads, _cuda, _near, _np, _offs, _round, _scan_case,
                                     _scan_tensors, _tb)

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


def _conv_case(lens, E, K, dtype, seed):
    rng = np.random.default_rng(seed)
    r, T, n = rng.standard_normal, sum(lens), len(lens)
    return (_round(r((T, E)), dtype), r((E, K)).astype(np.float32), r(E).astype(np.float32),
            _round(r((T, E)), dtype), _round(r((n, K - 1, E)), dtype), _round(r((n, K - 1, E)), dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,E", [(1500, 64), (2300, 37)])
def test_conv_gradients_of_many_short_sequences(n, E, dtype):
    """More sequences than partial sums: a thread takes several tiles, some of them empty."""
    print(f"conv gradients of many n={n} E={E} {dtype}", flush=True)
    lens = np.random.default_rng(n).integers(0, 6, n).tolist()
    lens[7], lens[n // 2] = 100, 33
    offs = _offs(lens)
    x, w, b, du, state, dend = _conv_case(lens, E, 4, dtype, E)
    td = DT[dtype]
    g = _tb().ssm_conv_backward(_cuda(x, td), _cuda(w), _cuda(b), _cuda(du, td), _cuda(offs, torch.int32),
                                state=_cuda(state, td), state_grad=_cuda(dend, td))
    r = osq.conv_backward(x, w, b, du, offs, state, dend, chain=600)  # (as above)
    for name in ("dx", "dw", "db", "dstate"):
        _near(name, g[name], r[name], r["bound"][name], HALF["f32" if name in ("dw", "db") else dtype])


@pytest.mark.parametrize("lens,E,dtype", [([16400, 0, 200], 512, "bf16"), ([3, 32900], 512, "f32"),
                                          ([9000, 200], 257, "f32"), ([70, 17100], 257, "bf16")])
def test_conv_of_many_rows(lens, E, dtype):
    """Forward tiles of 16 and 32 rows, vectors and single channels; gradients' tiles longer than 32 rows."""
    print(f"conv of many rows lens={lens} E={E} {dtype}", flush=True)
    K, td, offs = 4, DT[dtype], _offs(lens)
    x, w, b, du, state, dend = _conv_case(lens, E, K, dtype, E)
    X, W, Bv, O, S = _cuda(x, td), _cuda(w), _cuda(b), _cuda(offs, torch.int32), _cuda(state, td)
    end = torch.full(state.shape, NAN, dtype=td, device="cuda")
    u = _tb().ssm_conv(X, W, Bv, O, state=S, state_out=end)
    ref = osq.conv(x, w, b, offs, state)
    _near("u", u, ref["u"], ref["bound"], HALF[dtype])
    assert np.array_equal(_np(end), ref["end"])
    g = _tb().ssm_conv_backward(X, W, Bv, _cuda(du, td), O, state=S, state_grad=_cuda(dend, td))
    r = osq.conv_backward(x, w, b, du, offs, state, dend, chain=600)
    for name in ("dx", "dw", "db", "dstate"):
        _near(name, g[name], r[name], r["bound"][name], HALF["f32" if name in ("dw", "db") else dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,E,N", [([1100, 40], 64, 16), ([2, 2200], 33, 8)])
def test_scan_of_more_chunks_than_are_joined_at_once(lens, E, N, dtype):
    """Long sequences of few channels: 35 to 74 chunks, joined 32 at a time, with states and adjoints
    carried through. Steps of some 3e-3, so that they are not forgotten on the way."""
    print(f"scan of many chunks lens={lens} E={E} N={N} {dtype}", flush=True)
    a = _scan_case(lens, E, N, dtype, 101)
    a["b_dt"] = a["b_dt"] - 3
    offs, T, n = _offs(lens), sum(lens), len(lens)
    rng = np.random.default_rng(E)
    dy, dend = _round(rng.standard_normal((T, E)), dtype), rng.standard_normal((n, E, N)).astype(np.float32)
    k, O, L = _scan_tensors(a, dtype, T), _cuda(offs, torch.int32), max(lens)
    end = torch.full((n, E, N), NAN, device="cuda")
    y = _tb().ssm_scan(offs=O, L=L, state_out=end, **k)
    ref = osq.scan(offs=offs, **a)
    _near("y", y, ref["y"], ref["bound"]["y"], HALF[dtype])
    _near("end", end, ref["end"], ref["bound"]["end"], HALF["f32"])
    g = _tb().ssm_scan_backward(dy=_cuda(dy, DT[dtype]), offs=O, L=L, state_grad=_cuda(dend), **k)
    r = osq.scan_backward(dy=dy, offs=offs, dend=dend, **a)
    _check_scan_grads(g, r, dtype, T, ["du", "ddt", "dz", "dB", "dC", "dA_log", "dD", "db_dt", "dstate"])
    # the bound is that of a comparison: without the carried adjoint the results are outside
    lost = osq.scan_backward(dy=dy, offs=offs, dend=None, **a)
    assert (np.abs(lost["du"] - r["du"]) > r["bound"]["du"] + HALF[dtype] * np.abs(r["du"])).mean() > 0.05


@pytest.mark.parametrize("packed", [True, False])
def test_scan_gradients_of_several_sequences_to_a_workgroup(packed):
    """As for N 16 in fp32: N 8, bf16."""
    n, E, N = 1400, 1500, 8
    print(f"scan gradients, several sequences to a workgroup, packed={packed}", flush=True)
    rng = np.random.default_rng(28)
    lens = rng.integers(0, 4, n).tolist() if packed else [1] * n
    a = _scan_case(lens, E, N, "bf16", 29)
    T, offs = sum(lens), _offs(lens)
    dy, dend = _round(rng.standard_normal((T, E)), "bf16"), rng.standard_normal((n, E, N)).astype(np.float32)
    k = _scan_tensors(a, "bf16", T)
    if packed:
        k.update(offs=_cuda(offs, torch.int32), L=3)
    g = _tb().ssm_scan_backward(dy=_cuda(dy, torch.bfloat16), state_grad=_cuda(dend), **k)
    r = osq.scan_backward(dy=dy, offs=offs, dend=dend, **a)
    _check_scan_grads(g, r, "bf16", T, ["du", "ddt", "dz", "dB", "dC", "dA_log", "dD", "db_dt", "dstate"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "masked", "ties", "nan", "lowest"])
@pytest.mark.parametrize("V,ld,K", [(513, 520, 33), (8192, 8192, 64), (40, 41, 64)])
def test_logprobs_of_many_short_rows_with_many_alternatives(V, ld, K, kind, dtype):
    n = 300
    print(f"logprobs n={n} V={V} K={K} {kind} {dtype}", flush=True)
    rng = np.random.default_rng(V + K)
    x = _logits(rng, n, V, dtype, kind)
    buf = torch.full((n, ld), NAN, dtype=DT[dtype], device="cuda")
    buf[:, :V] = _cuda(x, DT[dtype])
    tok = rng.integers(0, V, n).astype(np.int32)
    got = _tb().logprobs(buf[:, :V], _cuda(tok, torch.int32), K, 0.7)
    _check_logprobs(got, list(x), tok, K, 0.7)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K,threads", [(32, 64), (20, 64), (33, 128), (64, 128)])
def test_logprobs_where_the_list_overflows(K, threads, dtype):
    """Fewer than K threads hold all the high entries of a row, thousands of them: the bound is
    a low entry, and more reach it than the list of four per thread holds."""
    n, V = 300, 8192
    print(f"logprobs overflow K={K} threads={threads} {dtype}", flush=True)
    ve = 4 if dtype == "f32" else 8
    rng = np.random.default_rng(K)
    x = rng.random((n, V)).astype(np.float32)
    x[:, np.arange(V) // ve % threads < K - 2] += 8.0
    x = torch.from_numpy(x).to(DT[dtype]).double().numpy()
    x[1, ::3], x[2, ::2] = np.nan, -np.inf
    x[3] = np.round(x[3])
    got = _tb().logprobs(_cuda(x, DT[dtype]), None, K)
    ref = ol.logprobs(list(x), None, K)
    assert np.array_equal(got["top"].cpu().numpy(), ref["top"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,E,N", [([70, 3, 40], 64, 16), ([300], 65, 8), ([9, 1, 30] * 200, 60, 8)])
def test_scan_gradients_of_steep_steps(lens, E, N, dtype):
    """Steps of 1e-26 to 40: decays of one, of nothing, and, with the last ones' products, between fp32's
    smallest numbers and zero."""
    print(f"scan gradients steep lens={lens[:3]} E={E} N={N} {dtype}", flush=True)
    a = _scan_case(lens, E, N, dtype, 111, steep=True)
    T, n, offs = sum(lens), len(lens), _offs(lens)
    rng = np.random.default_rng(112)
    dy, dend = _round(rng.standard_normal((T, E)), dtype), rng.standard_normal((n, E, N)).astype(np.float32)
    g = _tb().ssm_scan_backward(dy=_cuda(dy, DT[dtype]), offs=_cuda(offs, torch.int32), L=max(lens),
                                state_grad=_cuda(dend), **_scan_tensors(a, dtype, T))
    r = osq.scan_backward(dy=dy, offs=offs, dend=dend, **a)
    _check_scan_grads(g, r, dtype, T, ["du", "ddt", "dz", "dB", "dC", "dA_log", "dD", "db_dt", "dstate"])
