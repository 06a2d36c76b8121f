"""Layer norm and its gradients (tcl_layer_norm*) against the fp64 oracle (oracle/layer.py), within
its bound on fp32 arithmetic and half a step of the result's type."""
import numpy as np
import pytest
import torch

from oracle import layer as ol

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
NAN = float("nan")


def _tb():
    from paper_2604_12891_amd import binding as tb
    return tb


def _near(name, got, ref, bound, half):
    got = got.double().cpu().numpy()
    tol = bound + half * (np.abs(ref) + bound) + 1e-37
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (name, int(bad.sum()), float(np.nanmax(np.abs(got - ref) / tol)), np.argwhere(bad)[:4])


def _rows(a, dtype, ld, first, fill=NAN):
    """a's rows in a buffer of leading dimension ld, from element `first` on; the rest is fill."""
    n, C = a.shape
    buf = torch.full((first + n * ld + 8,), fill, dtype=dtype, device="cuda")
    v = buf[first:first + n * ld].view(n, ld)[:, :C]
    v.copy_(torch.from_numpy(a))
    return buf, v


# every kernel: 16, 32 and 64 lanes a row, two vectors a lane, workgroups of one, two and four vectors a
# thread, at both ends of their ranges in both types; widths that end inside a vector, rows that start anywhere
SIZES = [(1, 1), (5, 3), (33, 64), (7, 65), (3, 129), (40, 256), (9, 257), (5, 511), (3, 513), (2, 1031), (6, 2048),
         (3, 4097), (2, 8192), (3, 8201), (1, 16384), (2, 16383)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,C", SIZES)
@pytest.mark.parametrize("pad,first", [(0, 0), (5, 3)])
def test_norm_and_gradients(rows, C, pad, first, dtype):
    print(f"norm rows={rows} C={C} pad={pad} first={first} {dtype}", flush=True)
    rng = np.random.default_rng(C)
    td = DT[dtype]
    rnd = lambda a: torch.from_numpy(a).to(td).double().numpy()
    x, dy = rnd(rng.standard_normal((rows, C)) * 2 + 3.0), rnd(rng.standard_normal((rows, C)))
    w, b = rng.standard_normal(C).astype(np.float32), rng.standard_normal(C).astype(np.float32)
    _, X = _rows(x, td, C + pad, first)
    _, DY = _rows(dy, td, C + pad, first + 1)
    W, B = torch.from_numpy(w).cuda(), torch.from_numpy(b).cuda()
    for ww, bb in ((w, b), (None, None)):
        buf, out = _rows(np.zeros((rows, C)), td, C + pad, first, 7.0)
        y = _tb().layer_norm(X, None if ww is None else W, None if bb is None else B, out=out)
        r = ol.layer_norm(x, ww, bb)
        _near("y", y, r["y"], r["bound"], HALF[dtype])
        assert (buf == 7.0).sum() >= buf.numel() - rows * C  # nothing beside the rows is written
        buf, dx = _rows(np.zeros((rows, C)), td, C + pad, first, 7.0)
        g = _tb().layer_norm_backward(X, None if ww is None else W, DY, out=dict(dx=dx))
        r = ol.layer_norm_backward(x, ww, dy)
        _near("dx", g["dx"], r["dx"], r["bound"]["dx"], HALF[dtype])
        for name in ("dw", "db"):
            _near(name, g[name], r[name], r["bound"][name], HALF["f32"])
        assert (buf == 7.0).sum() >= buf.numel() - rows * C


@pytest.mark.parametrize("rows,C", [(5000, 40), (3000, 256), (2100, 2056), (1100, 5120), (600, 9001)])
def test_many_rows(rows, C):
    """More rows than workgroups; the same bits every time."""
    print(f"norm rows={rows} C={C}", flush=True)
    rng = np.random.default_rng(C)
    x, dy = rng.standard_normal((rows, C)).astype(np.float32), rng.standard_normal((rows, C)).astype(np.float32)
    w = rng.standard_normal(C).astype(np.float32)
    X, DY, W = (torch.from_numpy(a).cuda() for a in (x, dy, w))
    r = ol.layer_norm(x, w)
    _near("y", _tb().layer_norm(X, W), r["y"], r["bound"], HALF["f32"])
    g, r = _tb().layer_norm_backward(X, W, DY), ol.layer_norm_backward(x, w, dy)
    for name in ("dx", "dw", "db"):
        _near(name, g[name], r[name], r["bound"][name], HALF["f32"])
    again = _tb().layer_norm_backward(X, W, DY)
    assert all(torch.equal(g[k], again[k]) for k in g)


def test_rows_of_equal_values_and_levels():
    """A row of one value is its bias (the variance is 0, not the rounding of a difference); a large level
    does not eat the deviations."""
    x = torch.full((4, 1000), 1234.5, device="cuda")
    b = torch.arange(1000.0, device="cuda")
    assert torch.equal(_tb().layer_norm(x, None, b), b.expand(4, -1))
    rng = np.random.default_rng(0)
    x = (1000.0 + rng.standard_normal((6, 777))).astype(np.float32)
    r = ol.layer_norm(x)
    _near("y", _tb().layer_norm(torch.from_numpy(x).cuda()), r["y"], r["bound"], HALF["f32"])


def test_no_rows():
    for t in (torch.float32, torch.bfloat16):
        x = torch.empty(0, 12, dtype=t, device="cuda")
        assert _tb().layer_norm(x).shape == (0, 12)
        g = _tb().layer_norm_backward(x, None, x)
        assert g["dx"].shape == (0, 12) and not g["dw"].any() and not g["db"].any()


def test_gradients_are_differences():
    """Of the kernel's own forward pass: the directional difference of y . dy. With a step of 2^-6 of values of order
    1, third derivatives of order 10 give 10 step^2 / 6, and the roundings of y (2^-24 of 4, 600 of them with
    random signs) 2^-24 4 sqrt(600) / step."""
    torch.manual_seed(0)
    x, dy, w, dirn = (torch.randn(6, 100, device="cuda") for _ in range(4))
    w = w[0].contiguous()
    step = 2.0 ** -6
    dirn = dirn / dirn.norm()
    f = lambda s: (_tb().layer_norm(x + s * step * dirn, w).double() * dy.double()).sum()
    want = ((f(1.0) - f(-1.0)) / (2 * step)).item()
    got = (_tb().layer_norm_backward(x, w, dy)["dx"].double() * dirn.double()).sum().item()
    assert abs(got - want) < 10 * step ** 2 / 6 + 2.0 ** -24 * 4 * 600 ** 0.5 / step


def test_streams_and_graph():
    """On a stream of its own, and captured with its workspace: replays on new inputs give the eager bits."""
    tb = _tb()
    torch.manual_seed(1)
    x, dy, w = torch.randn(300, 520, device="cuda"), torch.randn(300, 520, device="cuda"), torch.randn(520, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y = tb.layer_norm(x, w, stream=s)
    g = tb.layer_norm_backward(x, w, dy, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, tb.layer_norm(x, w))
    ws, out = tb.layer_norm_workspace(torch.float32, 300, 520), {k: torch.empty_like(v) for k, v in g.items()}
    yo = torch.empty_like(y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tb.layer_norm(x, w, out=yo)
        tb.layer_norm_backward(x, w, dy, workspace=ws, out=out)
    for k in range(4):
        x.copy_(torch.randn_like(x) * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        want = tb.layer_norm_backward(x, w, dy)
        assert torch.equal(yo, tb.layer_norm(x, w)) and all(torch.equal(out[n], want[n]) for n in want)
