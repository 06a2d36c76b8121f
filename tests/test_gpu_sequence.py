"""The causal convolution and the selective scan with carried states
(tcl_ssm_conv, tcl_ssm_scan and their gradients) against the fp64 oracle
(oracle/sequence.py), which also gives the bound on fp32 arithmetic that
every comparison uses, plus half a step of the result's type where that is
bf16 (2^-8 of the value) or fp32 (2^-24)."""
import numpy as np
import pytest
import torch

from oracle import sequence as osq

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
NAN = float("nan")


def _tb():
    from paper_2604_12891_amd import binding as tb
    return tb


def _np(t):
    return t.double().cpu().numpy()


def _near(name, got, ref, bound, half):
    got = _np(got)
    tol = bound + half * (np.abs(ref) + bound) + 1e-37
    bad = ~(np.abs(got - ref) <= tol)
    assert not bad.any(), (name, int(bad.sum()), float(np.nanmax(np.abs(got - ref) / tol)), np.argwhere(bad)[:4])


def _rows(a, dtype, rows, ld=None, fill=NAN):
    """a's rows in a [rows, ld] buffer, the rest of it `fill` (NaN in what is read, where nothing
    may depend on it); a view of a's width."""
    a = np.asarray(a)
    buf = torch.full((rows, ld or a.shape[1]), fill, dtype=dtype, device="cuda")
    buf[:a.shape[0], :a.shape[1]] = torch.from_numpy(a).to("cuda", dtype)
    return buf[:, :a.shape[1]]


def _round(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DT[dtype]).double().numpy()


def _offs(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _cuda(a, dtype=torch.float32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)


# ---------------------------------------------------------------- convolution

CONV = [([1, 0, 25, 7, 2, 3], 64, 64), ([33, 1, 64, 0, 31], 100, 104), ([5], 3, 7), ([200, 129], 256, 264),
        ([0, 0], 8, 8), ([1] * 70, 40, 40)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [1, 2, 3, 4])
@pytest.mark.parametrize("lens,E,ld", CONV)
def test_conv_and_gradients(lens, E, ld, K, dtype):
    print(f"conv lens={lens} E={E} ld={ld} K={K} {dtype}", flush=True)
    rng = np.random.default_rng(E + K)
    offs, T, n, td = _offs(lens), sum(lens), len(lens), DT[dtype]
    x, du = _round(rng.standard_normal((T, E)), dtype), _round(rng.standard_normal((T, E)), dtype)
    w, b = rng.standard_normal((E, K)).astype(np.float32), rng.standard_normal(E).astype(np.float32)
    state, dend = (_round(rng.standard_normal((n, K - 1, E)), dtype) for _ in range(2))
    tb = _tb()
    rows = T + 3  # three rows that nobody owns
    X, DU = _rows(x, td, rows, ld), _rows(du, td, rows, ld)
    W, Bv, O = _cuda(w), _cuda(b), _cuda(offs, torch.int32)
    for st, bias in [(None, None), (state, b)]:
        S = _cuda(st, td)
        end = torch.full((n, K - 1, E), NAN, dtype=td, device="cuda")
        out = torch.full((rows, ld), 7.0, dtype=td, device="cuda")
        tb.ssm_conv(X, W, Bv if bias is not None else None, O, state=S, state_out=end, out=out[:, :E])
        ref = osq.conv(x, w, bias, offs, st)
        _near("u", out[:T, :E], ref["u"], ref["bound"], HALF[dtype])
        assert (out[T:] == 7.0).all() and (out[:, E:] == 7.0).all()
        assert np.array_equal(_np(end), ref["end"])
        if S is not None:  # in place
            tb.ssm_conv(X, W, Bv, O, state=S, state_out=S)
            assert torch.equal(S, end)
            S = _cuda(st, td)
        DE = None if st is None else _cuda(dend, td)
        g = tb.ssm_conv_backward(X, W, Bv if bias is not None else None, DU, O, state=S, state_grad=DE)
        r = osq.conv_backward(x, w, bias, du, offs, st, None if st is None else dend)
        _near("dx", g["dx"][:T], r["dx"], r["bound"]["dx"], HALF[dtype])
        _near("dw", g["dw"], r["dw"], r["bound"]["dw"], HALF["f32"])
        _near("db", g["db"], r["db"], r["bound"]["db"], HALF["f32"])
        if st is not None:
            _near("dstate", g["dstate"], r["dstate"], r["bound"]["dstate"], HALF[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,E,K", [(1, 1, 4), (7, 100, 2), (64, 512, 4), (300, 96, 3), (2, 64, 1)])
def test_conv_tokens_with_slots(n, E, K, dtype):
    """One token per sequence, states in a pool larger than the batch, some
    sequences without one; a second token continues the first."""
    print(f"conv tokens n={n} E={E} K={K} {dtype}", flush=True)
    rng = np.random.default_rng(n)
    td, pool = DT[dtype], n + 5
    slots = rng.permutation(pool)[:n].astype(np.int32)
    slots[n // 2] = -1
    if n > 3:
        slots[0] = pool  # past the pool: none
    x = [_round(rng.standard_normal((n, E)), dtype) for _ in range(2)]
    w, b = rng.standard_normal((E, K)).astype(np.float32), rng.standard_normal(E).astype(np.float32)
    st = _round(rng.standard_normal((pool, K - 1, E)), dtype)
    live = (slots >= 0) & (slots < pool)
    start = np.where(live[:, None, None], st[np.where(live, slots, 0)], 0.0)
    S, one = _cuda(st, td), np.arange(n + 1)
    want = st.copy()
    for t in range(2):
        u = _tb().ssm_conv(_cuda(x[t], td), _cuda(w), _cuda(b), state=S, state_out=S, slots=_cuda(slots, torch.int32))
        ref = osq.conv(x[t], w, b, one, start)
        _near("u", u, ref["u"], ref["bound"], HALF[dtype])
        start = np.where(live[:, None, None], ref["end"], 0.0)  # without a state it starts from zeros again
        want[slots[live]] = ref["end"][live]
        assert np.array_equal(_np(S), want)


# ---------------------------------------------------------------- selective scan

def _scan_case(lens, E, N, dtype, seed, full=True, steep=False):
    rng = np.random.default_rng(seed)
    T, n = sum(lens), len(lens)
    r = rng.standard_normal
    a = dict(u=_round(r((T, E)), dtype), dt=_round(r((T, E)), dtype), B=_round(r((T, N)), dtype),
             C=_round(r((T, N)), dtype), A_log=(np.log(np.arange(1, N + 1)) + 0.3 * r((E, N))).astype(np.float32))
    if steep:  # steps from none to states that are forgotten at once
        a["dt"] = _round(rng.choice([-60.0, -8.0, 0.0, 5.0, 40.0], (T, E)), dtype)
    if full:
        a.update(z=_round(2 * r((T, E)), dtype), D=r(E).astype(np.float32), b_dt=(r(E) - 3).astype(np.float32),
                 state=r((n, E, N)).astype(np.float32))
    return a


def _scan_tensors(a, dtype, rows, ld=None):
    """The case's arguments on the GPU; B and C are columns of one buffer."""
    td, N = DT[dtype], a["A_log"].shape[1]
    k = {name: _rows(a[name], td, rows, ld) for name in ("u", "dt", "z") if a.get(name) is not None}
    bc = torch.full((rows, 2 * N + 1), NAN, dtype=td, device="cuda")
    T = a["u"].shape[0]
    bc[:T, 1:N + 1], bc[:T, N + 1:] = _cuda(a["B"], td), _cuda(a["C"], td)
    k.update(B=bc[:, 1:N + 1], C=bc[:, N + 1:], A_log=_cuda(a["A_log"]), D=_cuda(a.get("D")), b_dt=_cuda(a.get("b_dt")),
             state=_cuda(a.get("state")))
    return k


SCAN = [([1, 0, 25, 7, 2], 64, 64), ([33, 1, 64, 0, 31, 65], 100, 105), ([5], 3, 3), ([300], 64, 64),
        ([257, 0, 130, 1], 70, 72), ([0, 0], 8, 8), ([9] * 40, 256, 256), ([40, 70], 513, 520), ([1], 1, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [8, 16])
@pytest.mark.parametrize("full", [True, False])
@pytest.mark.parametrize("lens,E,ld", SCAN)
def test_scan(lens, E, ld, full, N, dtype):
    print(f"scan lens={lens} E={E} ld={ld} N={N} {dtype} full={full}", flush=True)
    a = _scan_case(lens, E, N, dtype, E + N, full)
    offs, T, n = _offs(lens), sum(lens), len(lens)
    rows = T + 2
    k = _scan_tensors(a, dtype, rows, ld)
    end = torch.full((n, E, N), NAN, device="cuda")
    out = torch.full((rows, ld), 7.0, dtype=DT[dtype], device="cuda")
    ref = osq.scan(offs=offs, **a)
    for L in (max(lens), None):  # the bound that is exact, and the one that is not known
        k["offs"] = _cuda(offs, torch.int32)
        _tb().ssm_scan(L=L if L is None else max(L, 1), state_out=end, out=out[:, :E], **k)
        _near("y", out[:T, :E], ref["y"], ref["bound"]["y"], HALF[dtype])
        _near("end", end, ref["end"], ref["bound"]["end"], HALF["f32"])
        assert (out[T:] == 7.0).all() and (out[:, E:] == 7.0).all()
    if full:
        _tb().ssm_scan(L=max(max(lens), 1), state_out=k["state"], **k)  # in place
        _near("end", k["state"], ref["end"], ref["bound"]["end"], HALF["f32"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,E,N", [(300, 450, 16), (1100, 70, 8)])
def test_scan_of_many_sequences(n, E, N, dtype):
    """Batches large enough for one lane per channel, with slots, some sequences empty or
    without a state."""
    print(f"scan many n={n} E={E} N={N} {dtype}", flush=True)
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 12, n).tolist()
    lens[3] = 70
    a = _scan_case(lens, E, N, dtype, n)
    offs, T, pool = _offs(lens), sum(lens), n + 3
    slots = rng.permutation(pool)[:n].astype(np.int32)
    slots[5], slots[6] = -1, pool
    live = (slots >= 0) & (slots < pool)
    a["state"][~live] = 0.0
    k = _scan_tensors(a, dtype, T)
    S = torch.zeros(pool, E, N, device="cuda")
    at = torch.from_numpy(slots[live].astype(np.int64)).cuda()
    S[at] = _cuda(a["state"][live])
    y = _tb().ssm_scan(offs=_cuda(offs, torch.int32), L=70, state_out=S, slots=_cuda(slots, torch.int32),
                       **dict(k, state=S))
    ref = osq.scan(offs=offs, **a)
    _near("y", y, ref["y"], ref["bound"]["y"], HALF[dtype])
    _near("end", S[at], ref["end"][live], ref["bound"]["end"][live], HALF["f32"])
    S[at] = 0.0
    assert not S.any()  # the other places of the pool are as they were


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,E,N", [([70, 3, 40], 64, 16), ([300], 65, 8)])
def test_scan_of_steep_steps(lens, E, N, dtype):
    """Steps of 1e-26 to 40: states that stay, states that are forgotten."""
    print(f"scan steep lens={lens} E={E} N={N} {dtype}", flush=True)
    a = _scan_case(lens, E, N, dtype, 5, steep=True)
    k = _scan_tensors(a, dtype, sum(lens))
    end = torch.empty(len(lens), E, N, device="cuda")
    y = _tb().ssm_scan(offs=_cuda(_offs(lens), torch.int32), L=max(lens), state_out=end, **k)
    ref = osq.scan(offs=_offs(lens), **a)
    _near("y", y, ref["y"], ref["bound"]["y"], HALF[dtype])
    _near("end", end, ref["end"], ref["bound"]["end"], HALF["f32"])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [8, 16])
@pytest.mark.parametrize("n,E", [(1, 1), (5, 100), (64, 512), (270, 1024), (3, 2050)])
def test_scan_tokens_with_slots(n, E, N, dtype):
    print(f"scan tokens n={n} E={E} N={N} {dtype}", flush=True)
    a = [_scan_case([1] * n, E, N, dtype, n + t) for t in range(2)]
    pool = n + 4
    rng = np.random.default_rng(n)
    slots = rng.permutation(pool)[:n].astype(np.int32)
    slots[n // 2] = -1
    if n > 3:
        slots[0] = pool + 9
    live = (slots >= 0) & (slots < pool)
    st = rng.standard_normal((pool, E, N)).astype(np.float32)
    S, one = _cuda(st), np.arange(n + 1)
    for t in range(2):
        now = _np(S)
        k = dict(a[t], A_log=a[0]["A_log"], state=np.where(live[:, None, None], now[np.where(live, slots, 0)], 0.0))
        g = _scan_tensors(k, dtype, n)
        g["state"] = S
        y = _tb().ssm_scan(state_out=S, slots=_cuda(slots, torch.int32), **g)
        ref = osq.scan(offs=one, **k)
        _near("y", y, ref["y"], ref["bound"]["y"], HALF[dtype])
        got = _np(S)
        _near("end", S[torch.from_numpy(slots[live].astype(np.int64)).cuda()], ref["end"][live],
              ref["bound"]["end"][live], HALF["f32"])
        rest = np.setdiff1d(np.arange(pool), slots[live])
        assert np.array_equal(got[rest], now[rest])


def test_scan_in_chunks_of_a_prompt_and_tokens_is_the_whole():
    """A prompt in two calls and its last tokens one by one, over a pool of
    states, against the whole sequence at once."""
    E, N, T = 128, 16, 150
    a = _scan_case([T], E, N, "f32", 11)
    ref = osq.scan(offs=np.array([0, T]), **a)
    k = _scan_tensors(a, "f32", T)
    S, slots = torch.zeros(3, E, N, device="cuda"), torch.tensor([2], dtype=torch.int32, device="cuda")
    S[2] = k["state"][0]
    ys = []
    for lo, hi in [(0, 97), (97, 147), (147, 148), (148, 149), (149, 150)]:
        part = {m: v[lo:hi] if m in ("u", "dt", "B", "C", "z") else v for m, v in k.items()}
        offs = None if hi - lo == 1 else torch.tensor([0, hi - lo], dtype=torch.int32, device="cuda")
        ys.append(_tb().ssm_scan(offs=offs, state_out=S, slots=slots, **dict(part, state=S)))
    _near("y", torch.cat(ys), ref["y"], ref["bound"]["y"], HALF["f32"])
    _near("end", S[2:], ref["end"], ref["bound"]["end"], HALF["f32"])
    assert not S[:2].any()


def _check_scan_grads(g, r, dtype, T, names):
    for name in names:
        half = HALF[dtype] if name in ("du", "ddt", "dz", "dB", "dC") else HALF["f32"]
        got = g[name][:T] if name in ("du", "ddt", "dz", "dB", "dC") else g[name]
        _near(name, got, r[name], r["bound"][name], half)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [8, 16])
@pytest.mark.parametrize("full", [True, False])
@pytest.mark.parametrize("lens,E,ld", SCAN)
def test_scan_gradients(lens, E, ld, full, N, dtype):
    print(f"scan backward lens={lens} E={E} ld={ld} N={N} {dtype} full={full}", flush=True)
    a = _scan_case(lens, E, N, dtype, E + N + 1, full)
    offs, T, n = _offs(lens), sum(lens), len(lens)
    rng = np.random.default_rng(E)
    dy = _round(rng.standard_normal((T, E)), dtype)
    dend = rng.standard_normal((n, E, N)).astype(np.float32) if full else None
    k = _scan_tensors(a, dtype, T + 2, ld)
    g = _tb().ssm_scan_backward(dy=_rows(dy, DT[dtype], T + 2, ld), offs=_cuda(offs, torch.int32),
                                L=max(max(lens), 1), state_grad=_cuda(dend), **k)
    r = osq.scan_backward(dy=dy, offs=offs, dend=dend, **a)
    names = ["du", "ddt", "dB", "dC", "dA_log", "dD", "db_dt"] + (["dz", "dstate"] if full else [])
    _check_scan_grads(g, r, dtype, T, names)
    assert full or (g["dz"] is None and g["dstate"] is None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_gradients_of_single_tokens(dtype):
    n, E, N = 9, 130, 16
    a = _scan_case([1] * n, E, N, dtype, 3)
    rng = np.random.default_rng(4)
    dy, dend = _round(rng.standard_normal((n, E)), dtype), rng.standard_normal((n, E, N)).astype(np.float32)
    g = _tb().ssm_scan_backward(dy=_cuda(dy, DT[dtype]), state_grad=_cuda(dend), **_scan_tensors(a, dtype, n))
    r = osq.scan_backward(dy=dy, offs=np.arange(n + 1), dend=dend, **a)
    _check_scan_grads(g, r, dtype, n, ["du", "ddt", "dz", "dB", "dC", "dA_log", "dD", "db_dt", "dstate"])


@pytest.mark.parametrize("packed", [True, False])
def test_scan_gradients_of_many_short_sequences(packed):
    """Several sequences to a workgroup, some of them empty."""
    n, E, N = 1400, 1500, 16
    rng = np.random.default_rng(8)
    lens = rng.integers(0, 4, n).tolist() if packed else [1] * n
    a = _scan_case(lens, E, N, "f32", 9)
    T, offs = sum(lens), _offs(lens)
    dy, dend = rng.standard_normal((T, E)).astype(np.float32), rng.standard_normal((n, E, N)).astype(np.float32)
    k = _scan_tensors(a, "f32", T)
    if packed:
        k.update(offs=_cuda(offs, torch.int32), L=3)
    g = _tb().ssm_scan_backward(dy=_cuda(dy), state_grad=_cuda(dend), **k)
    r = osq.scan_backward(dy=dy, offs=offs, dend=dend, **a)
    _check_scan_grads(g, r, "f32", T, ["du", "ddt", "dz", "dB", "dC", "dA_log", "dD", "db_dt", "dstate"])


def test_workspace_covers_single_tokens():
    """As many rows as sequences: the workspace serves the call with offsets and the one without."""
    tb = _tb()
    for n, E in ((3990, 256), (4097, 256), (1400, 1500), (8130, 300), (100, 64)):
        u, bc = torch.zeros(n, E, device="cuda"), torch.zeros(n, 8, device="cuda")
        A = torch.zeros(E, 8, device="cuda")
        ws = tb.ssm_scan_workspace(n, n, E, 8, 1, backward=True)
        guard = torch.full((ws.numel() + 4096,), 255, dtype=torch.uint8, device="cuda")
        for offs in (None, torch.arange(n + 1, dtype=torch.int32, device="cuda")):
            tb.ssm_scan_backward(u, u, A, bc, bc, u, offs=offs, L=1, workspace=guard[:ws.numel()])
        torch.cuda.synchronize()
        assert (guard[ws.numel():] == 255).all(), (n, E)


def test_scan_gradient_is_a_difference():
    """The gradient along one direction of all inputs together against the
    forward operator's own central difference. The loss sums T E = 1,376 terms of size 1 to 10, off by
    some 1e-6 of each: about sqrt(1376) 1e-5 = 4e-4, over a step of 2e-3 0.2, where the gradient's terms
    along the direction have a root sum of squares of some 100 (9 inputs, 15,000 terms of size
    about 1); the difference's third-order term is 1e-6 of that. 1% of it is allowed."""
    E, N, lens = 32, 16, [40, 3]
    a = _scan_case(lens, E, N, "f32", 21)
    rng = np.random.default_rng(22)
    T = sum(lens)
    dy = rng.standard_normal((T, E)).astype(np.float32)
    names = dict(u="du", dt="ddt", B="dB", C="dC", z="dz", A_log="dA_log", D="dD", b_dt="db_dt", state="dstate")
    way = {m: rng.standard_normal(a[m].shape) for m in names}
    tb, offs = _tb(), _cuda(_offs(lens), torch.int32)

    def loss(s):
        k = _scan_tensors({m: a[m] + s * way[m] for m in names}, "f32", T)
        return float((tb.ssm_scan(offs=offs, L=40, **k).double().cpu().numpy() * dy).sum())

    g = tb.ssm_scan_backward(dy=_cuda(dy), offs=offs, L=40, **_scan_tensors(a, "f32", T))
    along = sum((_np(g[names[m]]) * way[m]).sum() for m in names)
    size = np.sqrt(sum(((_np(g[names[m]]) * way[m]) ** 2).sum() for m in names))
    step = 1e-3
    assert abs((loss(step) - loss(-step)) / (2 * step) - along) < 0.01 * size


def test_same_bits_every_time():
    lens, E, N = [300, 17, 129], 320, 16
    a = _scan_case(lens, E, N, "bf16", 31)
    k, offs = _scan_tensors(a, "bf16", sum(lens)), _cuda(_offs(lens), torch.int32)
    dy = torch.ones_like(k["u"])
    one = _tb().ssm_scan_backward(dy=dy, offs=offs, L=300, **k)
    for _ in range(3):
        two = _tb().ssm_scan_backward(dy=dy, offs=offs, L=300, **k)
        for name in one:
            assert torch.equal(one[name], two[name]), name


def test_captured_graphs_share_a_workspace():
    """Two graphs over one workspace, replayed in turn on another stream than the one they
    were made on, on new inputs, with eager calls between."""
    tb = _tb()
    lens, E, N, n = [200, 90, 400], 192, 16, 3
    T, offs = sum(lens), _cuda(_offs(lens), torch.int32)
    cases = [_scan_tensors(_scan_case(lens, E, N, "f32", 41 + i), "f32", T) for i in range(2)]
    ws = tb.ssm_scan_workspace(n, T, E, N, 400, backward=True)
    fws = tb.ssm_scan_workspace(n, T, E, N, 400)
    assert fws.numel() > 0
    dy = torch.randn(T, E, device="cuda")

    def both(k):
        end = torch.empty(n, E, N, device="cuda")
        y = tb.ssm_scan(offs=offs, L=400, state_out=end, workspace=fws, **k)
        return dict(tb.ssm_scan_backward(dy=dy, offs=offs, L=400, workspace=ws, **k), y=y, end=end)

    both(cases[0])
    torch.cuda.synchronize()
    graphs, outs = [], []
    for k in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(both(k))
        graphs.append(g)
    side = torch.cuda.Stream()
    for step in range(3):
        for k in cases:
            for m in ("u", "dt", "z"):
                k[m].copy_(torch.randn(T, E, device="cuda"))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for g in graphs:
                g.replay()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for k, o in zip(cases, outs):
            for name, v in both(k).items():
                assert torch.equal(v, o[name]), (step, name)


def test_far_rows():
    """Rows whose byte offsets pass 32 bits: single tokens in the last rows of a
    wide pool, and a long leading dimension."""
    tb, E, N = _tb(), 64, 16
    n = 40
    wide = torch.zeros(n, 60_000_000, dtype=torch.bfloat16, device="cuda")  # 4.8 GB, row 36 on past 4 GiB
    a = _scan_case([n], E, N, "bf16", 51)
    k = _scan_tensors(a, "bf16", n)
    wide[:, :E] = k["u"]
    offs = _cuda(np.array([0, n]), torch.int32)
    ref = osq.scan(offs=np.array([0, n]), **a)
    out = torch.zeros(n, 60_000_000, dtype=torch.bfloat16, device="cuda")
    tb.ssm_scan(offs=offs, L=n, out=out[:, :E], **dict(k, u=wide[:, :E]))
    _near("y", out[:, :E], ref["y"], ref["bound"]["y"], HALF["bf16"])
    del out
    w = torch.randn(E, 4, device="cuda")
    want = tb.ssm_conv(k["u"].contiguous(), w, offs=offs)
    assert torch.equal(tb.ssm_conv(wide[:, :E], w, offs=offs), want)
    del wide
    slots = 1_100_000  # states of 4 KB: 4.5 GB
    pool = torch.zeros(slots, E, N, device="cuda")
    at = torch.tensor([slots - 1, 0, slots - 2, 5], dtype=torch.int32, device="cuda")
    start = torch.randn(4, E, N, device="cuda")
    pool[at.long()] = start
    t = {m: v[:4] if m in ("u", "dt", "B", "C", "z") else v for m, v in k.items()}
    y = tb.ssm_scan(state_out=pool, slots=at, **dict(t, state=pool))
    end = torch.empty_like(start)
    assert torch.equal(y, tb.ssm_scan(state_out=end, **dict(t, state=start)))
    assert torch.equal(pool[at.long()], end)


def test_empty_sequences_alone():
    """Nothing but empty sequences, wider than one workgroup's channels: states and their
    gradients pass through, the parameters' gradients are zero."""
    tb, E, N, n = _tb(), 600, 16, 3
    none = torch.empty(0, E, device="cuda")
    bc = torch.empty(0, N, device="cuda")
    offs = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    A, st, ge = torch.zeros(E, N, device="cuda"), torch.randn(n, E, N, device="cuda"), torch.randn(n, E, N, device="cuda")
    end = torch.empty_like(st)
    assert tb.ssm_scan(none, none, A, bc, bc, offs=offs, state=st, state_out=end).shape == (0, E)
    assert torch.equal(end, st)
    g = tb.ssm_scan_backward(none, none, A, bc, bc, none, offs=offs, state=st, state_grad=ge)
    assert torch.equal(g["dstate"], ge) and not g["dA_log"].any() and not g["dD"].any() and not g["db_dt"].any()
    w, cs, cg = torch.randn(E, 4, device="cuda"), torch.randn(n, 3, E, device="cuda"), torch.randn(n, 3, E, device="cuda")
    ce = torch.empty_like(cs)
    tb.ssm_conv(none, w, offs=offs, state=cs, state_out=ce)
    assert torch.equal(ce, cs)
    g = tb.ssm_conv_backward(none, w, None, none, offs=offs, state=cs, state_grad=cg)
    assert torch.equal(g["dstate"], cg) and not g["dw"].any() and not g["db"].any()
    nobody = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert tb.ssm_scan(none, none, A, bc, bc, offs=nobody).shape == (0, E)
    assert tb.ssm_conv(none, w).shape == (0, E)


def test_more_tokens_than_a_grid_dimension():
    """Single tokens of more sequences than 4 x 65,535."""
    tb, E, N, n = _tb(), 8, 8, 270_001
    u, dt, B, C = (torch.randn(n, k, device="cuda") for k in (E, E, N, N))
    A = torch.zeros(E, N, device="cuda")
    end = torch.full((n, E, N), NAN, device="cuda")
    y = tb.ssm_scan(u, dt, A, B, C, state_out=end)
    d = torch.nn.functional.softplus(dt.double())
    s = (d * u.double())[:, :, None] * B.double()[:, None, :]
    # softplus within EPS_ACT, two products
    assert ((end.double() - s).abs() <= (osq.EPS_ACT + 3 * osq.EPS) * s.abs() + 1e-37).all()
    ref = (s * C.double()[:, None, :]).sum(-1)
    size = (s * C.double()[:, None, :]).abs().sum(-1)
    assert ((y.double() - ref).abs() <= (osq.EPS_ACT + (N + 4) * osq.EPS) * size + 1e-37).all()


def test_gradients_into_the_callers_tensors():
    """Rows that no sequence owns stay as they were in tensors the caller gives, wide ones among them."""
    tb, E, N, lens = _tb(), 70, 16, [33, 5]
    T, rows = 38, 44
    a = _scan_case(lens, E, N, "f32", 61)
    k = _scan_tensors(a, "f32", rows)
    offs = _cuda(_offs(lens), torch.int32)
    dy = _rows(np.ones((T, E)), torch.float32, rows)
    want = tb.ssm_scan_backward(dy=dy, offs=offs, L=33, **k)
    wide = torch.full((rows, 100), 7.0, device="cuda")
    out = dict(du=wide[:, :E], ddt=torch.zeros(rows, E, device="cuda"), dB=torch.zeros(rows, N, device="cuda"))
    got = tb.ssm_scan_backward(dy=dy, offs=offs, L=33, out=out, **k)
    assert got["du"] is out["du"] and (wide[T:] == 7.0).all() and (wide[:, E:] == 7.0).all()
    assert not out["ddt"][T:].any() and not out["dB"][T:].any()
    for name in want:
        part = slice(0, T) if name in ("du", "ddt", "dz", "dB", "dC") else slice(None)
        assert torch.equal(got[name][part], want[name][part]), name
    w = torch.randn(E, 4, device="cuda")
    x, du = k["u"], _rows(np.ones((T, E)), torch.float32, rows)
    dx = torch.full((rows, E), 7.0, device="cuda")
    g = tb.ssm_conv_backward(x, w, None, du, offs=offs, out=dict(dx=dx))
    assert g["dx"] is dx and (dx[T:] == 7.0).all() and torch.isfinite(g["dw"]).all()
    with pytest.raises(ValueError, match="dx"):
        tb.ssm_conv_backward(x, w, None, du, offs=offs, out=dict(dx=dx[:, :3]))


def test_on_a_stream_of_its_own():
    """Under a given stream results and workspaces belong to that stream: calls there with work
    and allocations on the current stream in between give what they give alone."""
    tb, E, N, lens = _tb(), 256, 16, [700, 300]
    T, offs = 1000, _cuda(_offs([700, 300]), torch.int32)
    k = _scan_tensors(_scan_case(lens, E, N, "f32", 71), "f32", T)
    dy = torch.randn(T, E, device="cuda")
    w = torch.randn(E, 4, device="cuda")
    y0 = tb.ssm_scan(offs=offs, L=700, **k)
    g0 = tb.ssm_scan_backward(dy=dy, offs=offs, L=700, **k)
    c0 = tb.ssm_conv_backward(k["u"], w, None, dy, offs=offs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        y = tb.ssm_scan(offs=offs, L=700, stream=side, **k)
        g = tb.ssm_scan_backward(dy=dy, offs=offs, L=700, stream=side, **k)
        c = tb.ssm_conv_backward(k["u"], w, None, dy, offs=offs, stream=side)
        noise = [torch.full((1 << 20,), NAN, device="cuda") for _ in range(8)]
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(y, y0)
        for a, b in ((g, g0), (c, c0)):
            for name in b:
                assert b[name] is None or torch.equal(a[name], b[name]), name
        del noise


def test_results_that_are_not_wanted():
    """NULL for every gradient that may be: the others are what they are with it."""
    tb, E, N, lens = _tb(), 96, 16, [70, 5]
    from paper_2604_12891_amd.binding import lib
    T, n = 75, 2
    offs = _cuda(_offs(lens), torch.int32)
    k = _scan_tensors(_scan_case(lens, E, N, "f32", 81), "f32", T)
    dy = torch.randn(T, E, device="cuda")
    k = dict(k, z=None, state=torch.randn(n, E, N, device="cuda"))
    full = tb.ssm_scan_backward(dy=dy, offs=offs, L=70, **k)
    _, a = tb._scan_args(*(k.get(m) for m in ("u", "dt", "A_log", "B", "C", "D", "z", "b_dt")), offs, n, 70, k["state"])
    r = {m: torch.empty_like(full[m]) for m in ("du", "ddt", "dB", "dC", "dA_log")}
    g = tb._PACK_GRADS.pack(r["du"].data_ptr(), E, r["ddt"].data_ptr(), E, r["dB"].data_ptr(), N, r["dC"].data_ptr(), N,
                            0, 0, r["dA_log"].data_ptr(), 0, 0, 0)
    ws = tb.ssm_scan_workspace(n, T, E, N, 70, backward=True)
    s = torch.cuda.current_stream().cuda_stream
    assert lib().tcl_ssm_scan_backward(a, dy.data_ptr(), E, None, g, ws.data_ptr(), ws.numel(), s) == 0
    for m in r:
        assert torch.equal(r[m], full[m]), m
    w, b = torch.randn(E, 4, device="cuda"), torch.randn(E, device="cuda")
    state = torch.randn(n, 3, E, device="cuda")
    full = tb.ssm_conv_backward(k["u"], w, b, dy, offs=offs, state=state)
    a = tb._conv_args(k["u"], w, b, offs, n, state)
    dx, dw = torch.empty(T, E, device="cuda"), torch.empty(E, 4, device="cuda")
    ws = tb.ssm_conv_workspace(n, T, E, 4)
    assert lib().tcl_ssm_conv_backward(a, dy.data_ptr(), E, None, dx.data_ptr(), E, dw.data_ptr(), None, None,
                                       ws.data_ptr(), ws.numel(), s) == 0
    assert torch.equal(dx, full["dx"]) and torch.equal(dw, full["dw"])


def test_one_state_read_by_several_sequences():
    """Without an output pool sequences may start from the same place: a common prefix."""
    tb, E, N, n = _tb(), 128, 16, 6
    pool, cpool = torch.randn(3, E, N, device="cuda"), torch.randn(3, 3, E, device="cuda")
    slots = torch.tensor([1, 1, 2, 1, -1, 3], dtype=torch.int32, device="cuda")
    A, w = torch.zeros(E, N, device="cuda"), torch.randn(E, 4, device="cuda")
    u, dt, x = (torch.randn(n, E, device="cuda") for _ in range(3))
    B, C = (torch.randn(n, N, device="cuda") for _ in range(2))
    offs = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    start = torch.stack([pool[1], pool[1], pool[2], pool[1], pool[0] * 0, pool[0] * 0])
    cstart = torch.stack([cpool[1], cpool[1], cpool[2], cpool[1], cpool[0] * 0, cpool[0] * 0])
    for o in (None, offs):
        assert torch.equal(tb.ssm_scan(u, dt, A, B, C, offs=o, state=pool, slots=slots),
                           tb.ssm_scan(u, dt, A, B, C, offs=o, state=start))
        assert torch.equal(tb.ssm_conv(x, w, offs=o, state=cpool, slots=slots), tb.ssm_conv(x, w, offs=o, state=cstart))


def test_captured_generation():
    """A prompt and its tokens with states updated in place, and the convolution's gradients, in one
    graph: every replay goes on from the states that the one before left, as eager calls do."""
    tb, E, N, lens = _tb(), 192, 16, [40, 3, 9]
    n, T, offs = 3, 52, _cuda(_offs([40, 3, 9]), torch.int32)
    k = _scan_tensors(_scan_case(lens, E, N, "bf16", 91), "bf16", T)
    one = {m: k[m][:n].contiguous() if m in ("u", "dt", "B", "C", "z") else k[m] for m in k}
    w = torch.randn(E, 4, device="cuda")
    ws = tb.ssm_conv_workspace(n, T, E, 4)

    def run(S, P):
        u = tb.ssm_conv(k["u"], w, offs=offs, state=P, state_out=P)
        y = tb.ssm_scan(offs=offs, L=40, **dict(k, u=u, state=S, state_out=S))
        v = tb.ssm_conv(one["u"], w, state=P, state_out=P)
        z = tb.ssm_scan(**dict(one, u=v, state=S, state_out=S))
        g = tb.ssm_conv_backward(k["u"], w, None, y, offs=offs, workspace=ws)
        return [y, z, g["dx"], g["dw"]]

    def states():
        return torch.zeros(n, E, N, device="cuda"), torch.zeros(n, 3, E, dtype=torch.bfloat16, device="cuda")

    S, P = states()
    run(S, P)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(S, P)
    S.zero_()
    P.zero_()
    eS, eP = states()
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = run(eS, eP)
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert torch.equal(S, eS) and torch.equal(P, eP)


def test_two_calls_at_once():
    """Calls on two streams, each with its own workspace, give what they give alone."""
    tb, E, N, lens = _tb(), 256, 16, [900, 100]
    T, offs = 1000, _cuda(_offs([900, 100]), torch.int32)
    cases = [_scan_tensors(_scan_case(lens, E, N, "f32", 95 + i), "f32", T) for i in range(2)]
    dy = torch.randn(T, E, device="cuda")

    def both(k, stream=None):
        g = tb.ssm_scan_backward(dy=dy, offs=offs, L=900, stream=stream, **k)
        return dict(g, y=tb.ssm_scan(offs=offs, L=900, stream=stream, **k))

    want = [both(k) for k in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        got.append([both(k, s) for k, s in zip(cases, streams)])
    torch.cuda.synchronize()
    for pair in got:
        for g, r in zip(pair, want):
            for name in r:
                assert r[name] is None or torch.equal(g[name], r[name]), name


@pytest.mark.parametrize("N", [8, 16])
def test_scan_gradients_of_short_sequences_by_length(N):
    """More short sequences, some of them empty, than the GPU takes at once: the longest go first,
    with the same bits every time. The first row that a sequence owns is row 2."""
    n, E = 700, 70
    print(f"scan gradients by length n={n} E={E} N={N}", flush=True)
    rng = np.random.default_rng(18)
    lens = rng.integers(0, 31, n).tolist()
    a = _scan_case(lens, E, N, "f32", 19)
    a["state"] = rng.standard_normal((n, E, N)).astype(np.float32)
    T, offs = sum(lens), _offs(lens)
    dy, dend = rng.standard_normal((T, E)).astype(np.float32), rng.standard_normal((n, E, N)).astype(np.float32)
    k = _scan_tensors(a, "f32", T)
    for name in ("u", "dt", "z", "B", "C"):
        k[name] = torch.cat([torch.full_like(k[name][:2], NAN), k[name]])
    args = dict(k, dy=torch.cat([torch.full((2, E), NAN, device="cuda"), _cuda(dy)]), state_grad=_cuda(dend),
                offs=_cuda(offs + 2, torch.int32), L=30)
    out = {m: torch.full((T + 2, w), 7.0, device="cuda") for m, w in dict(du=E, ddt=E, dz=E, dB=N, dC=N).items()}
    g = _tb().ssm_scan_backward(out=out, **args)
    assert all((g[m][:2] == 7.0).all() for m in out)
    again = _tb().ssm_scan_backward(**args)
    assert all(torch.equal(g[m][2:] if m in out else g[m], again[m][2:] if m in out else again[m]) for m in g)
    r = osq.scan_backward(dy=dy, offs=offs, dend=dend, **a)
    _check_scan_grads({m: v[2:] if m in out else v for m, v in g.items()}, r, "f32", T,
                      ["du", "ddt", "dz", "dB", "dC", "dA_log", "dD", "db_dt", "dstate"])
