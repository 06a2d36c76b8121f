"""Log probabilities with entropy and top alternatives (tcl_logprobs) and
distillation from a teacher's top logits (tcl_distill_topk) against the fp64
oracle (oracle/logits.py), and the operators together as a model would run
them.

Tolerances count fp32 roundings (EPS = 2^-24). A difference of logits over
the temperature is off by 3 EPS of itself; a sum over a row of V is a chain of V / 256 + 64 terms
at most in a thread, then a tree; the logarithm adds its own rounding."""
import numpy as np
import pytest
import torch

from oracle import logits as ol

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _tb():
    from paper_2604_12891_amd import binding as tb
    return tb


def _np(t):
    return t.double().cpu().numpy()


def _cuda(a, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype)


def _near(name, got, ref, tol):
    got, ref = _np(got) if torch.is_tensor(got) else got, np.asarray(ref, np.float64)
    # past fp32's largest number (a lowest value over a temperature below 1: -3.4e38 / 0.7 = -4.9e38)
    # the nearest fp32 value is an infinity
    ref = np.where(np.abs(ref) > 3.4028236e38, np.copysign(np.inf, ref), ref)
    with np.errstate(invalid="ignore"):
        ok = (np.abs(got - ref) <= tol) | (got == ref) | (np.isnan(got) & np.isnan(ref))
    assert ok.all(), (name, np.argwhere(~ok)[:5], got[~ok][:5], ref[~ok][:5])


def _spread(rows, temperature):
    """Per row: mean of |z - max| under the softmax, its second moment, log of the sum."""
    o = []
    for x in rows:
        z = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64)) / temperature
        m = z.max() if z.size else -np.inf
        if not np.isfinite(m):
            o.append((0.0, 0.0, 0.0))
            continue
        e = np.exp(z - m)
        d = np.where(e > 0, m - z, 0.0)
        o.append(((e * d).sum() / e.sum(), (e * d * d).sum() / e.sum(), np.log(e.sum())))
    return np.array(o)


def _check_logprobs(got, rows, tokens, K, temperature, first=None):
    ref = ol.logprobs(rows, tokens, K, temperature, first)
    sp = _spread(rows, temperature)
    V = max((len(x) for x in rows), default=0)
    c = V / 256 + 64
    ls = EPS * (3 * sp[:, 0] + c + 4 + 2 * sp[:, 2])  # log of the sum
    if tokens is not None:
        lp = np.nan_to_num(ref["logp"], nan=0.0, neginf=0.0)
        _near("logp", got["logp"], ref["logp"], ls + 4 * EPS * (np.abs(lp) + sp[:, 2]))
    _near("entropy", got["entropy"], ref["entropy"],
          ls + EPS * ((2 * c + 8) * sp[:, 0] + 6 * sp[:, 1] + 3 * sp[:, 0] ** 2))
    if K:
        assert np.array_equal(got["top"].cpu().numpy(), ref["top"])
        tl = np.nan_to_num(ref["top_logp"], neginf=0.0)
        _near("top_logp", got["top_logp"], ref["top_logp"], ls[:, None] + 4 * EPS * (np.abs(tl) + sp[:, 2:]))


def _logits(rng, n, V, dtype, kind):
    x = 2.5 * rng.standard_normal((n, V)) + 3 * rng.standard_normal((n, 1))
    if kind == "masked":
        x[rng.random((n, V)) < 0.3] = -np.inf
        x[0] = -np.inf  # a row whose mask leaves nothing
        if n > 2:
            x[2] = -np.inf
            x[2, V // 2] = 1.0
    if kind == "ties":
        x = np.round(x) * 0.5
        x[n // 2] = 0.25
        x[rng.random((n, V)) < 0.05] = -0.0
    if kind == "nan":
        x[rng.random((n, V)) < 0.1] = np.nan
        x[0] = np.nan
        x[n - 1, : V // 2] = np.nan
        x[n - 1, V // 2:] = -np.inf
    if kind == "lowest":  # masks of the type's lowest value, and a sorted row
        x[rng.random((n, V)) < 0.5] = torch.finfo(DT[dtype]).min
        x[n - 1] = -np.arange(V) * 0.01
    return torch.from_numpy(x.astype(np.float32)).to(DT[dtype]).double().numpy()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "masked", "ties", "nan", "lowest"])
@pytest.mark.parametrize("n,V,ld,K", [(3, 1, 1, 4), (5, 7, 9, 7), (4, 64, 64, 1), (6, 1000, 1003, 20),
                                      (2, 4099, 4099, 64), (3, 50001, 50001, 10), (600, 513, 520, 5), (1, 20000, 20000, 0)])
def test_logprobs(n, V, ld, K, kind, dtype):
    print(f"logprobs n={n} V={V} ld={ld} K={K} {kind} {dtype}", flush=True)
    rng = np.random.default_rng(n + V)
    x = _logits(rng, n, V, dtype, kind)
    buf = torch.full((n, ld), float("nan"), dtype=DT[dtype], device="cuda")
    buf[:, :V] = _cuda(x, DT[dtype])
    tok = rng.integers(0, V, n).astype(np.int32)
    if n > 2:
        tok[1], tok[2] = -1, V
    for temperature in (1.0, 0.7):
        got = _tb().logprobs(buf[:, :V], _cuda(tok, torch.int32), K, temperature)
        _check_logprobs(got, list(x), tok, K, temperature)
    got = _tb().logprobs(buf[:, :V])  # the entropy alone
    assert got["logp"] is None and got["top"] is None
    _check_logprobs(got, list(x), None, 0, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", [[0, 1, 5, 64, 0, 300, 4096, 17], [70000, 3], [40] * 700])
def test_logprobs_of_segments(sizes, dtype):
    """tcl_topk's segments, at every alignment; indices count from the array's start."""
    print(f"logprobs segments {sizes[:8]} {dtype}", flush=True)
    rng = np.random.default_rng(len(sizes))
    offs = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    x = _logits(rng, 1, int(offs[-1]), dtype, "ties")[0]
    rows = [x[a:b] for a, b in zip(offs[:-1], offs[1:])]
    tok = (offs[:-1] + [rng.integers(0, max(s, 1)) for s in sizes]).astype(np.int32)
    for max_len in (max(sizes), None):
        got = _tb().logprobs(_cuda(x, DT[dtype]), _cuda(tok, torch.int32), 16,
                             seg_offsets=_cuda(offs, torch.int32), max_len=max_len)
        _check_logprobs(got, rows, tok, 16, 1.0, offs[:-1])
    if dtype == "f32":
        assert torch.equal(got["top"], _tb().topk(_cuda(x), _cuda(offs, torch.int32), 16))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logprobs_of_rows_made_of_one_stretch(dtype):
    """Whole columns of a thread's entries above every other thread's, so that far
    more entries reach the bound than the list holds."""
    n, V, K = 513, 40000, 64
    ve = 4 if dtype == "f32" else 8
    rng = np.random.default_rng(7)
    x = rng.random((n, V)).astype(np.float32)
    col = np.arange(V) // ve % 256
    x[:, col < 60] += 8.0
    x[:, col == 99] -= 4.0
    x = torch.from_numpy(x).to(DT[dtype]).double().numpy()
    got = _tb().logprobs(_cuda(x, DT[dtype]), None, K)
    pick = [0, 100, 512]
    ref = ol.logprobs([x[i] for i in pick], None, K)
    assert np.array_equal(got["top"].cpu().numpy()[pick], ref["top"])


def _teacher(rng, rows, K, first=None):
    n = len(rows)
    top = np.full((n, K), -1, np.int32)
    val = rng.standard_normal((n, K)).astype(np.float32) * 3
    for r, x in enumerate(rows):
        k = min(K, len(x))
        top[r, :k] = rng.permutation(len(x))[:k] + (0 if first is None else first[r])
    return top, val


def _check_distill(got, rows, top, val, w, temperature, dtype, first=None, flat=False):
    ref = ol.distill(rows, top, val, w, temperature, first)
    V = max((len(x) for x in rows), default=0)
    c = V / 256 + 64
    sp = _spread(rows, temperature)
    first = np.zeros(len(rows), np.int64) if first is None else first
    loss = _np(got["loss"])
    grad = None if got["grad"] is None else _np(got["grad"])
    pos = 0
    for r, x in enumerate(rows):
        x = np.asarray(x, np.float64)
        at = top[r].astype(np.int64) - first[r]
        have = (top[r] >= 0) & (at >= 0) & (at < x.size)
        lq = ol._log_softmax(val[r][have].astype(np.float64) / temperature)
        lp = ol._log_softmax(x / temperature)
        tol, gt = 0.0, np.zeros(x.size)
        if lq is not None and lp is not None:
            q, z = np.exp(lq), np.abs(val[r][have] / temperature)
            # log q is off by a few roundings of its logits and of their sum, and so, relatively, is q
            eq = EPS * (4 * (z + z[np.isfinite(z)].max(initial=0.0)) + len(q) / 64 + 12)
            ep = EPS * (4 * (np.where(np.isfinite(lp), np.abs(lp), 0) + sp[r, 2]) + 3 * sp[r, 0] + c + 4)
            k = q > 0
            i = at[have][k]
            both = np.abs(lq[k]) + np.where(np.isfinite(lp[i]), np.abs(lp[i]), 0)
            tol = (q[k] * ((eq[k] + ep[i]) * 1.0 + (eq[k] + (len(q) + 4) * EPS) * both)).sum()
            gt = np.exp(lp) * (ep + 4 * EPS)
            np.add.at(gt, i, q[k] * (eq[k] + (len(q) + 4) * EPS))
            gt *= (1.0 if w is None else abs(float(w[r]))) / temperature
        _near(f"loss {r}", loss[r:r + 1], ref["loss"][r:r + 1], tol)
        if grad is not None:
            g = ref["grad"][r]
            half = 2.0 ** -8 if dtype == "bf16" else EPS
            mine = grad[pos:pos + x.size] if flat else grad[r]
            _near(f"grad {r}", mine, g, gt + half * (np.abs(g) + gt) + 1e-37)
            pos += x.size


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["plain", "masked", "lowest"])
@pytest.mark.parametrize("n,V,ld,K", [(3, 1, 1, 2), (5, 7, 9, 7), (6, 1000, 1003, 20), (2, 4099, 4099, 64),
                                      (3, 50001, 50001, 10), (600, 250, 250, 5), (600, 1000, 1001, 8),
                                      (520, 6001, 6001, 33), (4, 3000, 3000, 1024)])
def test_distill(n, V, ld, K, kind, dtype):
    print(f"distill n={n} V={V} ld={ld} K={K} {kind} {dtype}", flush=True)
    rng = np.random.default_rng(n + V + K)
    x = _logits(rng, n, V, dtype, kind)
    top, val = _teacher(rng, x, K)
    if n > 4 and V > 3 and K > 3:
        top[1] = -1                    # no teacher
        val[3] = -np.inf               # a teacher with nothing left
        top[4, 1], top[4, 2] = top[4, 0], V + 5  # an entry twice, one outside
        val[0, K // 2] = -np.inf
    w = rng.random(n).astype(np.float32)
    buf = torch.full((n, ld), 5.0, dtype=DT[dtype], device="cuda")
    buf[:, :V] = _cuda(x, DT[dtype])
    out = torch.full((n, ld), 7.0, dtype=DT[dtype], device="cuda")
    args = dict(top=_cuda(top, torch.int32), teacher=_cuda(val), weight=_cuda(w), temperature=1.7)
    got = _tb().distill_topk(buf[:, :V], grad=out[:, :V], **args)
    _check_distill(got, list(x), top, val, w, 1.7, dtype)
    assert (out[:, V:] == 7.0).all() and (buf[:, V:] == 5.0).all()
    alone = _tb().distill_topk(buf[:, :V], grad=False, **dict(args, weight=None))
    assert alone["grad"] is None and torch.equal(alone["loss"], got["loss"])
    inplace = _tb().distill_topk(buf[:, :V], grad=buf[:, :V], **args)
    assert torch.equal(inplace["loss"], got["loss"]) and torch.equal(buf[:, :V], out[:, :V])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,V", [(515, 17000), (514, 70001), (513, 140003), (259, 70001), (258, 150001)])
def test_distill_rows_of_every_length(n, V, dtype):
    """Rows that the registers hold, longer ones whose rest is read again, and few long ones, which are
    split over workgroups."""
    print(f"distill rows n={n} V={V} {dtype}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(V)
    x = (2 * torch.randn(n, V, generator=g, device="cuda")).to(DT[dtype])
    top = torch.randint(0, V, (n, 12), generator=g, device="cuda", dtype=torch.int32)
    val = 2 * torch.randn(n, 12, generator=g, device="cuda")
    got = _tb().distill_topk(x, top, val)
    pick = [0, 1, 257, n - 1]
    rows = [_np(x[i]) for i in pick]
    _check_distill({k: v[pick] for k, v in got.items()}, rows, top[pick].cpu().numpy(), val[pick].cpu().numpy(), None,
                   1.0, dtype)
    # every row's gradient sums to zero: p and q do. Each entry is off by half a step of its type
    # and 2e-5 of itself, and the absolute values sum to 2 at most.
    assert (got["grad"].double().sum(1).abs() < 2 * (2.0 ** -8 if dtype == "bf16" else 2e-5)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes,K", [([0, 1, 5, 64, 0, 300, 4096, 17], 16), ([30000, 3], 40), ([33] * 600, 8)])
def test_distill_of_segments(sizes, K, dtype):
    print(f"distill segments {sizes[:8]} K={K} {dtype}", flush=True)
    rng = np.random.default_rng(len(sizes) + K)
    offs = np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)
    x = _logits(rng, 1, int(offs[-1]), dtype, "plain")[0]
    rows = [x[a:b] for a, b in zip(offs[:-1], offs[1:])]
    top, val = _teacher(rng, rows, K, offs[:-1])
    top[-1, 0] = offs[-2] - 1  # the neighbour's entry: not this row's
    w = rng.random(len(sizes)).astype(np.float32)
    out = torch.full((int(offs[-1]) + 1,), 7.0, dtype=DT[dtype], device="cuda")
    for grad in (out[1:], True):  # at another alignment than the logits, and at the same
        got = _tb().distill_topk(_cuda(x, DT[dtype]), _cuda(top, torch.int32), _cuda(val), _cuda(w), 2.0,
                                 seg_offsets=_cuda(offs, torch.int32), max_len=max(sizes), grad=grad)
        _check_distill(got, rows, top, val, w, 2.0, dtype, offs[:-1], flat=True)
    assert out[0] == 7.0


@pytest.mark.parametrize("n", [3, 600])
def test_distill_of_nan(n):
    """A NaN, of the student or of the teacher, shows in its row and in no other;
    one of the teacher's at an entry that does not count does not."""
    V, K = 2500, 6
    g = torch.Generator(device="cuda").manual_seed(n)
    x = torch.randn(n, V, generator=g, device="cuda")
    top = torch.randint(0, V, (n, K), generator=g, device="cuda", dtype=torch.int32)
    val = torch.randn(n, K, generator=g, device="cuda")
    x[0, 17] = float("nan")
    val[1, 2] = float("nan")
    top[2, 3], val[2, 3] = -1, float("nan")
    got = _tb().distill_topk(x, top, val)
    bad = torch.isnan(got["loss"]).cpu()
    assert bad[0] and bad[1] and not bad[2:].any()
    assert torch.isnan(got["grad"][0]).all() and not torch.isnan(got["grad"][2:]).any()


def test_captured_calls():
    """Both operators in one captured graph over one workspace, replayed on new logits."""
    tb = _tb()
    n, V, K = 6, 9001, 12
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(n, V, generator=g, device="cuda")
    teacher = torch.randn(n, V, generator=g, device="cuda")
    tok = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    ws = tb.logits_workspace(n, V, K)
    assert ws.numel() > 0

    def both():
        t = tb.logprobs(teacher, tok, K, workspace=ws)
        return dict(t, **tb.distill_topk(x, t["top"], t["top_logp"], workspace=ws))

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for _ in range(3):
        x.copy_(torch.randn(n, V, device="cuda"))
        teacher.copy_(torch.randn(n, V, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for k, v in both().items():
            assert torch.equal(v, out[k]), k


def test_far_rows():
    """Rows past 4 GiB."""
    n, V = 40, 60_000_000
    x = torch.full((n, V), -30.0, dtype=torch.bfloat16, device="cuda")
    x[n - 1, V - 1] = 5.0
    x[n - 1, 11] = 4.0
    got = _tb().logprobs(x, None, 2)
    assert got["top"][n - 1].tolist() == [V - 1, 11] and got["top"][0].tolist() == [0, 1]
    top = torch.full((n, 1), V - 1, dtype=torch.int32, device="cuda")
    r = _tb().distill_topk(x, top, torch.zeros(n, 1, device="cuda"), grad=x)
    # log p of the one entry: 0 - log(1 + e^-1 + 6e7 e^-35)
    assert abs(float(r["loss"][n - 1]) - np.log(1 + np.exp(-1))) < 1e-5
    assert abs(float(x[n - 1, V - 1]) + 1 - 1 / (1 + np.exp(-1))) < 2.0 ** -8 and float(x[0, V - 1]) < -0.99


def _block64(p, x, offs):
    """A Mamba mixer with a vocabulary head, in 64 bits with torch's autograd."""
    logits = []
    for lo, hi in zip(offs[:-1], offs[1:]):
        xs = x[lo:hi]
        pad = torch.cat([torch.zeros(3, xs.shape[1], dtype=torch.float64), xs])
        pre = p["conv_b"] + sum(p["conv_w"][:, k] * pad[k:k + hi - lo] for k in range(4))
        u = pre * torch.sigmoid(pre)
        proj = u @ p["W_x"].T
        R, N = p["W_dt"].shape[1], p["A_log"].shape[1]
        d = torch.nn.functional.softplus(proj[:, :R] @ p["W_dt"].T + p["b_dt"])
        s, A = torch.zeros(xs.shape[1], N, dtype=torch.float64), -torch.exp(p["A_log"])
        ys = []
        for t in range(hi - lo):
            s = torch.exp(d[t][:, None] * A) * s + (d[t] * u[t])[:, None] * proj[t, R:R + N]
            ys.append((s * proj[t, R + N:]).sum(1) + p["D"] * u[t])
        logits.append(torch.stack(ys) @ p["W_o"].T)
    return torch.cat(logits)


def test_a_student_learns_from_a_teacher():
    """The operators together: a mixer (convolution, projections, scan) with a head gives
    logits; a teacher's log probabilities and top alternatives are what the student is distilled from,
    and the gradients go back through scan and convolution. All against autograd
    in 64 bits; the fp32 products and operators are sums of at most 300 terms, 1e-4 of the largest
    gradient covers their 300 roundings of 6e-8 forwards and back."""
    tb = _tb()
    E, N, R, V, K = 48, 16, 4, 300, 8
    lens = [21, 1, 40]
    offs = np.concatenate([[0], np.cumsum(lens)])
    T = int(offs[-1])
    rng = np.random.default_rng(9)

    def params(seed):
        r = np.random.default_rng(seed).standard_normal
        return dict(conv_w=0.5 * r((E, 4)), conv_b=0.1 * r(E), W_x=r((R + 2 * N, E)) / np.sqrt(E),
                    W_dt=0.5 * r((E, R)), b_dt=r(E) - 3, A_log=0.3 * r((E, N)), D=r(E), W_o=2 * r((V, E)) / np.sqrt(E))

    x = rng.standard_normal((T, E)).astype(np.float32)
    ps, pt = ({k: torch.from_numpy(v.astype(np.float32)).double() for k, v in params(s).items()} for s in (1, 2))
    X, O = _cuda(x), _cuda(offs, torch.int32)
    w = rng.random(T).astype(np.float32)

    def forward(p):
        p = {k: v.float().cuda() for k, v in p.items()}
        u = tb.ssm_conv(X, p["conv_w"], p["conv_b"], O)
        proj = u @ p["W_x"].T
        dt = proj[:, :R] @ p["W_dt"].T
        y = tb.ssm_scan(u, dt, p["A_log"], proj[:, R:R + N], proj[:, R + N:], D=p["D"], b_dt=p["b_dt"], offs=O, L=40)
        return p, u, proj, dt, y, y @ p["W_o"].T

    taught = tb.logprobs(forward(pt)[-1], K=K)
    p, u, proj, dt, y, logits = forward(ps)
    out = tb.distill_topk(logits, taught["top"], taught["top_logp"], _cuda(w), temperature=1.5)
    dlogits = out["grad"]
    dy = dlogits @ p["W_o"]
    g = tb.ssm_scan_backward(u, dt, p["A_log"], proj[:, R:R + N], proj[:, R + N:], dy, D=p["D"], b_dt=p["b_dt"],
                             offs=O, L=40)
    dproj = torch.cat([g["ddt"] @ p["W_dt"], g["dB"], g["dC"]], 1)
    c = tb.ssm_conv_backward(X, p["conv_w"], p["conv_b"], g["du"] + dproj @ p["W_x"], O)
    got = dict(conv_w=c["dw"], conv_b=c["db"], W_x=dproj.T @ u, W_dt=g["ddt"].T @ proj[:, :R], b_dt=g["db_dt"],
               A_log=g["dA_log"], D=g["dD"], W_o=dlogits.T @ y, x=c["dx"])

    leaf = {k: v.clone().requires_grad_() for k, v in ps.items()}
    lx = torch.from_numpy(x).double().requires_grad_()
    with torch.no_grad():
        t64 = torch.log_softmax(_block64(pt, lx, offs), 1)
        val, idx = t64.topk(K, 1)
    assert torch.equal(idx.int(), taught["top"].cpu())
    lq = torch.log_softmax(val / 1.5, 1)
    lp = torch.log_softmax(_block64(leaf, lx, offs) / 1.5, 1).gather(1, idx)
    loss = (lq.exp() * (lq - lp)).sum(1)
    (loss * torch.from_numpy(w).double()).sum().backward()
    np.testing.assert_allclose(_np(out["loss"]), loss.detach().numpy(), rtol=1e-4, atol=1e-5)
    for name, v in got.items():
        ref = (lx if name == "x" else leaf[name]).grad.numpy()
        np.testing.assert_allclose(_np(v), ref, rtol=0, atol=1e-4 * np.abs(ref).max(), err_msg=name)

    # and the student answers token by token as it does at once
    S = torch.zeros(1, E, N, device="cuda")
    cs = torch.zeros(1, 3, E, device="cuda")
    for t in range(lens[0]):
        ut = tb.ssm_conv(X[t:t + 1], p["conv_w"], p["conv_b"], state=cs, state_out=cs)
        pr = ut @ p["W_x"].T
        yt = tb.ssm_scan(ut, pr[:, :R] @ p["W_dt"].T, p["A_log"], pr[:, R:R + N], pr[:, R + N:], D=p["D"],
                         b_dt=p["b_dt"], state=S, state_out=S)
        np.testing.assert_allclose(_np(yt[0]), _np(y[t]), rtol=0, atol=1e-5 * float(y.abs().max()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,V", [(3, 2500), (2, 70001), (600, 150)])
@pytest.mark.parametrize("temperature", [1e-30, 1e-9, 1e30])
def test_extreme_temperatures(n, V, temperature, dtype):
    """Masked rows at temperatures that leave one entry, or spread all entries evenly. The logits are
    small integers, so differences are exact and a value is off by the roundings of 1 / temperature, of a product
    or two and of a logarithm: 8 EPS of it at most, and half a step of a bf16 gradient. No entry that
    the mask takes has any of it."""
    print(f"extreme n={n} V={V} T={temperature} {dtype}", flush=True)
    tb, rng = _tb(), np.random.default_rng(V)
    x = -(1.0 + rng.integers(0, 199, (n, V)))
    x[rng.random((n, V)) < 0.3] = -np.inf
    peak = rng.integers(5, V, n)
    x[np.arange(n), peak] = 4.0
    x[:, :5] = [-3, -7, -11, -1, -2]
    top = np.tile(np.array([1, 0, 3, 2, 4], np.int32), (n, 1))
    val = np.tile(np.array([-1, 2, 0.5, -np.inf, 1.5], np.float32), (n, 1))
    top[0], val[0] = peak[0], 1e9  # (one entry five times, of logits that a division would take out of range)
    X = _cuda(x, DT[dtype])
    live = np.isfinite(x).sum(1)
    one = np.zeros((n, V))
    one[np.arange(n), peak] = 1
    t32 = float(np.float32(temperature))
    if temperature < 1:
        p, q = one, np.zeros((n, V))
        q[:, 0] = 1
        loss, ent = np.full(n, 7 / t32), np.zeros(n)
        logp = (x - 4) / t32
    else:
        p, q = np.isfinite(x) / live[:, None], np.zeros((n, V))
        q[:, [1, 0, 3, 4]] = 0.25
        loss, ent = np.log(live) - np.log(4), np.log(live)
        logp = np.where(np.isfinite(x), -np.log(live)[:, None], -np.inf)
    q[0] = one[0]
    loss[0] = (0 if temperature < 1 else np.log(live[0])) - np.log(5)
    got = tb.distill_topk(X, _cuda(top, torch.int32), _cuda(val), temperature=temperature)
    half = 2.0 ** -8 if dtype == "bf16" else 0
    _near("loss", got["loss"], loss, 8 * EPS * (np.abs(loss) + 2 * np.log(5)))
    _near("grad", got["grad"], (p - q) / t32, (8 * EPS + half) * (p + q) / t32)
    tok = np.where(np.arange(n) % 2, peak, 2).astype(np.int32)
    got = tb.logprobs(X, _cuda(tok, torch.int32), 2, temperature)
    lp = logp[np.arange(n), tok]
    _near("logp", got["logp"], lp, 8 * EPS * np.abs(lp))
    _near("entropy", got["entropy"], ent, 8 * EPS * ent)
    first = np.stack([logp[np.arange(n), peak], logp[:, 3]], 1)
    assert np.array_equal(got["top"].cpu().numpy()[:, 0], peak)
    _near("top", got["top_logp"][:, 0], first[:, 0], 8 * EPS * np.abs(first[:, 0]))


def test_results_that_are_not_wanted():
    """NULL for every result that may be: the others are what they are with it."""
    tb = _tb()
    from paper_2604_12891_amd.binding import lib
    n, V, K = 5, 3000, 6
    g = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(n, V, generator=g, device="cuda")
    tok = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    full = tb.logprobs(x, tok, K)
    top = torch.empty(n, K, dtype=torch.int32, device="cuda")
    lp, en = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ws = tb.logits_workspace(n, V, K)
    w = (ws.data_ptr(), ws.numel())
    s = torch.cuda.current_stream().cuda_stream
    assert lib().tcl_logprobs(0, n, V, x.data_ptr(), V, None, 1.0, None, K, None, None, top.data_ptr(), None, *w, s) == 0
    assert torch.equal(top, full["top"])
    assert lib().tcl_logprobs(0, n, V, x.data_ptr(), V, None, 1.0, tok.data_ptr(), 0, lp.data_ptr(), None, None, None,
                              *w, s) == 0
    assert torch.equal(lp, full["logp"])
    assert lib().tcl_logprobs(0, n, V, x.data_ptr(), V, None, 1.0, None, 0, None, en.data_ptr(), None, None, *w, s) == 0
    assert torch.equal(en, full["entropy"])


@pytest.mark.parametrize("n,V,K", [(5, 255, 257), (244, 1000, 20), (3, 70001, 64)])
def test_distill_of_masks_beyond_fp32(n, V, K):
    """Where the mask is the type's lowest value and the temperature below 1, log p is beyond fp32 (-6.8e38),
    and the loss, with the teacher's small probability there, is often not."""
    print(f"distill beyond n={n} V={V} K={K}", flush=True)
    rng = np.random.default_rng(n + V)
    x = _logits(rng, n, V, "f32", "lowest")
    top, val = _teacher(rng, x, K)
    val *= 2  # (probabilities down to e^-40)
    got = _tb().distill_topk(_cuda(x), _cuda(top, torch.int32), _cuda(val), temperature=0.5)
    _check_distill(got, list(x), top, val, None, 0.5, "f32")
    assert torch.isfinite(got["loss"]).any()
