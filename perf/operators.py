"""The sequence and logit operators of this framework, as cases that can be
timed and compared: the causal convolution and the selective scan with their
carried states (prompts, single tokens, gradients), the log probabilities of
given entries with entropy and top alternatives, and distillation from a
teacher's top logits.

  own                 False: `run` is the operators' plain form, elementary
                      torch operations in 32 bits; True: the framework's calls
  listed()            the cases, dicts of plain values
  draw(rng)           one more case of the same ranges
  prepare(case, seed) inputs and buffers, as a program holds them
  run(state)          one pass through an operator; its outputs
  work(case)          bytes and operations that one pass cannot do without
  exact(case, seed)   the same outputs in 64 bits

Sequences are packed: sequence i owns rows offs[i] .. offs[i+1]-1 of every
activation. Activations have the unit variance that normalised layers give
them, step sizes softplus(dt + b_dt) around [1e-3, 1e-1], decay rates
1 .. N jittered per channel. Logits have a spread of 2.5 around a row's own
level, a part of them masked to -inf where a case says so.
"""
from __future__ import annotations

import math

import torch

own = False

# The widths of this repository's own models (d_inner 128, 256 and 512, d_state
# 8 and 16) and generic ones of language models; odd ones are drawn too.


def listed():
    return [
        # convolution: one token of each of a batch of sequences, states in a pool
        dict(name="conv_token_bf16", kind="conv", dtype="bf16", n=256, L=1, lo=1, E=4096, K=4, pool=384),
        # convolution, forward and backward, on packed documents of uneven length
        dict(name="conv_train_bf16", kind="conv_train", dtype="bf16", n=8, L=4096, lo=512, E=4096, K=4, carry=False),
        # the smallest call: a few programs that grow by one statement each, latency only
        dict(name="scan_token_few_f32", kind="scan", dtype="f32", n=4, L=1, lo=1, E=512, N=16, pool=4),
        # a serving batch, one token each, states in a pool
        dict(name="scan_token_bf16", kind="scan", dtype="bf16", n=256, L=1, lo=1, E=4096, N=16, pool=384),
        # one tuning round's candidate programs
        dict(name="scan_round_f32", kind="scan", dtype="f32", n=4096, L=25, lo=5, E=512, N=16, pool=0),
        # one long prompt, whose end state is kept
        dict(name="scan_prompt_bf16", kind="scan", dtype="bf16", n=1, L=8192, lo=8000, E=4096, N=16, pool=1),
        # gradients on the distillation student's batch of short programs
        dict(name="scan_train_short_f32", kind="scan_train", dtype="f32", n=1024, L=25, lo=5, E=256, N=16, carry=False),
        # gradients on longer documents, state and its gradient carried over from and to the neighbours
        dict(name="scan_train_long_bf16", kind="scan_train", dtype="bf16", n=4, L=2048, lo=1500, E=2048, N=16,
             carry=True),
        # a few rows of a decoder's step, odd width: the chosen token, entropy and a few alternatives
        dict(name="logprobs_few_f32", kind="logprobs", dtype="f32", n=4, V=50001, K=8, ragged=False, masked=0.0),
        # a teacher answers for a whole batch of positions, part of the entries masked
        dict(name="logprobs_batch_bf16", kind="logprobs", dtype="bf16", n=4096, V=32768, K=20, ragged=False,
             masked=0.1),
        # the tasks of a tuning round: candidates of uneven number, the teacher's best 64 of each
        dict(name="distill_tasks_f32", kind="distill", dtype="f32", n=16, V=4096, K=64, ragged=True, masked=0.0),
        # a student's training batch over a large vocabulary
        dict(name="distill_batch_bf16", kind="distill", dtype="bf16", n=2048, V=131072, K=32, ragged=False, masked=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["conv", "conv_train", "scan", "scan", "scan_token", "scan_train", "scan_train", "logprobs",
                       "logprobs", "distill", "distill"])
    dtype = rng.choice(["f32", "bf16"])
    if kind in ("logprobs", "distill"):
        V = _log(rng, 40, 131072)
        n = _log(rng, 1, min(8192, (134_000_000 if dtype == "bf16" else 67_000_000) // V))
        return dict(kind=kind, dtype=dtype, n=n, V=V, K=rng.choice([1, 5, 10, 20, 32, 64]), ragged=rng.random() < 0.3,
                    masked=rng.choice([0.0, 0.0, 0.2]))
    E = rng.choice([rng.choice([128, 256, 512, 1024, 2048, 4096]), 8 * _log(rng, 8, 512), _log(rng, 60, 4096)])
    if kind == "scan_token":
        n = _log(rng, 1, 1_040_000 // E)
        return dict(kind="scan", dtype=dtype, n=n, L=1, lo=1, E=E, N=rng.choice([8, 16]), pool=n + rng.randint(0, n))
    L = _log(rng, 2, 8192 if kind != "scan_train" else 2048)
    n = _log(rng, 1, max(1, min(4096, 16_000_000 // (E * L))))
    lo = rng.choice([1, max(1, L // 5), L])
    if kind == "conv":
        return dict(kind=kind, dtype=dtype, n=n, L=L, lo=lo, E=E, K=rng.choice([2, 3, 4, 4]), pool=rng.choice([0, n]))
    if kind == "conv_train":
        return dict(kind=kind, dtype=dtype, n=n, L=L, lo=lo, E=E, K=rng.choice([2, 3, 4, 4]),
                    carry=rng.random() < 0.5)
    if kind == "scan":
        return dict(kind=kind, dtype=dtype, n=n, L=L, lo=lo, E=E, N=rng.choice([8, 16, 16]), pool=rng.choice([0, n]))
    return dict(kind=kind, dtype=dtype, n=n, L=L, lo=lo, E=E, N=rng.choice([8, 16, 16]), carry=rng.random() < 0.5)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case):
    """The lengths of a case's sequences (of its rows' entries): the case's
    own, whatever the seed, which only orders them."""
    n, L = case["n"], case.get("L") or case["V"]
    lo = case["lo"] if "L" in case else max(1, int(0.3 * L)) if case["ragged"] else L
    g = torch.Generator().manual_seed(1000003 * n + L)
    return torch.randint(lo, L + 1, (n,), generator=g)


def _offsets(case, g):
    lengths = _lengths(case).cuda()[torch.randperm(case["n"], generator=g, device="cuda")]
    offs = torch.zeros(case["n"] + 1, dtype=torch.int32, device="cuda")
    offs[1:] = lengths.cumsum(0)
    return offs


def _packing(case, g):
    """Offsets (None for single tokens) and the number of rows."""
    if case["L"] == 1:
        return None, case["n"]
    return _offsets(case, g), int(_lengths(case).sum())


def _slots(case, g):
    """Where each sequence's state is in the pool; a batch of four single
    tokens or more is padded with a sequence that has none."""
    slots = torch.randperm(case["pool"], generator=g, device="cuda")[:case["n"]].int()
    if case["L"] == 1 and case["n"] >= 4:
        slots[case["n"] // 2] = -1
    return slots


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = _type(case)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    s = dict(case=case)
    kind = case["kind"]
    if kind in ("logprobs", "distill"):
        n, V, K = case["n"], case["V"], case["K"]
        if case["ragged"]:
            # candidates of uneven number, V at most
            s["offs"] = _offsets(case, g)
            size = s["offs"][1:] - s["offs"][:-1]
            x = 2.5 * randn(int(_lengths(case).sum()))
        else:
            size = torch.full((n,), V, dtype=torch.int32, device="cuda")
            s["offs"] = None
            x = 2.5 * randn(n, V) + randn(n, 1)
        if case["masked"]:
            x.masked_fill_(rand(*x.shape) < case["masked"], -math.inf)
        s["logits"] = x.to(t)
        if kind == "logprobs":
            tok = (rand(n) * size).int().clamp_(max=size - 1)
            s["tokens"] = tok if s["offs"] is None else tok + s["offs"][:-1]
        else:
            # a teacher that mostly agrees with the student
            teacher = x + 1.5 * randn(*x.shape)
            rows = teacher if s["offs"] is None else _segments(teacher, s["offs"], V)
            val, idx = rows.topk(min(K, rows.shape[1]), dim=1)
            if idx.shape[1] < K:
                val = torch.nn.functional.pad(val, (0, K - idx.shape[1]), value=-math.inf)
                idx = torch.nn.functional.pad(idx, (0, K - idx.shape[1]), value=V)
            none = idx >= size[:, None]
            if s["offs"] is not None:
                idx = idx + s["offs"][:-1, None]
            s["top"] = torch.where(none, -1, idx).int()
            s["teacher"] = val
            s["weight"] = rand(n) / n
        if own:
            from paper_2604_12891_amd import binding as tb
            s["tb"] = tb
            s["ws"] = tb.logits_workspace(n, V, K)
        return s

    E = case["E"]
    s["offs"], rows = _packing(case, g)
    if kind in ("conv", "conv_train"):
        K = case["K"]
        s["x"] = randn(rows, E).to(t)
        s["w"] = (2 * rand(E, K) - 1) / math.sqrt(K)
        s["b"] = (2 * rand(E) - 1) / math.sqrt(K)
        state = (K - 1, E), t
    else:
        N = case["N"]
        # u and the gate as the layers give them; dt, B and C as they leave one
        # projection, each row's columns beside each other
        s["u"] = torch.nn.functional.silu(randn(rows, E)).to(t)
        s["z"] = randn(rows, E).to(t)
        s["dt"] = (0.5 * randn(rows, E)).to(t)
        bc = randn(rows, 2 * N).to(t)
        s["B"], s["C"] = bc[:, :N], bc[:, N:]
        s["A_log"] = torch.log(torch.arange(1, N + 1, device="cuda").float()) + 0.3 * randn(E, N)
        s["D"] = 1.0 + 0.5 * randn(E)
        d = torch.exp(math.log(1e-3) + (math.log(1e-1) - math.log(1e-3)) * rand(E))
        s["b_dt"] = d + torch.log(-torch.expm1(-d))
        state = (E, N), torch.float32
    shape, st = state
    if kind in ("conv", "scan"):
        s["state"] = s["state_out"] = s["slots"] = None
        if case["pool"]:
            s["slots"] = _slots(case, g)
            s["state"] = (0.5 * randn(case["pool"], *shape)).to(st)
            s["state_out"] = torch.zeros(case["pool"], *shape, dtype=st, device="cuda")
    else:
        s["grad"] = randn(rows, E).to(t)
        s["state"] = s["state_grad"] = None
        if case["carry"]:
            s["state"] = (0.5 * randn(case["n"], *shape)).to(st)
            s["state_grad"] = (0.1 * randn(case["n"], *shape)).to(st)
    if own:
        from paper_2604_12891_amd import binding as tb
        s["tb"] = tb
        if kind == "conv_train":
            s["ws"] = tb.ssm_conv_workspace(case["n"], rows, E, case["K"])
        elif kind == "scan":
            s["ws"] = tb.ssm_scan_workspace(case["n"], rows, E, case["N"], case["L"])
        elif kind == "scan_train":
            s["ws"] = tb.ssm_scan_workspace(case["n"], rows, E, case["N"], case["L"], backward=True)
        if kind in ("conv", "scan"):
            s["out"] = torch.empty(rows, E, dtype=t, device="cuda")
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    tb, case = s["tb"], s["case"]
    kind = case["kind"]
    if kind == "conv":
        tb.ssm_conv(s["x"], s["w"], s["b"], offs=s["offs"], state=s["state"], state_out=s["state_out"],
                    slots=s["slots"], out=s["out"])
        return dict(u=s["out"], state=s["state_out"])
    if kind == "conv_train":
        u = tb.ssm_conv(s["x"], s["w"], s["b"], offs=s["offs"], state=s["state"])
        return dict(tb.ssm_conv_backward(s["x"], s["w"], s["b"], s["grad"], offs=s["offs"], state=s["state"],
                                         state_grad=s["state_grad"], workspace=s["ws"]), u=u)
    if kind == "scan":
        tb.ssm_scan(s["u"], s["dt"], s["A_log"], s["B"], s["C"], D=s["D"], z=s["z"], b_dt=s["b_dt"], offs=s["offs"],
                    L=case["L"], state=s["state"], state_out=s["state_out"], slots=s["slots"], out=s["out"],
                    workspace=s["ws"])
        return dict(y=s["out"], state=s["state_out"])
    if kind == "scan_train":
        return tb.ssm_scan_backward(s["u"], s["dt"], s["A_log"], s["B"], s["C"], s["grad"], D=s["D"], z=s["z"],
                                    b_dt=s["b_dt"], offs=s["offs"], L=case["L"], state=s["state"],
                                    state_grad=s["state_grad"], workspace=s["ws"])
    if kind == "logprobs":
        return tb.logprobs(s["logits"], s["tokens"], K=case["K"], seg_offsets=s["offs"], max_len=case["V"],
                           workspace=s["ws"])
    return tb.distill_topk(s["logits"], s["top"], s["teacher"], weight=s["weight"], temperature=2.0,
                           seg_offsets=s["offs"], max_len=case["V"], workspace=s["ws"])


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "conv":
        return _plain_conv(s)
    if kind == "conv_train":
        return _plain_conv_train(s)
    if kind == "scan":
        return _plain_scan(s)
    if kind == "scan_train":
        return _plain_scan_train(s)
    if kind == "logprobs":
        return _plain_logprobs(s)
    return _plain_distill(s)


# --- packed rows and dense batches

def _rows_of(offs, n, L, device):
    """Row of token t of sequence i, and whether there is one: [n, L]."""
    t = torch.arange(L, device=device)
    if offs is None:
        return torch.arange(n, device=device)[:, None], torch.ones(n, 1, dtype=torch.bool, device=device)
    idx = offs[:-1, None].long() + t
    return idx, idx < offs[1:, None]


def _dense(a, idx, live):
    """Packed rows as a padded batch [n, L, ...] in 32 bits, zero where there
    is no token."""
    d = a.float()[torch.where(live, idx, 0)]
    return d * live.view(*live.shape, *([1] * (a.dim() - 1)))


def _picked(state, slots):
    """The sequences' states out of the pool, zeros for those without one."""
    if state is None:
        return None
    if slots is None:
        return state.float()
    ok = (slots >= 0) & (slots < state.shape[0])
    st = state.float()[torch.where(ok, slots, 0).long()]
    return st * ok.view(-1, *([1] * (st.dim() - 1)))


def _kept(state_out, slots, st):
    """Their new states written into the pool."""
    if state_out is None:
        return None
    if slots is None:
        state_out.copy_(st)
    else:
        ok = (slots >= 0) & (slots < state_out.shape[0])
        state_out[slots[ok].long()] = st[ok].to(state_out.dtype)
    return state_out


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _softplus(x):
    return torch.log1p(torch.exp(-x.abs())) + x.clamp(min=0)


# --- convolution

def _conv_window(s, slots):
    case = s["case"]
    K = case["K"]
    idx, live = _rows_of(s["offs"], case["n"], case["L"], s["x"].device)
    x = _dense(s["x"], idx, live)
    before = _picked(s["state"], slots)
    if before is None:
        before = torch.zeros(case["n"], K - 1, case["E"], device=x.device)
    return torch.cat([before, x], 1), idx, live


def _plain_conv(s):
    case = s["case"]
    K, n = case["K"], case["n"]
    win, idx, live = _conv_window(s, s["slots"])
    L = live.shape[1]
    pre = s["b"] + sum(s["w"][:, k] * win[:, k:k + L] for k in range(K))
    u = (pre * _sigmoid(pre))[live].to(s["x"].dtype)
    out = None
    if s["state_out"] is not None:
        last = live.sum(1)[:, None] + torch.arange(K - 1, device=u.device)
        out = _kept(s["state_out"], s["slots"], win[torch.arange(n, device=u.device)[:, None], last])
    return dict(u=u, state=out)


def _plain_conv_train(s):
    case = s["case"]
    K, n, E = case["K"], case["n"], case["E"]
    t = s["x"].dtype
    win, idx, live = _conv_window(s, None)
    L = live.shape[1]
    pre = s["b"] + sum(s["w"][:, k] * win[:, k:k + L] for k in range(K))
    sig = _sigmoid(pre)
    u = (pre * sig)[live].to(t)
    g = _dense(s["grad"], idx, live) * (sig * (1.0 + pre * (1.0 - sig)))
    dwin = torch.zeros_like(win)
    dw = torch.empty(E, K, device=g.device)
    for k in range(K):
        dwin[:, k:k + L] += s["w"][:, k] * g
        dw[:, k] = (g * win[:, k:k + L]).sum((0, 1))
    if s["state_grad"] is not None:
        last = live.sum(1)[:, None] + torch.arange(K - 1, device=g.device)
        dwin[torch.arange(n, device=g.device)[:, None], last] += s["state_grad"].float()
    dstate = dwin[:, :K - 1].to(t) if s["state"] is not None else None
    return dict(dx=dwin[:, K - 1:][live].to(t), dw=dw, db=g.sum((0, 1)), dstate=dstate, u=u)


# --- selective scan

def _scan_inputs(s):
    case = s["case"]
    idx, live = _rows_of(s["offs"], case["n"], case["L"], s["u"].device)
    u, v, z, B, C = (_dense(s[k], idx, live) for k in ("u", "dt", "z", "B", "C"))
    v = v + s["b_dt"]
    d = _softplus(v) * live[:, :, None]
    return live, u, v, d, z, B, C, -torch.exp(s["A_log"])


def _plain_scan(s):
    case = s["case"]
    live, u, _, d, z, B, C, A = _scan_inputs(s)
    st = _picked(s["state"], s["slots"])
    if st is None:
        st = torch.zeros(case["n"], *A.shape, device=u.device)
    ys = []
    for t in range(live.shape[1]):
        # past a sequence's end d is 0: the state stays as it is
        st = torch.exp(d[:, t, :, None] * A) * st + (d[:, t] * u[:, t])[:, :, None] * B[:, t, None, :]
        ys.append((st * C[:, t, None, :]).sum(-1))
    y = (torch.stack(ys, 1) + s["D"] * u) * z * _sigmoid(z)
    return dict(y=y[live].to(s["u"].dtype), state=_kept(s["state_out"], s["slots"], st))


def _plain_scan_train(s):
    case = s["case"]
    t_ = s["u"].dtype
    live, u, v, d, z, B, C, A = _scan_inputs(s)
    n, L = live.shape
    idx, _ = _rows_of(s["offs"], n, case["L"], u.device)
    dy = _dense(s["grad"], idx, live)
    sz = _sigmoid(z)
    q = dy * z * sz
    S = torch.empty(L + 1, n, *A.shape, device=u.device)
    S[0] = 0.0 if s["state"] is None else s["state"]
    y = torch.empty_like(u)
    for t in range(L):
        S[t + 1] = torch.exp(d[:, t, :, None] * A) * S[t] + (d[:, t] * u[:, t])[:, :, None] * B[:, t, None, :]
        y[:, t] = (S[t + 1] * C[:, t, None, :]).sum(-1)
    dz = dy * (y + s["D"] * u) * sz * (1.0 + z * (1.0 - sz))
    dB, dC = torch.empty_like(B), torch.empty_like(C)
    du, dd = torch.empty_like(u), torch.empty_like(u)
    dA = torch.zeros_like(A)
    g = torch.zeros(n, *A.shape, device=u.device) if s["state_grad"] is None else s["state_grad"].clone()
    for t in reversed(range(L)):
        g = g + q[:, t, :, None] * C[:, t, None, :]
        dC[:, t] = (q[:, t, :, None] * S[t + 1]).sum(1)
        dB[:, t] = (g * (d[:, t] * u[:, t])[:, :, None]).sum(1)
        gB = (g * B[:, t, None, :]).sum(-1)
        g = g * torch.exp(d[:, t, :, None] * A)
        gs = g * S[t]
        dd[:, t] = (gs * A).sum(-1) + u[:, t] * gB
        du[:, t] = s["D"] * q[:, t] + d[:, t] * gB
        dA += (gs * d[:, t, :, None]).sum(0)
    ddt = dd * _sigmoid(v) * live[:, :, None]
    packed = {k: a[live].to(t_) for k, a in dict(du=du, ddt=ddt, dz=dz, dB=dB, dC=dC).items()}
    return dict(packed, dA_log=dA * A, dD=(q * u).sum((0, 1)), db_dt=ddt.sum((0, 1)),
                dstate=g if s["state"] is not None else None)


# --- logits

def _segments(x, offs, V):
    """Ragged segments as rows of V, -inf where there is no entry."""
    idx = offs[:-1, None].long() + torch.arange(V, device=x.device)
    live = idx < offs[1:, None]
    return torch.where(live, x[torch.where(live, idx, 0)], -math.inf)


def _logit_rows(s):
    x = s["logits"].float()
    if s["offs"] is None:
        return x, 0
    return _segments(x, s["offs"], s["case"]["V"]), s["offs"][:-1, None].long()


def _plain_logprobs(s):
    case = s["case"]
    x, base = _logit_rows(s)
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    tok = s["tokens"][:, None].long() - base
    logp = (x.gather(1, tok) - lse)[:, 0]
    entropy = torch.log(total[:, 0]) - (e * (x - m).clamp(min=-1e30)).sum(1) / total[:, 0]
    K = min(case["K"], x.shape[1])
    val, idx = x.sort(dim=1, descending=True, stable=True)
    val, idx = val[:, :K], idx[:, :K]
    short = torch.zeros_like(idx, dtype=torch.bool)
    if s["offs"] is not None:
        short = idx >= (s["offs"][1:] - s["offs"][:-1])[:, None]
    pad = (0, case["K"] - K)
    top = torch.nn.functional.pad(torch.where(short, -1, idx + base), pad, value=-1).int()
    top_logp = torch.nn.functional.pad(torch.where(short, -math.inf, val - lse), pad, value=-math.inf)
    return dict(logp=logp, entropy=entropy, top=top, top_logp=top_logp)


def _plain_distill(s):
    case = s["case"]
    x, base = _logit_rows(s)
    x = x / 2.0
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    have = s["top"] >= 0
    idx = torch.where(have, s["top"].long() - base, 0)
    r = torch.where(have, s["teacher"] / 2.0, -math.inf)
    r = r - r.amax(1, keepdim=True)
    q = torch.exp(r)
    log_q = r - torch.log(q.sum(1, keepdim=True))
    q = torch.exp(log_q)
    logp = x.gather(1, idx) - m - torch.log(total)
    loss = torch.where(q > 0, q * (log_q - logp), 0.0).sum(1)
    w = s["weight"][:, None] / 2.0
    grad = (e / total).scatter_add_(1, idx, -q) * w
    if s["offs"] is not None:
        size = s["offs"][1:] - s["offs"][:-1]
        grad = grad[torch.arange(case["V"], device=x.device) < size[:, None]]
    return dict(loss=loss, grad=grad.to(s["logits"].dtype))


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    sz = 2 if case["dtype"] == "bf16" else 4
    n, kind = case["n"], case["kind"]
    if kind in ("logprobs", "distill"):
        K = case["K"]
        entries = int(_lengths(case).sum())
        if kind == "logprobs":
            # maximum, exponential and two sums
            return dict(bytes=entries * sz + n * (8 * K + 12), flops=6 * entries)
        return dict(bytes=2 * entries * sz + n * (8 * K + 8), flops=8 * entries)
    E = case["E"]
    rows = int(_lengths(case).sum())
    index = 4 * (n + 1) if case["L"] > 1 else 0
    if kind in ("conv", "conv_train"):
        K = case["K"]
        state = n * (K - 1) * E * sz
        if kind == "conv":
            return dict(bytes=2 * rows * E * sz + (2 * state if case["pool"] else 0) + 4 * E * (K + 1) + index,
                        flops=rows * E * (2 * K + 5))
        # x and du read, u and dx written
        return dict(bytes=4 * rows * E * sz + (3 * state if case["carry"] else 0) + 8 * E * (K + 1) + index,
                    flops=rows * E * (6 * K + 15))
    N = case["N"]
    state = 4 * n * E * N
    weights = 4 * E * (N + 2)
    if kind == "scan":
        # per state: a product and exponential, two products and two sums each
        return dict(bytes=rows * (4 * E + 2 * N) * sz + (2 * state if case["pool"] else 0) + weights + index,
                    flops=rows * E * (7 * N + 20))
    # u, dt, z, dy read, three gradients written, states and adjoints formed
    return dict(bytes=rows * (7 * E + 4 * N) * sz + (3 * state if case["carry"] else 0) + 2 * weights + index,
                flops=rows * E * (22 * N + 40))


# ---------------------------------------------------------------------------
# in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"conv": _exact_conv, "conv_train": _exact_conv_train, "scan": _exact_scan, "scan_train": _exact_scan_train,
            "logprobs": _exact_logprobs, "distill": _exact_distill}[case["kind"]](s)


def _positions(s, rows):
    """Of every packed row: its sequence and its place in it."""
    n = s["case"]["n"]
    dev = "cuda"
    if s["offs"] is None:
        return torch.arange(n, device=dev), torch.zeros(n, dtype=torch.long, device=dev), torch.ones(n, device=dev).long()
    lens = (s["offs"][1:] - s["offs"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(n, device=dev), lens)
    return seq, torch.arange(rows, device=dev) - s["offs"][:-1].long()[seq], lens


def _start64(state, slots, n, shape):
    out = torch.zeros(n, *shape, dtype=torch.float64, device="cuda")
    if state is None:
        return out
    if slots is None:
        out.copy_(state)
        return out
    for i, j in enumerate(slots.tolist()):
        if 0 <= j < state.shape[0]:
            out[i] = state[j]
    return out


def _end64(state_out, slots, end):
    if state_out is None:
        return None
    out = torch.zeros(state_out.shape, dtype=torch.float64, device="cuda")
    for i, j in enumerate(range(len(end)) if slots is None else slots.tolist()):
        if 0 <= j < out.shape[0]:
            out[j] = end[i]
    return out


def _taps(x, start, seq, pos, j):
    """x_{t-j} of every row, out of the sequence's state before its start."""
    K1 = start.shape[1]
    rows = torch.arange(x.shape[0], device=x.device)
    inside = pos >= j
    v = x[torch.where(inside, rows - j, rows)]
    if K1:
        back = start[seq, (K1 + pos - j).clamp(0, K1 - 1)]
        return torch.where(inside[:, None], v, back)
    return v


def _exact_conv(s):
    case = s["case"]
    K, E = case["K"], case["E"]
    x, w = s["x"].double(), s["w"].double()
    seq, pos, lens = _positions(s, x.shape[0])
    start = _start64(s["state"], s["slots"], case["n"], (K - 1, E))
    pre = s["b"].double().expand_as(x).clone()
    for j in range(K):
        pre += w[:, K - 1 - j] * _taps(x, start, seq, pos, j)
    end = start.clone()
    ext = torch.cat([start.reshape(-1, E), x])
    first = torch.cumsum(lens, 0) - lens
    for k in range(K - 1):
        t = lens - (K - 1) + k  # the token the new state's row k holds
        old = torch.arange(case["n"], device=x.device) * (K - 1) + K - 1 + t
        end[:, k] = ext[torch.where(t >= 0, case["n"] * (K - 1) + first + t, old)]
    return dict(u=pre / (1 + torch.exp(-pre)), state=_end64(s["state_out"], s["slots"], end))


def _exact_conv_train(s):
    case = s["case"]
    K, E, n = case["K"], case["E"], case["n"]
    x, w = s["x"].double(), s["w"].double()
    seq, pos, lens = _positions(s, x.shape[0])
    start = _start64(s["state"], None, n, (K - 1, E))
    pre = s["b"].double().expand_as(x).clone()
    for j in range(K):
        pre += w[:, K - 1 - j] * _taps(x, start, seq, pos, j)
    sig = torch.sigmoid(pre)
    g = s["grad"].double() * sig * (1 + pre * (1 - sig))
    dx = torch.zeros_like(x)
    dstart = torch.zeros_like(start)
    dw = torch.empty(E, K, dtype=torch.float64, device=x.device)
    rows = torch.arange(x.shape[0], device=x.device)
    left = lens[seq] - 1 - pos
    for j in range(K):
        # row t's value goes into row t + j
        dx += torch.where((left >= j)[:, None], g[(rows + j).clamp(max=x.shape[0] - 1)], 0.0) * w[:, K - 1 - j]
        dw[:, K - 1 - j] = (g * _taps(x, start, seq, pos, j)).sum(0)
        early = (pos < j).nonzero()[:, 0]
        dstart.index_put_((seq[early], K - 1 + pos[early] - j), g[early] * w[:, K - 1 - j], accumulate=True)
    if s["state_grad"] is not None:
        sg = s["state_grad"].double()
        for k in range(K - 1):
            t = lens - (K - 1) + k
            first = torch.cumsum(lens, 0) - lens
            has = (t >= 0).nonzero()[:, 0]
            dx[(first + t)[has]] += sg[has, k]
            not_ = (t < 0).nonzero()[:, 0]
            dstart[not_, (K - 1 + t)[not_]] += sg[not_, k]
    return dict(dx=dx, dw=dw, db=g.sum(0), dstate=dstart if s["state"] is not None else None, u=pre * sig)


def _prefix(a, b):
    """x_t = a_t x_{t-1} + b_t from x_{-1} = 0, along dim 1, by doubling."""
    a, b = a.clone(), b.clone()
    k = 1
    while k < a.shape[1]:
        b = torch.cat([b[:, :k], b[:, k:] + a[:, k:] * b[:, :-k]], 1)
        a = torch.cat([a[:, :k], a[:, k:] * a[:, :-k]], 1)
        k *= 2
    return b


def _scan64(s, backward):
    """Blocks of channels, padded batch, the recurrences by doubling."""
    case = s["case"]
    n, E, N = case["n"], case["E"], case["N"]
    rows = s["u"].shape[0]
    seq, pos, lens = _positions(s, rows)
    L = int(lens.max())
    dev = "cuda"

    def pad(a):
        out = torch.zeros(n, L, *a.shape[1:], dtype=torch.float64, device=dev)
        out[seq, pos] = a.double()
        return out

    Bm, Cm = pad(s["B"])[:, :, None], pad(s["C"])[:, :, None]
    live = torch.zeros(n, L, 1, dtype=torch.bool, device=dev)
    live[seq, pos] = True
    start = _start64(s["state"], None if backward else s["slots"], n, (E, N))
    t64 = dict(dtype=torch.float64, device=dev)
    o = {k: torch.empty(rows, E, **t64) for k in (("du", "ddt", "dz") if backward else ("y",))}
    end = torch.empty(n, E, N, **t64)
    if backward:
        o.update(dB=torch.zeros(rows, N, **t64), dC=torch.zeros(rows, N, **t64), dA_log=torch.empty(E, N, **t64),
                 dD=torch.empty(E, **t64), db_dt=torch.empty(E, **t64))
    step = max(1, min(E, int(1.0e8 // (n * L * N))))
    for e0 in range(0, E, step):
        c = slice(e0, min(E, e0 + step))
        u, z = pad(s["u"][:, c]), pad(s["z"][:, c])
        v = pad(s["dt"][:, c]) + s["b_dt"][c].double()
        d = torch.where(live, torch.nn.functional.softplus(v, threshold=1e4), 0.0)
        A = -torch.exp(s["A_log"][c].double())
        a = torch.exp(d[..., None] * A)
        b = (d * u)[..., None] * Bm
        b[:, 0] += a[:, 0] * start[:, c]
        S = _prefix(a, b)
        end[:, c] = S[:, -1]
        ypre = (S * Cm).sum(-1) + s["D"][c].double() * u
        sz = torch.sigmoid(z)
        if not backward:
            o["y"][:, c] = (ypre * z * sz)[seq, pos]
            continue
        dy = pad(s["grad"][:, c])
        q = dy * z * sz
        r = q[..., None] * Cm
        if s["state_grad"] is not None:
            r[:, -1] += s["state_grad"][:, c].double()
        nxt = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1)
        G = _prefix(nxt.flip(1), r.flip(1)).flip(1)
        gB = (G * Bm).sum(-1)
        prev = torch.cat([start[:, None, c], S[:, :-1]], 1)
        gs = G * a * prev
        ddt = ((gs * A).sum(-1) + u * gB) * torch.sigmoid(v)
        ddt = torch.where(live, ddt, 0.0)
        o["du"][:, c] = (s["D"][c].double() * q + d * gB)[seq, pos]
        o["ddt"][:, c] = ddt[seq, pos]
        o["dz"][:, c] = (dy * ypre * sz * (1 + z * (1 - sz)))[seq, pos]
        o["dB"] += (G * (d * u)[..., None]).sum(2)[seq, pos]
        o["dC"] += (S * q[..., None]).sum(2)[seq, pos]
        o["dA_log"][c] = (gs * d[..., None]).sum((0, 1)) * A
        o["dD"][c] = (q * u).sum((0, 1))
        o["db_dt"][c] = ddt.sum((0, 1))
        end[:, c] = a[:, 0] * G[:, 0]
    return o, end


def _exact_scan(s):
    o, end = _scan64(s, False)
    return dict(y=o["y"], state=_end64(s["state_out"], s["slots"], end))


def _exact_scan_train(s):
    o, end = _scan64(s, True)
    return dict(o, dstate=end if s["state"] is not None else None)


def _exact_logprobs(s):
    case = s["case"]
    x = s["logits"]
    n, K = case["n"], case["K"]
    ends = None if s["offs"] is None else s["offs"].tolist()
    r = dict(logp=[], entropy=[], top=[], top_logp=[])
    group = n if ends is None else 1  # rows of one length go together
    for i in range(0, n, group):
        rows = x.double() if ends is None else x[ends[i]:ends[i + 1]].double()[None]
        base = 0 if ends is None else ends[i]
        lse = torch.logsumexp(rows, 1, keepdim=True)
        lp = rows - lse
        r["logp"].append(lp.gather(1, s["tokens"][i:i + group, None].long() - base)[:, 0])
        r["entropy"].append(-torch.special.xlogy(torch.exp(lp), torch.exp(lp)).sum(1))
        k = min(K, rows.shape[1])
        idx = torch.argsort(-rows, dim=1, stable=True)[:, :k]
        top = torch.full((len(rows), K), -1, dtype=torch.int32, device=x.device)
        top_logp = torch.full((len(rows), K), -math.inf, dtype=torch.float64, device=x.device)
        top[:, :k] = (idx + base).int()
        top_logp[:, :k] = lp.gather(1, idx)
        r["top"].append(top)
        r["top_logp"].append(top_logp)
    return {k: torch.cat(v) for k, v in r.items()}


def _exact_distill(s):
    case = s["case"]
    x, T = s["logits"], 2.0
    n = case["n"]
    ends = None if s["offs"] is None else s["offs"].tolist()
    loss = torch.empty(n, dtype=torch.float64, device=x.device)
    grad = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    group = 64 if ends is None else 1
    for i in range(0, n, group):
        j = min(n, i + group)
        part = x[i:j] if ends is None else x[ends[i]:ends[i + 1]][None]
        base = 0 if ends is None else ends[i]
        lp = torch.log_softmax(part.double() / T, 1)
        g = torch.exp(lp)
        for k in range(i, j) if ends is not None else [slice(i, j)]:
            top = s["top"][k].reshape(-1, s["top"].shape[1]).long()
            have = top >= 0
            lq = torch.log_softmax(torch.where(have, s["teacher"][k].reshape(top.shape).double() / T, -math.inf), 1)
            q = torch.exp(lq)
            at = torch.where(have, top - base, 0)
            term = torch.where(q > 0, q * (lq - lp.gather(1, at)), 0.0)
            loss[i:j] = term.sum(1)
            g.scatter_add_(1, at, -q)
        g = g * s["weight"][i:j, None].double() / T
        if ends is None:
            grad[i:j] = g
        else:
            grad[ends[i]:ends[i + 1]] = g[0]
    return dict(loss=loss, grad=grad)
