"""More operators of layers that carry states and of models that answer, as
cases that can be timed and compared: layer norm with its gradients, the gated
delta rule with carried states (prompts, single tokens, gradients), and beam
search's selection with the reordering of the beams' states.

  own                 False: `run` is the operators' plain form, elementary
                      torch operations in 32 bits; True: the framework's calls
  listed()            the cases, dicts of plain values
  draw(rng)           one more case of the same ranges
  prepare(case, seed) inputs and buffers, as a program holds them
  run(state)          one pass through an operator; its outputs
  work(case)          bytes and operations that one pass cannot do without
  exact(case, seed)   the same outputs in 64 bits

Sequences are packed: sequence i owns rows offs[i] .. offs[i+1]-1 of every
activation. Queries and keys have unit length, as layers that use the rule give
them; several value heads share a key head. Decays are exp(g) with g around
-0.003 to -1, write strengths beta in (0, 1). Beams' scores are sums of log
probabilities, some beams of a group dead or ended.
"""
from __future__ import annotations

import math

import torch

own = False


def listed():
    return [
        # the smallest call: the norm of a few sequences' tokens, latency only
        dict(name="norm_token_bf16", kind="norm", dtype="bf16", rows=16, C=2048),
        # forward and backward over the rows of a training batch, a width that is no power of two
        dict(name="norm_train_bf16", kind="norm_train", dtype="bf16", rows=16384, C=5120),
        # the same at this repository's own width, where rows are many and short
        dict(name="norm_train_narrow_f32", kind="norm_train", dtype="f32", rows=102400, C=256),
        # one token of each of a few sequences, latency only
        dict(name="delta_token_few_f32", kind="delta", dtype="f32", n=4, L=1, lo=1, Hk=4, H=4, Dk=64, Dv=64, pool=4),
        # a serving batch, one token each, states in a pool
        dict(name="delta_token_bf16", kind="delta", dtype="bf16", n=192, L=1, lo=1, Hk=16, H=32, Dk=128, Dv=128,
             pool=256),
        # one long prompt, whose end state is kept
        dict(name="delta_prompt_bf16", kind="delta", dtype="bf16", n=1, L=8192, lo=8000, Hk=16, H=32, Dk=128, Dv=128,
             pool=1),
        # gradients on packed documents of uneven length, states and their gradients carried from and to neighbours
        dict(name="delta_train_bf16", kind="delta_train", dtype="bf16", n=4, L=2048, lo=700, Hk=8, H=16, Dk=128,
             Dv=128, carry=True),
        # gradients on short sequences, 64 wide heads
        dict(name="delta_train_f32", kind="delta_train", dtype="f32", n=64, L=256, lo=9, Hk=8, H=8, Dk=64, Dv=64,
             carry=False),
        # one request of four beams, an odd vocabulary
        dict(name="select_few_f32", kind="select", dtype="f32", groups=1, W=4, K=4, V=50001, masked=0.0),
        # a batch of requests, twice as many candidates as beams, part of the entries masked
        dict(name="select_batch_bf16", kind="select", dtype="bf16", groups=64, W=8, K=16, V=131072, masked=0.1),
        # the convolution's and the rule's states of one small request
        dict(name="reorder_few_f32", kind="reorder", dtype="f32", groups=1, W=4, pool=6, conv=3 * 768, state=4 * 64 * 64),
        # those of a batch of requests, in pools that hold other sequences too
        dict(name="reorder_batch_bf16", kind="reorder", dtype="bf16", groups=48, W=8, pool=400, conv=3 * 8192,
             state=32 * 128 * 128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_train", "norm_train", "delta", "delta", "delta_token", "delta_train",
                       "delta_train", "select", "select", "reorder"])
    dtype = rng.choice(["f32", "bf16"])
    if kind in ("norm", "norm_train"):
        C = rng.choice([rng.choice([64, 128, 256, 512, 1024, 2048, 4096, 8192]), 8 * _log(rng, 8, 1024),
                        _log(rng, 30, 16384)])
        return dict(kind=kind, dtype=dtype, rows=_log(rng, 1, (83_000_000 if dtype == "bf16" else 41_000_000) // C), C=C)
    if kind == "select":
        V = _log(rng, 50, 131072)
        W = rng.choice([1, 2, 3, 4, 5, 8, 10, 16])
        groups = _log(rng, 1, max(1, min(256, (66_000_000 if dtype == "bf16" else 33_000_000) // (V * W))))
        return dict(kind=kind, dtype=dtype, groups=groups, W=W, K=rng.choice([W, 2 * W]), V=V,
                    masked=rng.choice([0.0, 0.0, 0.2]))
    if kind == "reorder":
        W = rng.choice([1, 2, 3, 4, 5, 8, 10, 16, 32])
        groups = _log(rng, 1, max(1, 384 // W))
        n = groups * W
        state = _log(rng, 64, min(500_000, 200_000_000 // n))
        return dict(kind=kind, dtype=dtype, groups=groups, W=W, pool=n + rng.randint(0, 8),
                    conv=rng.randint(1, 3) * rng.choice([rng.randint(60, 900), 8 * rng.randint(16, 1024)]), state=state)
    Hk = rng.choice([1, 2, 3, 4, 8, 16])
    H = Hk * rng.choice([1, 1, 2, 3])
    wide = rng.random() < 0.6
    Dk = rng.choice([64, 128]) if wide else 8 * rng.randint(1, 16)
    Dv = rng.choice([Dk, Dk, 2 * Dk]) if wide else 8 * rng.randint(1, 32)
    if kind == "delta_token":
        n = _log(rng, 1, max(1, min(2048, 100_000_000 // (H * Dk * Dv))))
        return dict(kind="delta", dtype=dtype, n=n, L=1, lo=1, Hk=Hk, H=H, Dk=Dk, Dv=Dv, pool=n + rng.randint(0, n))
    train = kind == "delta_train"
    L = _log(rng, 2, 1600 if train else 6000)
    most = (1_000_000_000 if train else 2_000_000_000) // (H * Dk * Dv * L)
    n = _log(rng, 1, max(1, min(512, most)))
    lo = rng.choice([1, max(1, L // 5), L])
    if train:
        return dict(kind=kind, dtype=dtype, n=n, L=L, lo=lo, Hk=Hk, H=H, Dk=Dk, Dv=Dv, carry=rng.random() < 0.5)
    return dict(kind=kind, dtype=dtype, n=n, L=L, lo=lo, Hk=Hk, H=H, Dk=Dk, Dv=Dv, pool=rng.choice([0, n]))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case):
    """The lengths of a case's sequences: the case's own, whatever the seed,
    which only orders them."""
    n, L = case["n"], case["L"]
    g = torch.Generator().manual_seed(1000003 * n + L)
    return torch.randint(case["lo"], L + 1, (n,), generator=g)


def _parents(case, g):
    """Children of a group's beams as a search gives them: a good beam has
    several, so that about a third of the beams has none."""
    G, W = case["groups"], case["W"]
    p = torch.randint(0, W, (G, W), generator=g, device="cuda")
    q = torch.arange(W, device="cuda").expand(G, W)
    p = torch.where(torch.rand(G, W, generator=g, device="cuda") < 0.5, p, q)
    p = p + W * torch.arange(G, device="cuda")[:, None]
    if G * W >= 16:
        p[G // 2, W - 1] = -1  # a group with fewer candidates than beams
    return p.int()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = _type(case)
    kind = case["kind"]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    s = dict(case=case)
    if kind in ("norm", "norm_train"):
        rows, C = case["rows"], case["C"]
        # rows with a level and a spread of their own, some channels larger than the others
        x = randn(rows, C) * (0.3 + 2.0 * rand(rows, 1)) + 0.5 * randn(rows, 1)
        s["x"] = x.mul_(torch.exp(0.5 * randn(C))).to(t)
        s["w"] = 1.0 + 0.3 * randn(C)
        s["b"] = 0.3 * randn(C)
        if kind == "norm_train":
            s["dy"] = randn(rows, C).to(t)
        return s
    if kind == "select":
        G, W, V = case["groups"], case["W"], case["V"]
        x = 2.5 * randn(G * W, V) + randn(G * W, 1)
        if case["masked"]:
            x.masked_fill_(rand(G * W, V) < case["masked"], -math.inf)
        s["logits"] = x.to(t)
        s["score"] = -20.0 * rand(G, 1) - 3.0 * rand(G, W)
        s["ended"] = torch.full((G, W), -1, dtype=torch.int32, device="cuda")
        if W > 2:
            s["ended"][::2, W - 1] = 2  # the end token
            s["score"][::3, 0] = -math.inf  # a beam that is none yet
        return s
    if kind == "reorder":
        n, pool = case["groups"] * case["W"], case["pool"]
        s["parent"] = _parents(case, g)
        s["slots"] = torch.randperm(pool, generator=g, device="cuda")[:n].int().view(case["groups"], case["W"])
        s["pools"] = [randn(pool, case["conv"]).to(t), randn(pool, case["state"])]
        return s

    H, Hk, Dk, Dv, n = case["H"], case["Hk"], case["Dk"], case["Dv"], case["n"]
    rows = int(_lengths(case).sum())
    s["offs"] = None
    if case["L"] > 1:
        lengths = _lengths(case).cuda()[torch.randperm(n, generator=g, device="cuda")]
        s["offs"] = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        s["offs"][1:] = lengths.cumsum(0)
    unit = lambda a: a / (a * a).sum(-1, keepdim=True).sqrt()  # noqa: E731
    s["q"] = unit(randn(rows, Hk, Dk)).to(t)
    s["k"] = unit(randn(rows, Hk, Dk)).to(t)
    v = randn(rows, H, Dv)
    s["v"] = (v / (1.0 + torch.exp(-v))).to(t)
    # decays of the heads' own rates, some heads that hardly forget
    rate = torch.exp(math.log(0.03) + math.log(30.0) * rand(H))
    s["g"] = -rate * (0.1 + rand(rows, H))
    s["beta"] = 1.0 / (1.0 + torch.exp(-randn(rows, H)))
    if kind == "delta":
        s["state"] = s["state_out"] = s["slots"] = None
        if case["pool"]:
            s["slots"] = torch.randperm(case["pool"], generator=g, device="cuda")[:n].int()
            if case["L"] == 1 and n >= 8:
                s["slots"][n // 2] = -1  # a sequence that pads the batch
            s["state"] = 0.2 * randn(case["pool"], H, Dk, Dv)
            s["state_out"] = torch.zeros(case["pool"], H, Dk, Dv, device="cuda")
    else:
        s["do"] = randn(rows, H, Dv).to(t)
        s["state"] = s["state_grad"] = None
        if case["carry"]:
            s["state"] = 0.2 * randn(n, H, Dk, Dv)
            s["state_grad"] = 0.1 * randn(n, H, Dk, Dv)
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    if own:
        return _own(s)
    return {"norm": _plain_norm, "norm_train": _plain_norm, "delta": _plain_delta, "delta_train": _plain_delta_train,
            "select": _plain_select, "reorder": _plain_reorder}[s["case"]["kind"]](s)


def _own(s):
    from paper_2604_12891_amd import binding as tb
    kind = s["case"]["kind"]
    if kind == "norm":
        return dict(y=tb.layer_norm(s["x"], s["w"], s["b"]))
    if kind == "norm_train":
        y = tb.layer_norm(s["x"], s["w"], s["b"])
        return dict(tb.layer_norm_backward(s["x"], s["w"], s["dy"]), y=y)
    if kind == "delta":
        o = tb.delta_rule(s["q"], s["k"], s["v"], s["g"], s["beta"], offs=s["offs"], state=s["state"],
                          state_out=s["state_out"], slots=s["slots"])
        return dict(o=o, state=s["state_out"])
    if kind == "delta_train":
        return tb.delta_rule_backward(s["q"], s["k"], s["v"], s["g"], s["beta"], s["do"], offs=s["offs"],
                                      state=s["state"], state_grad=s["state_grad"])
    if kind == "select":
        return tb.beam_select(s["logits"], s["score"], K=s["case"]["K"], ended=s["ended"])
    slots = tb.beam_reorder(s["parent"], s["slots"], s["pools"])
    return dict(slots=slots, conv=s["pools"][0], state=s["pools"][1])


# --- layer norm

def _plain_norm(s):
    x, w, b = s["x"].float(), s["w"], s["b"]
    t = s["x"].dtype
    c = x - x.mean(1, keepdim=True)
    r = 1.0 / ((c * c).mean(1, keepdim=True) + 1e-5).sqrt()
    h = c * r
    y = (h * w + b).to(t)
    if s["case"]["kind"] == "norm":
        return dict(y=y)
    dy = s["dy"].float()
    g = dy * w
    dx = r * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return dict(y=y, dx=dx.to(t), dw=(dy * h).sum(0), db=dy.sum(0))


# --- gated delta rule

def _dense(a, s):
    """Packed rows as a padded batch [n, L, ...] in 32 bits, zero where there
    is no token."""
    if s["offs"] is None:
        return a.float()[:, None]
    idx = s["offs"][:-1, None].long() + torch.arange(s["case"]["L"], device=a.device)
    live = idx < s["offs"][1:, None]
    d = a.float()[torch.where(live, idx, 0)]
    return d * live.view(*live.shape, *([1] * (a.dim() - 1)))


def _live(s):
    n, L = s["case"]["n"], s["case"]["L"]
    if s["offs"] is None:
        return torch.ones(n, 1, dtype=torch.bool, device="cuda")
    return torch.arange(L, device="cuda") < (s["offs"][1:] - s["offs"][:-1])[:, None]


def _delta_inputs(s):
    case = s["case"]
    r = case["H"] // case["Hk"]
    q, k = (_dense(s[x], s).repeat_interleave(r, 2) for x in ("q", "k"))
    # past a sequence's end g and beta are 0: the state stays as it is
    return q / math.sqrt(case["Dk"]), k, _dense(s["v"], s), torch.exp(_dense(s["g"], s)), _dense(s["beta"], s)


def _plain_delta(s):
    case = s["case"]
    q, k, v, a, beta = _delta_inputs(s)
    S = torch.zeros(case["n"], case["H"], case["Dk"], case["Dv"], device=q.device)
    ok = None
    if s["state"] is not None:
        ok = (s["slots"] >= 0) & (s["slots"] < case["pool"])
        S = s["state"][torch.where(ok, s["slots"], 0).long()] * ok[:, None, None, None]
    o = torch.empty_like(v)
    for t in range(q.shape[1]):
        S = S * a[:, t, :, None, None]
        u = beta[:, t, :, None] * (v[:, t] - (S * k[:, t, :, :, None]).sum(2))
        S = S + k[:, t, :, :, None] * u[:, :, None, :]
        o[:, t] = (S * q[:, t, :, :, None]).sum(2)
    if s["state_out"] is not None:
        s["state_out"][s["slots"][ok].long()] = S[ok]
    return dict(o=o[_live(s)].to(s["v"].dtype), state=s["state_out"])


def _plain_delta_train(s):
    case = s["case"]
    n, H, Hk, Dk, Dv = (case[x] for x in ("n", "H", "Hk", "Dk", "Dv"))
    t_ = s["v"].dtype
    q, k, v, a, beta = _delta_inputs(s)
    do = _dense(s["do"], s)
    L = q.shape[1]
    S = torch.empty(L + 1, n, H, Dk, Dv, device=q.device)
    S[0] = 0.0 if s["state"] is None else s["state"]
    u = torch.empty_like(v)
    for t in range(L):
        torch.mul(S[t], a[:, t, :, None, None], out=S[t + 1])
        u[:, t] = v[:, t] - (S[t + 1] * k[:, t, :, :, None]).sum(2)
        S[t + 1] += k[:, t, :, :, None] * (beta[:, t, :, None] * u[:, t])[:, :, None, :]
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    da, dbeta = torch.empty_like(a), torch.empty_like(beta)
    G = torch.zeros(n, H, Dk, Dv, device=q.device) if s["state_grad"] is None else s["state_grad"].clone()
    for t in reversed(range(L)):
        G = G + q[:, t, :, :, None] * do[:, t, :, None, :]
        dq[:, t] = (S[t + 1] * do[:, t, :, None, :]).sum(3)
        du = (G * k[:, t, :, :, None]).sum(2)
        dbeta[:, t] = (du * u[:, t]).sum(2)
        du = du * beta[:, t, :, None]
        dv[:, t] = du
        # the key writes with u and reads the decayed state
        D = S[t] * a[:, t, :, None, None]
        dk[:, t] = (G * (beta[:, t, :, None] * u[:, t])[:, :, None, :]).sum(3) - (D * du[:, :, None, :]).sum(3)
        G = G - k[:, t, :, :, None] * du[:, :, None, :]
        da[:, t] = (G * D).sum((2, 3))
        G = G * a[:, t, :, None, None]
    live = _live(s)
    dq = dq.view(n, L, Hk, H // Hk, Dk).sum(3) / math.sqrt(Dk)
    dk = dk.view(n, L, Hk, H // Hk, Dk).sum(3)
    return dict(dq=dq[live].to(t_), dk=dk[live].to(t_), dv=dv[live].to(t_), dg=da[live], dbeta=dbeta[live],
                dstate=G if s["state"] is not None else None)


# --- beam search

def _plain_select(s):
    case = s["case"]
    G, W, V, K = (case[x] for x in ("groups", "W", "V", "K"))
    # candidates next to each other in their order are told apart in 64 bits
    x = s["logits"].double()
    m = x.amax(1, keepdim=True)
    x = x - (m + torch.log(torch.exp(x - m).sum(1, keepdim=True)))
    cand = (s["score"].double().view(-1, 1) + x).view(G, W, V)
    # an ended beam is a candidate itself, as its end token
    ended = s["ended"][:, :, None].long()
    only = torch.arange(V, device=x.device) == ended
    cand = torch.where(ended >= 0, torch.where(only, s["score"].double()[:, :, None], -math.inf), cand).view(G, W * V)
    k = min(K, W * V)
    val, idx = cand.sort(dim=1, descending=True, stable=True)
    val, idx = val[:, :k], idx[:, :k]
    none = val == -math.inf
    pad = torch.nn.functional.pad
    parent = torch.where(none, -1, idx // V + W * torch.arange(G, device=x.device)[:, None])
    return dict(parent=pad(parent, (0, K - k), value=-1).int(),
                token=pad(torch.where(none, -1, idx % V), (0, K - k), value=-1).int(),
                score=pad(val, (0, K - k), value=-math.inf).float())


def _plain_reorder(s):
    case = s["case"]
    G, W = case["groups"], case["W"]
    base = W * torch.arange(G, device="cuda")[:, None]
    p = s["parent"].long() - base
    has = (p >= 0) & (p < W)
    order = torch.arange(W, device="cuda")
    same = (p[:, :, None] == p[:, None, :]) & has[:, :, None]
    first = has & ~(same & (order[None, :] < order[:, None])).any(2)
    childless = ~((p[:, None, :] == order[None, :, None]) & has[:, None, :]).any(2)
    # the others take the childless beams' places, both in their order
    free = torch.sort((~childless).int(), dim=1, stable=True)[1]
    rank = (torch.cumsum((~first).int(), 1) - 1).clamp(min=0)
    parent = torch.where(has, p, 0)
    slots = s["slots"].gather(1, torch.where(first, parent, free.gather(1, rank)))
    source = s["slots"].gather(1, parent)
    moved = has & ~first
    for pool in s["pools"]:
        pool[slots[moved].long()] = pool[source[moved].long()]
    return dict(slots=slots, conv=s["pools"][0], state=s["pools"][1])


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    sz = 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if kind == "norm":
        return dict(bytes=2 * case["rows"] * case["C"] * sz + 8 * case["C"], flops=8 * case["rows"] * case["C"])
    if kind == "norm_train":
        # x and dy read, y and dx written
        return dict(bytes=4 * case["rows"] * case["C"] * sz + 16 * case["C"], flops=24 * case["rows"] * case["C"])
    if kind == "select":
        n = case["groups"] * case["W"]
        # beams that are dead or have ended are not read
        if case["W"] > 2:
            n -= (case["groups"] + 1) // 2 + (case["groups"] + 2) // 3
        return dict(bytes=n * case["V"] * sz + case["groups"] * (8 * case["W"] + 12 * case["K"]), flops=4 * n * case["V"])
    if kind == "reorder":
        g = torch.Generator(device="cuda").manual_seed(1)
        p = _parents(case, g)
        # beams that keep no state of their own: one copy for each second child
        copies = int((p >= 0).sum()) - len(set(p[p >= 0].tolist()))
        return dict(bytes=2 * max(copies, 1) * (case["conv"] * sz + 4 * case["state"]) + 12 * p.numel(), flops=0)
    rows = int(_lengths(case).sum())
    H, Hk, Dk, Dv, n = (case[x] for x in ("H", "Hk", "Dk", "Dv", "n"))
    state = 4 * n * H * Dk * Dv
    acts = rows * (2 * Hk * Dk + 2 * H * Dv) * sz + 8 * rows * H
    # per token and head: decay, read, write and answer of a state
    if kind == "delta":
        return dict(bytes=acts + (2 * state if case["pool"] else 0), flops=7 * rows * H * Dk * Dv)
    # q, k, v, do read, three gradients written; states formed, adjoints walked back
    return dict(bytes=acts + rows * (2 * Hk * Dk + H * Dv) * sz + 8 * rows * H + (3 * state if case["carry"] else 0),
                flops=20 * rows * H * Dk * Dv)


# ---------------------------------------------------------------------------
# in 64 bits
# ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "norm_train": _exact_norm, "delta": _exact_delta, "delta_train": _exact_delta,
            "select": _exact_select, "reorder": _exact_reorder}[case["kind"]](s)


def _exact_norm(s):
    train = s["case"]["kind"] == "norm_train"
    C = s["case"]["C"]
    w, b = s["w"].double(), s["b"].double()
    y, dx = [], []
    dw, db = torch.zeros_like(w), torch.zeros_like(w)
    for part in torch.arange(len(s["x"]), device="cuda").split(4096):
        x = s["x"][part].double()
        var, mean = torch.var_mean(x, 1, unbiased=False, keepdim=True)
        h = (x - mean) * torch.rsqrt(var + 1e-5)
        y.append(torch.addcmul(b, h, w))
        if train:
            dy = s["dy"][part].double()
            dh = dy * w
            both = torch.stack([torch.ones_like(h), h])  # what the norm takes out of a gradient
            dx.append((dh - (both * (both * dh).sum(2, keepdim=True) / C).sum(0)) * torch.rsqrt(var + 1e-5))
            dw += (h * dy).sum(0)
            db += dy.sum(0)
    r = dict(y=torch.cat(y))
    if train:
        r.update(dx=torch.cat(dx), dw=dw, db=db)
    return r


def _exact_delta(s):
    """In chunks of 32 tokens, each a triangular system for what its tokens
    write; gradients by torch's own differentiation of that."""
    case = s["case"]
    train = case["kind"] == "delta_train"
    n, H, Hk, Dk, Dv, L = (case[x] for x in ("n", "H", "Hk", "Dk", "Dv", "L"))
    rows = len(s["q"])
    dev = "cuda"
    lens = torch.ones(n, dtype=torch.long, device=dev) if s["offs"] is None else (s["offs"][1:] - s["offs"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(n, device=dev), lens)
    pos = torch.arange(rows, device=dev) - (torch.cumsum(lens, 0) - lens)[seq]
    T = 32
    chunks = -(-L // T)
    start = torch.zeros(n, H, Dk, Dv, dtype=torch.float64, device=dev)
    slots = None if train or s["slots"] is None else s["slots"].tolist()
    if s["state"] is not None:
        for i, j in enumerate(range(n) if train else slots):
            if 0 <= j < len(s["state"]):
                start[i] = s["state"][j]
    leaf = {x: s[x].double() for x in ("q", "k", "v", "g", "beta")}
    leaf["state"] = start
    if train:
        for x in leaf.values():
            x.requires_grad_(True)
        do = torch.zeros(n, chunks * T, H, Dv, dtype=torch.float64, device=dev)
        do[seq, pos] = s["do"].double()

    def pad(a):
        full = torch.zeros(n, chunks * T, *a.shape[1:], dtype=torch.float64, device=dev)
        full = full.index_put((seq, pos), a)
        return full.transpose(1, 2)  # [n, heads, time, ...]

    share = torch.arange(H, device=dev) // (H // Hk)
    q, k = pad(leaf["q"])[:, share] * Dk ** -0.5, pad(leaf["k"])[:, share]
    v, g, beta = pad(leaf["v"]), pad(leaf["g"]), pad(leaf["beta"])
    lower = torch.tril(torch.ones(T, T, dtype=torch.bool, device=dev))
    eye = torch.eye(T, dtype=torch.float64, device=dev)
    S, loss, out = leaf["state"], 0.0, []
    for c in range(chunks):
        at = slice(c * T, (c + 1) * T)
        qc, kc, vc, bc = q[:, :, at], k[:, :, at], v[:, :, at], beta[:, :, at, None]
        G = torch.cumsum(g[:, :, at], 2)
        decay = torch.exp(torch.where(lower, G[..., :, None] - G[..., None, :], -1e9))
        kt = kc.transpose(2, 3).contiguous()
        M = eye + bc * torch.tril(decay * torch.matmul(kc, kt), -1)
        e = torch.exp(G)[..., None]
        u = torch.linalg.solve_triangular(M, bc * (vc - e * torch.matmul(kc, S)), upper=False)
        o = e * torch.matmul(qc, S) + torch.matmul(decay * torch.matmul(qc, kt), u)
        S = e[:, :, -1:] * S + torch.matmul((kc * torch.exp(G[:, :, -1:] - G)[..., None]).transpose(2, 3).contiguous(), u)
        if train:
            loss = loss + (o.transpose(1, 2) * do[:, at]).sum()
        else:
            out.append(o.transpose(1, 2))
    if not train:
        end = None
        if s["state_out"] is not None:
            end = torch.zeros(s["state_out"].shape, dtype=torch.float64, device=dev)
            for i, j in enumerate(slots):
                if 0 <= j < len(end):
                    end[j] = S[i]
        return dict(o=torch.cat(out, 1)[seq, pos], state=end)
    if s["state_grad"] is not None:
        loss = loss + (S * s["state_grad"].double()).sum()
    names = list(leaf)
    grads = dict(zip(names, torch.autograd.grad(loss, [leaf[x] for x in names])))
    return dict({"d" + x: grads[x] for x in names if x != "state"},
                dstate=grads["state"] if s["state"] is not None else None)


def _exact_select(s):
    case = s["case"]
    G, W, V, K = (case[x] for x in ("groups", "W", "V", "K"))
    parent = torch.full((G, K), -1, dtype=torch.int32, device="cuda")
    token, score = parent.clone(), torch.full((G, K), -math.inf, dtype=torch.float64, device="cuda")
    ended = s["ended"].tolist()
    for g in range(G):
        lp = torch.log_softmax(s["logits"][g * W:(g + 1) * W].double(), 1) + s["score"][g, :, None].double()
        for w in range(W):
            if ended[g][w] >= 0:
                lp[w] = -math.inf
                lp[w, ended[g][w]] = s["score"][g, w].double()
        best = torch.argsort(-lp.reshape(-1), stable=True)[:K]
        best = best[lp.reshape(-1)[best] > -math.inf]
        parent[g, :len(best)] = (best // V + g * W).int()
        token[g, :len(best)] = (best % V).int()
        score[g, :len(best)] = lp.reshape(-1)[best]
    return dict(parent=parent, token=token, score=score)


def _exact_reorder(s):
    G, W = s["case"]["groups"], s["case"]["W"]
    old, parent = s["slots"].tolist(), s["parent"].tolist()
    new, pools = [], [p.double() for p in s["pools"]]
    for g in range(G):
        kept, got = set(), [None] * W
        for i, p in enumerate(parent[g]):
            if g * W <= p < (g + 1) * W and p not in kept:
                kept.add(p)
                got[i] = old[g][p - g * W]
        free = [old[g][w] for w in range(W) if g * W + w not in kept]
        for i, p in enumerate(parent[g]):
            if got[i] is None:
                got[i] = free.pop(0)
                if g * W <= p < (g + 1) * W:
                    for a, b in zip(pools, s["pools"]):
                        a[got[i]] = b[old[g][p - g * W]].double()
        new.append(got)
    return dict(slots=torch.tensor(new, dtype=torch.int32, device="cuda"), conv=pools[0], state=pools[1])
