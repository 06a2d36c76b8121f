"""Calls of layer norm, the delta rule and beam search at the edges of what their documentation
allows: pools and arrays past 32 bits, slots in prompts, sequences of very different lengths, NaN that stays
where it is."""
import numpy as np
import pytest
import torch

from oracle import layer as ol
from oracle import search as osr
from tests.test_gpu_delta import DT, GRADS, _case, _gpu, _near, tolerance

pytestmark = pytest.mark.gpu
NAN = float("nan")


def _tb():
    from paper_2604_12891_amd import binding as tb
    return tb


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [[70, 130, 0, 65, 64], [200] + [1] * 20, [3, 2, 5]])
def test_prompts_with_slots(lens, dtype):
    """States in a pool by slots, some sequences without one; other places untouched; a result with a leading
    dimension."""
    print(f"prompts with slots lens={lens} {dtype}", flush=True)
    tb, rng, n, H, Dk, Dv = _tb(), np.random.default_rng(1), len(lens), 2, 40, 48
    pool = n + 4
    slots = rng.permutation(pool)[:n].astype(np.int32)
    slots[1] = -1
    slots[-1] = pool + 7
    live = (slots >= 0) & (slots < pool)
    a = _case(lens, 1, H, Dk, Dv, dtype, 4, False)
    x, offs, T = _gpu(a, dtype, True), torch.from_numpy(a["offs"]).cuda(), sum(lens)
    start = rng.standard_normal((pool, H, Dk, Dv)).astype(np.float32)
    a["state"] = np.where(live[:, None, None, None], start[np.where(live, slots, 0)], 0).astype(np.float64)
    r = ol.delta_rule(**a)
    want = start.astype(np.float64)
    want[slots[live]] = r["end"][live]
    S = torch.from_numpy(start).cuda()
    wide = torch.full((T + 2, H * Dv + 9), 7.0, dtype=DT[dtype], device="cuda")
    out = wide[:, 1:1 + H * Dv].unflatten(1, (H, Dv))
    tb.delta_rule(**x, offs=offs, state=S, state_out=S, slots=torch.from_numpy(slots).cuda(), out=out)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    _near("o", out[:T], r["o"], tolerance(Dk, lens) + half)
    _near("pool", S, want, tolerance(Dk, lens))
    rest = np.setdiff1d(np.arange(pool), slots[live])
    assert np.array_equal(S.cpu().numpy()[rest], start[rest])
    assert (wide[T:] == 7.0).all() and (wide[:, 0] == 7.0).all() and (wide[:, 1 + H * Dv:] == 7.0).all()
    # end states kept without states to start from
    S.fill_(7.0)
    a["state"] = None
    end = ol.delta_rule(**a)["end"]
    tb.delta_rule(**x, offs=offs, state_out=S, slots=torch.from_numpy(slots).cuda())
    _near("ends", S[torch.from_numpy(slots[live]).long()], end[live], tolerance(Dk, lens))
    assert (S[torch.from_numpy(rest).long()] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_stays_in_its_sequence_and_head(dtype):
    """NaN in one head's value, or in a key, of one sequence: other sequences' and other heads' results have the
    same bits as without."""
    tb, lens, H, D = _tb(), [90, 40, 70], 4, 64
    a = _case(lens, 2, H, D, D, dtype, 6)
    offs, S = torch.from_numpy(a["offs"]).cuda(), torch.from_numpy(a["state"]).float().cuda()
    do = torch.randn(sum(lens), H, D, device="cuda").to(DT[dtype])

    def results(x):
        end = torch.empty_like(S)
        o = tb.delta_rule(**x, offs=offs, state=S, state_out=end)
        g = tb.delta_rule_backward(**x, do=do, offs=offs, state=S, state_grad=S)
        return dict(g, o=o, end=end)

    x = _gpu(a, dtype, False, spare=0)
    clean = results(x)
    for name, head, hit in (("v", 1, [1]), ("k", 1, [2, 3]), ("g", 0, [0]), ("beta", 3, [3])):
        y = dict(x, **{name: x[name].clone()})
        y[name][100, head] = NAN  # in the second sequence
        r = results(y)
        other = torch.tensor([h for h in range(H) if h not in hit], device="cuda")
        rows = torch.cat([torch.arange(0, 90), torch.arange(130, 200)]).cuda()
        for k in ("o", "dv", "dg", "dbeta"):
            assert torch.equal(r[k][rows], clean[k][rows]) and torch.equal(r[k][:, other], clean[k][:, other]), (name, k)
        for k in ("dq", "dk"):  # (key heads: heads 0 and 1 share the first)
            other_k = 1 - hit[0] // 2
            assert torch.equal(r[k][rows], clean[k][rows]) and torch.equal(r[k][:, other_k], clean[k][:, other_k]), (name, k)
        for k in ("end", "dstate"):
            assert torch.equal(r[k][[0, 2]], clean[k][[0, 2]]) and torch.equal(r[k][:, other], clean[k][:, other]), (name, k)
        assert torch.isnan(r["o"][100:130, hit[0]]).any()


def test_states_past_32_bits():
    """Slots whose states lie beyond 2^32 bytes of their pool, read and written there."""
    tb, H, D, pool = _tb(), 32, 128, 2100  # 2 MiB each
    S = torch.zeros(pool, H, D, D, device="cuda")
    for lens in ([1] * 2, [80, 70]):
        a = _case(lens, 16, H, D, D, "bf16", 8)
        x = _gpu(a, "bf16", False, spare=0)
        at = torch.tensor([pool - 1, pool - 30], dtype=torch.int32, device="cuda")
        S[at.long()] = torch.from_numpy(a["state"]).float().cuda()
        S[pool - 1 - 2048] = 7.0  # where a 32-bit address would end up
        offs = None if lens[0] == 1 else torch.from_numpy(a["offs"]).cuda()
        tb.delta_rule(**x, offs=offs, state=S, state_out=S, slots=at)
        _near("pool", S[at.long()], ol.delta_rule(**a)["end"], tolerance(D, lens))
        assert (S[pool - 1 - 2048] == 7.0).all()
    parent = torch.tensor([[1, 1, 1, 0]], dtype=torch.int32, device="cuda")
    slots = torch.tensor([[0, pool - 1, 3, pool - 2]], dtype=torch.int32, device="cuda")
    kept = S[pool - 1].clone()
    new = tb.beam_reorder(parent, slots, [S])
    assert new.tolist() == [[pool - 1, 3, pool - 2, 0]]
    assert all(torch.equal(S[i], kept) for i in (pool - 1, 3, pool - 2))


def test_rows_past_32_bits():
    """Rows of activations and logits whose first entry is beyond 2^31 entries."""
    tb = _tb()
    x = torch.zeros((1 << 20) + 3, 2100, dtype=torch.bfloat16, device="cuda")
    x[-1] = torch.randn(2100, device="cuda").bfloat16()
    y = tb.layer_norm(x)
    assert torch.equal(y[-1:], tb.layer_norm(x[-1:])) and not y[:-1].any()
    del y
    g = tb.layer_norm_backward(x, None, x)
    one = tb.layer_norm_backward(x[-1:], None, x[-1:])
    assert torch.equal(g["dx"][-1:], one["dx"])
    # (rows of zeros add nothing to the sums)
    assert torch.equal(g["db"], x[-1].float()) and torch.equal(g["dw"], one["dw"])
    del g
    x = x.view(-1)[:16500 * 131072].view(16500, 131072)
    x.zero_()
    x[-2, 5] = x[-1, 7] = 9.0
    s = torch.zeros(16500 // 4, 4, device="cuda")
    r = tb.beam_select(x, s, 3)
    want = osr.beam_select(x[-4:].double().cpu().numpy(), np.zeros((1, 4)), 3)
    assert np.array_equal(r["parent"][-1].cpu().numpy(), want["parent"][0] + 16496)
    assert np.array_equal(r["token"][-1].cpu().numpy(), want["token"][0])


def test_gradients_of_empty_and_single_sequences():
    """Sequences of no tokens pass their state's gradient on; nothing else is touched."""
    tb, H, D = _tb(), 2, 16
    a = _case([0, 0, 1, 0], 1, H, D, D, "f32", 11)
    x, offs = _gpu(a, "f32", False, spare=0), torch.from_numpy(a["offs"]).cuda()
    S, dend = torch.from_numpy(a["state"]).float().cuda(), torch.randn(4, H, D, D, device="cuda")
    do = torch.randn(1, H, D, device="cuda")
    g = tb.delta_rule_backward(**x, do=do, offs=offs, state=S, state_grad=dend)
    assert torch.equal(g["dstate"][[0, 1, 3]], dend[[0, 1, 3]])
    r = ol.delta_rule_backward(do=do.double().cpu().numpy(), dend=dend.double().cpu().numpy(), **a)
    for k in GRADS:
        _near(k, g[k], r[k], tolerance(D, [1]))
    end = torch.full_like(S, 7.0)
    tb.delta_rule(**x, offs=offs, state=S, state_out=end)
    assert torch.equal(end[[0, 1, 3]], S[[0, 1, 3]])


def test_two_calls_at_once():
    """Calls on two streams with workspaces of their own give what they give alone."""
    tb, lens, H, D = _tb(), [130, 70], 4, 128
    cases = [_case(lens, 2, H, D, D, "bf16", 20 + i) for i in range(2)]
    xs = [_gpu(a, "bf16", False, spare=0) for a in cases]
    offs = torch.from_numpy(cases[0]["offs"]).cuda()
    do = torch.randn(200, H, D, device="cuda").bfloat16()
    alone = [tb.delta_rule_backward(**x, do=do, offs=offs) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(3):
        both = [tb.delta_rule_backward(**x, do=do, offs=offs, stream=s) for x, s in zip(xs, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(b[k], r[k]) for b, r in zip(both, alone) for k in ("dq", "dk", "dv", "dg", "dbeta"))
