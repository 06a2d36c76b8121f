"""What layer norm, the gated delta rule and beam search refuse, on the host, before any device work: in
the C entry points (pointers below are never dereferenced) and in the binding."""
import ctypes

import pytest
import torch

from paper_2604_12891_amd import binding as tb

FAKE = 1 << 20
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return tb.lib()


def _call(f, ok, **kw):
    assert not set(kw) - set(ok)
    return f(*{**ok, **kw}.values())


# ------------------------------------------------------------------ layer norm

NORM_BAD = [(dict(dtype=2), -1), (dict(rows=-1), -1), (dict(C=0), -1), (dict(C=16385), -2), (dict(rows=(1 << 30) + 1), -2),
            (dict(ldx=99), -1), (dict(eps=-1e-9), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
            (dict(x=None), -1), (dict(x=FAKE + 2), -1), (dict(dtype=1, x=FAKE + 1), -1)]


@pytest.mark.parametrize("kw,want", NORM_BAD)
def test_norm_refusals(lib, kw, want):
    ok = dict(dtype=0, rows=20, C=100, x=FAKE, ldx=1 << 20, w=FAKE, b=None, eps=1e-5, y=FAKE, ldy=1 << 20, stream=None)
    assert _call(lib.tcl_layer_norm, ok, **kw) == want
    ok = dict(dtype=0, rows=20, C=100, x=FAKE, ldx=1 << 20, w=FAKE, eps=1e-5, dy=FAKE, lddy=1 << 20, dx=FAKE, lddx=1 << 20,
              dw=FAKE, db=FAKE, ws=FAKE, n=BIG, stream=None)
    assert _call(lib.tcl_layer_norm_backward, ok, **kw) == want


def test_norm_call_refusals(lib):
    ok = dict(dtype=0, rows=20, C=100, x=FAKE, ldx=100, w=FAKE, b=None, eps=1e-5, y=FAKE, ldy=100, stream=None)
    for kw in (dict(y=None), dict(y=FAKE + 2), dict(ldy=99)):
        assert _call(lib.tcl_layer_norm, ok, **kw) == -1
    assert _call(lib.tcl_layer_norm, ok, rows=0, x=None, y=None) == 0
    need = lib.tcl_layer_norm_workspace_bytes(0, 20, 100)
    assert need > 0
    for bad in ((2, 20, 100), (0, 0, 100), (0, -1, 100), (0, 20, 0), (0, 20, 16385)):
        assert lib.tcl_layer_norm_workspace_bytes(*bad) == 0
    ok = dict(dtype=0, rows=20, C=100, x=FAKE, ldx=100, w=None, eps=1e-5, dy=FAKE, lddy=100, dx=FAKE, lddx=100, dw=FAKE,
              db=None, ws=FAKE, n=need, stream=None)
    for kw, want in ((dict(dy=None), -1), (dict(dx=None), -1), (dict(dw=None), -1), (dict(dy=FAKE + 1), -1),
                     (dict(dx=FAKE + 2), -1), (dict(lddy=99), -1), (dict(lddx=99), -1), (dict(ws=None), -1),
                     (dict(ws=FAKE + 16), -1), (dict(n=need - 1), -3)):
        assert _call(lib.tcl_layer_norm_backward, ok, **kw) == want


# ------------------------------------------------------------------ gated delta rule

def _delta(**kw):
    a = dict(dtype=0, n_seq=4, rows=200, Hk=2, H=4, Dk=64, Dv=32, scale=0.125, d_offs=FAKE, d_q=FAKE, ldq=128, d_k=FAKE,
             ldk=128, d_v=FAKE, ldv=128, d_g=FAKE, ldg=4, d_beta=FAKE, ldbeta=4, d_state=None)
    assert not set(kw) - set(a)
    return tb.DeltaRuleArgs(*{**a, **kw}.values())


def _grads(**kw):
    g = dict(d_dq=FAKE, lddq=1 << 20, d_dk=FAKE, lddk=1 << 20, d_dv=FAKE, lddv=1 << 20, d_dg=FAKE, lddg=1 << 20, d_dbeta=FAKE,
             lddbeta=1 << 20, d_dstate=None)
    return tb.DeltaRuleGrads(*{**g, **kw}.values())


DELTA_BAD = [(dict(dtype=2), -1), (dict(n_seq=-1), -1), (dict(rows=-1), -1), (dict(d_offs=None), -1), (dict(Hk=0), -2),
             (dict(Hk=3), -2), (dict(H=1), -2), (dict(Hk=1, H=1025), -2), (dict(Dk=4), -2), (dict(Dk=65), -2),
             (dict(Dk=136), -2), (dict(Dv=0), -2), (dict(Dv=264), -2), (dict(Dv=12), -2), (dict(rows=(1 << 26) + 1), -2),
             (dict(n_seq=1 << 18), -2), (dict(ldq=127), -1), (dict(ldk=127), -1), (dict(ldv=127), -1), (dict(ldg=3), -1),
             (dict(ldbeta=3), -1), (dict(d_q=None), -1), (dict(d_k=None), -1), (dict(d_v=None), -1), (dict(d_g=None), -1),
             (dict(d_beta=None), -1), (dict(d_q=FAKE + 2), -1), (dict(dtype=1, d_v=FAKE + 1), -1),
             (dict(d_state=FAKE + 8), -1)]


@pytest.mark.parametrize("kw,want", DELTA_BAD)
def test_delta_refusals(lib, kw, want):
    a = _delta(**kw)
    assert lib.tcl_delta_rule(ctypes.byref(a), None, 1 << 20, None, FAKE, 1 << 20, FAKE, BIG, None) == want
    g = _grads()
    assert lib.tcl_delta_rule_backward(ctypes.byref(a), FAKE, 1 << 20, None, ctypes.byref(g), FAKE, BIG, None) == want


def test_delta_call_refusals(lib):
    sizes = (0, 4, 200, 2, 4, 64, 32)
    need = lib.tcl_delta_rule_workspace_bytes(*sizes)
    assert need > 0 and lib.tcl_delta_rule_workspace_bytes(0, 0, 0, 2, 4, 64, 32) == 0
    for i, bad in ((0, 2), (1, -1), (2, -1), (3, 3), (4, 0), (5, 12), (6, 7)):
        assert lib.tcl_delta_rule_workspace_bytes(*sizes[:i], bad, *sizes[i + 1:]) == 0
        assert lib.tcl_delta_rule_backward_workspace_bytes(*sizes[:i], bad, *sizes[i + 1:]) == 0
    a = _delta(d_state=FAKE)
    ok = dict(a=ctypes.byref(a), slots=None, n_slots=4, so=None, o=FAKE, ldo=128, ws=FAKE, n=need, stream=None)
    for kw, want in ((dict(a=None), -1), (dict(n_slots=3), -1), (dict(n_slots=-1, slots=FAKE), -1), (dict(o=None), -1),
                     (dict(o=FAKE + 2), -1), (dict(ldo=127), -1), (dict(so=FAKE + 4), -1), (dict(ws=None), -1),
                     (dict(ws=FAKE + 8), -1), (dict(n=need - 1), -3)):
        assert _call(lib.tcl_delta_rule, ok, **kw) == want
    none = _delta(n_seq=0, rows=0)
    assert _call(lib.tcl_delta_rule, ok, a=ctypes.byref(none), o=None) == 0  # nothing to do
    need = lib.tcl_delta_rule_backward_workspace_bytes(*sizes)
    g = _grads()
    ok = dict(a=ctypes.byref(a), do=FAKE, lddo=128, dso=None, g=ctypes.byref(g), ws=FAKE, n=need, stream=None)
    for kw, want in ((dict(a=None), -1), (dict(a=ctypes.byref(none)), -1), (dict(g=None), -1), (dict(do=None), -1),
                     (dict(do=FAKE + 1), -1), (dict(lddo=127), -1), (dict(dso=FAKE + 4), -1), (dict(ws=None), -1),
                     (dict(ws=FAKE + 128), -1), (dict(n=need - 1), -3)):
        assert _call(lib.tcl_delta_rule_backward, ok, **kw) == want
    for kw in (dict(d_dq=None), dict(d_dk=None), dict(d_dv=None), dict(d_dg=None), dict(d_dbeta=None), dict(lddq=127),
               dict(lddk=127), dict(lddv=127), dict(lddg=3), dict(lddbeta=3), dict(d_dstate=FAKE + 8), dict(d_dk=FAKE + 2)):
        assert _call(lib.tcl_delta_rule_backward, ok, g=ctypes.byref(_grads(**kw))) == -1, kw


def test_delta_limits(lib):
    """Leading dimensions whose chunk would not be addressed in 31 bits, and launches of 2^32 threads, are refused; the
    largest that are not come to the next check."""
    top = 1 << 22
    ok = dict(a=None, slots=None, n_slots=1 << 20, so=None, o=None, ldo=128, ws=FAKE, n=BIG, stream=None)
    call = lambda ldo=128, **kw: _call(lib.tcl_delta_rule, ok, a=ctypes.byref(_delta(**kw)), ldo=ldo)
    for name in ("ldq", "ldk", "ldv"):
        assert call(**{name: top}) == -1  # (no o)
        assert call(**{name: top + 1}) == -2
    assert call(ldo=top) == -1 and call(ldo=top + 1) == -2
    # a token of each sequence: 2^22 heads of sequences; packed: 2^19; gradients: 2^19 for both
    token = dict(rows=1 << 18, n_seq=1 << 18, d_offs=None, Hk=1, ldg=16, ldbeta=16, ldv=512)
    assert call(ldo=512, H=15, **token) == -1
    assert call(ldo=512, H=16, **token) == -2
    packed = dict(n_seq=1 << 17, Hk=1)
    assert call(H=3, **packed) == -1 and call(H=4, **packed) == -2
    grads = dict(a=None, do=None, lddo=512, dso=None, g=ctypes.byref(_grads()), ws=FAKE, n=BIG, stream=None)
    back = lambda g=None, lddo=512, **kw: _call(lib.tcl_delta_rule_backward, grads, a=ctypes.byref(_delta(**kw)), lddo=lddo,
                                                g=ctypes.byref(_grads(**(g or {}))))
    token.update(rows=1 << 17, n_seq=1 << 17)
    assert back(H=3, **token) == -1  # (no dO)
    assert back(lddo=top) == -1 and back(lddo=top + 1) == -2
    for name in ("lddq", "lddk", "lddv"):
        assert back({name: top}) == -1 and back({name: top + 1}) == -2
    grads["do"] = FAKE
    assert back(H=4, **token) == -2


def test_delta_layouts():
    """The structures' bytes as the binding packs them are the structures."""
    v = list(range(1, 20))
    packed = tb._PACK_DELTA.pack(*v[:7], 0.5, *v[7:])
    a = tb.DeltaRuleArgs.from_buffer_copy(packed)
    assert ctypes.sizeof(a) == len(packed)
    assert [getattr(a, n) for n, _ in a._fields_] == v[:7] + [0.5] + v[7:]
    g = tb.DeltaRuleGrads.from_buffer_copy(tb._PACK_DELTA_GRADS.pack(*v[:11]))
    assert [getattr(g, n) for n, _ in g._fields_] == v[:11]


# ------------------------------------------------------------------ beam search

SELECT = dict(dtype=0, G=3, W=4, V=100, x=FAKE, ld=100, T=1.0, score=FAKE, ended=None, K=8, parent=FAKE, token=FAKE,
              out=2 * FAKE, ws=FAKE, n=BIG, stream=None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=2), -1), (dict(G=-1), -1), (dict(W=0), -1), (dict(W=65), -2), (dict(K=0), -2), (dict(K=65), -2),
    (dict(G=1 << 20), -2), (dict(V=0), -1), (dict(V=(1 << 30) + 1, ld=BIG), -2), (dict(ld=99), -1), (dict(T=0.0), -1),
    (dict(T=float("nan")), -1), (dict(x=None), -1), (dict(x=FAKE + 2), -1), (dict(score=None), -1), (dict(parent=None), -1),
    (dict(token=None), -1), (dict(out=None), -1), (dict(out=FAKE), -1), (dict(ws=None), -1), (dict(ws=FAKE + 8), -1),
    (dict(n=10), -3), (dict(G=0, x=None, score=None, ws=None), 0)])
def test_select_refusals(lib, kw, want):
    assert _call(lib.tcl_beam_select, SELECT, **kw) == want


def test_select_workspace(lib):
    assert lib.tcl_beam_select_workspace_bytes(3, 4, 100, 8) > 0
    for bad in ((0, 4, 100, 8), (-1, 4, 100, 8), (3, 65, 100, 8), (3, 4, 0, 8), (3, 4, 100, 65), (1 << 20, 4, 100, 8)):
        assert lib.tcl_beam_select_workspace_bytes(*bad) == 0


def test_reorder_refusals(lib):
    pools = (tb.BeamPool * 2)((FAKE, 100), (FAKE, 7))
    ok = dict(G=3, W=4, parent=FAKE, slots=2 * FAKE, n_slots=12, out=3 * FAKE, n=2, pools=pools, stream=None)
    for kw, want in ((dict(G=-1), -1), (dict(W=0), -1), (dict(W=65), -2), (dict(G=1 << 20), -2), (dict(n_slots=-1), -1),
                     (dict(n=-1), -1), (dict(pools=None), -1), (dict(parent=None), -1), (dict(slots=None), -1),
                     (dict(out=None), -1), (dict(out=2 * FAKE), -1), (dict(out=2 * FAKE + 44), -1), (dict(out=FAKE - 44), -1),
                     (dict(pools=(tb.BeamPool * 2)((FAKE, 100), (FAKE, 0))), -2),
                     (dict(pools=(tb.BeamPool * 2)((FAKE, (1 << 31) + 1), (FAKE, 7))), -2),
                     (dict(pools=(tb.BeamPool * 2)((None, 100), (FAKE, 7))), -1),
                     (dict(G=0, parent=None, slots=None, out=None), 0)):
        assert _call(lib.tcl_beam_reorder, ok, **kw) == want, kw


# ------------------------------------------------------------------ the binding

def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        tb.layer_norm(x)
    with pytest.raises(ValueError):
        tb.layer_norm_backward(x, None, x)
    h = torch.zeros(4, 1, 8)
    with pytest.raises(ValueError):
        tb.delta_rule(h, h, h, torch.zeros(4, 1), torch.zeros(4, 1))
    with pytest.raises(ValueError):
        tb.delta_rule(x, x, x, x, x)
    with pytest.raises(ValueError):
        tb.beam_select(x, torch.zeros(1, 4))
    with pytest.raises(ValueError):
        tb.beam_reorder(torch.zeros(1, 4, dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int32), [])


def test_heads_of_rows():
    """[rows, heads, width] with contiguous rows and a leading dimension; anything else is refused."""
    t = torch.zeros(6, 2, 8)
    shape = t.shape
    assert tb._heads_ld("t", t, torch.float32, shape, t) == 16
    wide = torch.zeros(6, 40)[:, 3:19].unflatten(1, (2, 8))
    assert tb._heads_ld("t", wide, torch.float32, shape, t) == 40
    for bad in (torch.zeros(6, 8, 2).transpose(1, 2), torch.zeros(6, 3, 8)[:, ::2], torch.zeros(2, 6, 8).transpose(0, 1),
                torch.zeros(6, 2, 8, dtype=torch.bfloat16), torch.zeros(1, 2, 8).expand(6, 2, 8), torch.zeros(6, 2, 9)):
        with pytest.raises(ValueError):
            tb._heads_ld("t", bad, torch.float32, shape, t)
