"""What the sequence and logit operators refuse, on the host, before any device
work: in the C entry points (pointers below are never dereferenced) and in
the binding."""
import ctypes

import pytest
import torch

from paper_2604_12891_amd import binding as tb

FAKE = 1 << 20


@pytest.fixture(scope="module")
def lib():
    return tb.lib()


def _conv(**kw):
    a = dict(dtype=0, n_seq=4, rows=20, E=64, K=4, d_offs=FAKE, d_x=FAKE, ldx=64, d_w=FAKE, d_b=FAKE, d_state=None)
    a.update(kw)
    return tb.SsmConvArgs(**a)


def _scan(**kw):
    a = dict(dtype=0, n_seq=4, rows=20, E=64, N=16, L=25, d_offs=FAKE, d_u=FAKE, ldu=64, d_dt=FAKE, lddt=64, d_B=FAKE,
             ldB=16, d_C=FAKE, ldC=16, d_z=FAKE, ldz=64, d_A_log=FAKE, d_D=None, d_b_dt=None, d_state=None)
    a.update(kw)
    return tb.SsmScanArgs(**a)


SEQ_BAD = [(dict(dtype=2), -1), (dict(n_seq=-1), -1), (dict(rows=-1), -1), (dict(d_offs=None), -1),
           (dict(E=0), -2), (dict(E=65537), -2), (dict(rows=1 << 30, E=60000), -2)]


@pytest.mark.parametrize("kw,want", SEQ_BAD + [(dict(K=0), -2), (dict(K=5), -2), (dict(ldx=63), -1),
                                               (dict(d_x=None), -1), (dict(d_w=None), -1)])
def test_conv_refusals(lib, kw, want):
    kw = dict(dict(ldx=1 << 20) if "E" in kw and kw["E"] > 64 else {}, **kw)
    a = _conv(**kw)
    assert lib.tcl_ssm_conv(ctypes.byref(a), None, 4, None, FAKE, 1 << 20, None) == want
    assert lib.tcl_ssm_conv_backward(ctypes.byref(a), FAKE, 1 << 20, None, FAKE, 1 << 20, FAKE, FAKE, None, FAKE,
                                     1 << 40, None) == want


def test_conv_call_refusals(lib):
    a = _conv(d_state=FAKE)
    ok = dict(a=ctypes.byref(a), slots=None, n_slots=4, so=None, u=FAKE, ldu=64, stream=None)

    def fwd(**kw):
        return lib.tcl_ssm_conv(*dict(ok, **kw).values())

    assert fwd(a=None) == -1
    assert fwd(n_slots=3) == -1       # no slots: a state per sequence
    assert fwd(n_slots=-1, slots=FAKE) == -1
    assert fwd(u=None) == -1
    assert fwd(ldu=63) == -1
    need = lib.tcl_ssm_conv_workspace_bytes(4, 20, 64, 4)
    assert need > 0 and lib.tcl_ssm_conv_workspace_bytes(4, 20, 64, 5) == 0
    okb = dict(a=ctypes.byref(a), du=FAKE, lddu=64, dso=None, dx=FAKE, lddx=64, dw=FAKE, db=None, ds=None, ws=FAKE,
               n=need, stream=None)

    def bwd(**kw):
        return lib.tcl_ssm_conv_backward(*dict(okb, **kw).values())

    assert bwd(n=need - 1) == -3
    assert b"needs" in lib.tcl_last_error()
    assert bwd(ws=None) == -1
    assert bwd(ws=FAKE + 16) == -1
    assert bwd(dw=None) == -1
    assert bwd(lddx=1) == -1
    none = _conv(n_seq=0, rows=0)
    assert bwd(a=ctypes.byref(none)) == -1
    assert lib.tcl_ssm_conv(ctypes.byref(none), None, 0, None, None, 64, None) == 0  # nothing to do


@pytest.mark.parametrize("kw,want", SEQ_BAD + [
    (dict(N=4), -2), (dict(N=32), -2), (dict(L=0), -1), (dict(ldu=63), -1), (dict(lddt=1), -1), (dict(ldB=15), -1),
    (dict(ldC=0), -1), (dict(ldz=63), -1), (dict(d_u=None), -1), (dict(d_dt=None), -1), (dict(d_B=None), -1),
    (dict(d_C=None), -1), (dict(d_A_log=None), -1), (dict(d_A_log=FAKE + 4), -1), (dict(d_state=FAKE + 8), -1)])
def test_scan_refusals(lib, kw, want):
    if kw.get("E", 0) > 64:
        kw = dict(kw, ldu=1 << 20, lddt=1 << 20, ldz=1 << 20)
    a = _scan(**kw)
    assert lib.tcl_ssm_scan(ctypes.byref(a), None, 4, None, FAKE, 1 << 20, FAKE, 1 << 40, None) == want
    g = tb.SsmScanGrads(*[FAKE, 1 << 20] * 5, FAKE, FAKE, FAKE, None)
    assert lib.tcl_ssm_scan_backward(ctypes.byref(a), FAKE, 1 << 20, None, ctypes.byref(g), FAKE, 1 << 40,
                                     None) == want


def test_scan_call_refusals(lib):
    a = _scan(n_seq=1, rows=5000, L=5000, d_state=FAKE)
    need = lib.tcl_ssm_scan_workspace_bytes(1, 5000, 64, 16, 5000)
    assert need > 0 and lib.tcl_ssm_scan_workspace_bytes(4096, 60000, 512, 16, 25) == 0
    ok = dict(a=ctypes.byref(a), slots=None, n_slots=1, so=None, y=FAKE, ldy=64, ws=FAKE, n=need, stream=None)

    def fwd(**kw):
        return lib.tcl_ssm_scan(*dict(ok, **kw).values())

    assert fwd(a=None) == -1
    assert fwd(n=need - 1) == -3
    assert fwd(ws=None) == -1
    assert fwd(ws=FAKE + 8) == -1
    assert fwd(n_slots=0) == -1
    assert fwd(so=FAKE + 4) == -1
    assert fwd(y=None) == -1
    assert fwd(ldy=1) == -1
    need = lib.tcl_ssm_scan_backward_workspace_bytes(1, 5000, 64, 16, 5000)
    g = dict(d_du=FAKE, lddu=64, d_ddt=FAKE, ldddt=64, d_dB=FAKE, lddB=16, d_dC=FAKE, lddC=16, d_dz=FAKE, lddz=64,
             d_dA_log=FAKE, d_dD=None, d_db_dt=None, d_dstate=None)

    def bwd(n=need, ws=FAKE, **kw):
        gs = tb.SsmScanGrads(**dict(g, **kw))
        return lib.tcl_ssm_scan_backward(ctypes.byref(a), FAKE, 64, None, ctypes.byref(gs), ws, n, None)

    assert bwd(n=need - 1) == -3
    assert bwd(ws=None) == -1
    for k in ("d_du", "d_ddt", "d_dB", "d_dC", "d_dz", "d_dA_log"):
        assert bwd(**{k: None}) == -1, k
    for k in ("lddu", "ldddt", "lddB", "lddC", "lddz"):
        assert bwd(**{k: 7}) == -1, k
    assert lib.tcl_ssm_scan_backward(ctypes.byref(a), FAKE, 64, None, None, FAKE, need, None) == -1


def test_scan_backward_refuses_misaligned_state_gradients(lib):
    a = _scan(n_seq=2, rows=20, L=20, d_state=FAKE)
    for dend, dstate in ((FAKE + 4, None), (None, FAKE + 8)):
        g = tb.SsmScanGrads(*[FAKE, 64] * 5, FAKE, None, None, dstate)
        assert lib.tcl_ssm_scan_backward(ctypes.byref(a), FAKE, 64, dend, ctypes.byref(g), FAKE, 1 << 40, None) == -1
        assert b"aligned" in lib.tcl_last_error()


def test_more_rows_than_indices_hold(lib):
    for kw in (dict(rows=(1 << 30) + 1), dict(n_seq=(1 << 30) + 1)):
        a = _scan(E=1, ldu=1, lddt=1, ldz=1, **kw)
        assert lib.tcl_ssm_scan(ctypes.byref(a), None, 1 << 30, None, FAKE, 1, FAKE, 1 << 40, None) == -2
        c = _conv(E=1, ldx=1, **kw)
        assert lib.tcl_ssm_conv(ctypes.byref(c), None, 1 << 30, None, FAKE, 1, None) == -2


def test_logit_refusals(lib):
    ok = dict(dtype=0, n=4, V=5000, x=FAKE, ld=5000, offs=None, temp=1.0, tok=FAKE, K=8, lp=FAKE, en=FAKE, top=FAKE,
              tl=FAKE, ws=FAKE, bytes=1 << 40, stream=None)

    def lp(**kw):
        return lib.tcl_logprobs(*dict(ok, **kw).values())

    need = lib.tcl_logits_workspace_bytes(4, 5000, 8)
    assert need > 0 and lib.tcl_logits_workspace_bytes(4096, 5000, 8) == 0
    okd = dict(dtype=0, n=4, V=5000, x=FAKE, ld=5000, offs=None, temp=1.0, K=8, top=FAKE, val=FAKE, w=None, loss=FAKE,
               grad=FAKE + 4096, ldg=5000, ws=FAKE, bytes=1 << 40, stream=None)

    def di(**kw):
        return lib.tcl_distill_topk(*dict(okd, **kw).values())

    for f in (lp, di):
        for kw, want in [(dict(dtype=3), -1), (dict(n=-1), -1), (dict(V=0), -1), (dict(V=(1 << 30) + 1, ld=1 << 31), -2),
                         (dict(ld=4999), -1), (dict(temp=0.0), -1), (dict(temp=-1.0), -1),
                         (dict(temp=float("nan")), -1), (dict(temp=float("inf")), -1), (dict(temp=1e-42), -1),
                         (dict(x=None), -1), (dict(x=FAKE + 2), -1), (dict(ws=None), -1), (dict(ws=FAKE + 8), -1),
                         (dict(bytes=16), -3)]:
            assert f(**kw) == want, kw
        assert f(n=0, x=None) == 0
    assert lp(K=65) == -2
    assert lp(K=-1) == -2
    assert lp(tok=None) == -1
    assert lp(top=None) == -1
    assert di(K=0) == -2
    assert di(K=1025) == -2
    assert di(top=None) == -1
    assert di(val=None) == -1
    assert di(loss=None) == -1
    assert di(ldg=4999) == -1
    assert di(grad=FAKE, ldg=6000) == -1   # in place, another leading dimension
    assert di(grad=FAKE + 2) == -1


def test_binding_refuses_tensors_elsewhere():
    """The binding checks where its tensors are before it calls the library."""
    x, w = torch.zeros(3, 8), torch.zeros(8, 4)
    with pytest.raises(ValueError, match="current device"):
        tb.ssm_conv(x, w)
    with pytest.raises(ValueError, match="current device"):
        tb.ssm_scan(x, x, torch.zeros(8, 16), torch.zeros(3, 16), torch.zeros(3, 16))
    with pytest.raises(ValueError, match="current device"):
        tb.logprobs(x)
    with pytest.raises(ValueError, match="current device"):
        tb.distill_topk(x, torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, 2))


def test_binding_checks_tensors():
    x = torch.zeros(6, 8)
    tb._expect("a", None, torch.float32, (6, 8), x)
    tb._expect("a", x, torch.float32, (6, 8), x)
    tb._expect("a", torch.zeros(6, 20)[:, 3:11], torch.float32, (6, 8), x, rows=True)
    with pytest.raises(ValueError, match="a: "):
        tb._expect("a", x.bfloat16(), torch.float32, (6, 8), x)
    with pytest.raises(ValueError, match="a: "):
        tb._expect("a", x, torch.float32, (6, 9), x)
    with pytest.raises(ValueError, match="contiguous"):
        tb._expect("a", torch.zeros(6, 20)[:, 3:11], torch.float32, (6, 8), x)
    with pytest.raises(ValueError, match="contiguous"):
        tb._expect("a", torch.zeros(8, 6).t(), torch.float32, (6, 8), x, rows=True)
    with pytest.raises(ValueError, match="contiguous"):
        tb._expect("a", torch.zeros(1, 8).expand(6, 8), torch.float32, (6, 8), x, rows=True)
    with pytest.raises(ValueError, match="fp32 or bf16"):
        tb._dtype(x.half())
    assert tb._ld(torch.zeros(6, 20)[:, 3:11]) == 20 and tb._ld(torch.zeros(1, 8)) == 8
    pool = torch.zeros(5, 3, 8)
    assert tb._pools(pool, pool, None, 5, (3, 8), torch.float32, x) == 5
    with pytest.raises(ValueError, match="pools"):
        tb._pools(pool, pool[:4], None, 5, (3, 8), torch.float32, x)
    with pytest.raises(ValueError, match="slots"):
        tb._pools(pool, None, torch.zeros(4, dtype=torch.int32), 5, (3, 8), torch.float32, x)
    with pytest.raises(ValueError, match="state"):
        tb._pools(pool[0], None, None, 5, (3, 8), torch.float32, x)


def test_packed_arguments_have_the_structures_layout():
    for pack, struct in ((tb._PACK_CONV, tb.SsmConvArgs), (tb._PACK_SCAN, tb.SsmScanArgs),
                         (tb._PACK_GRADS, tb.SsmScanGrads)):
        assert pack.size == ctypes.sizeof(struct)
        values = list(range(1, len(struct._fields_) + 1))
        back = struct.from_buffer_copy(pack.pack(*values))
        assert [getattr(back, n) for n, _ in struct._fields_] == values


def test_sizes_beyond_a_launch_are_refused(lib):
    """What would need more threads than one launch has."""
    def conv(n, rows, E, offs):
        a = tb.SsmConvArgs(0, n, rows, E, 4, offs, FAKE, 1 << 20, FAKE, None, None)
        return lib.tcl_ssm_conv(ctypes.byref(a), None, n, None, FAKE, 1 << 20, None)

    def scan(n, rows, E, offs):
        a = tb.SsmScanArgs(0, n, rows, E, 16, 8, offs, FAKE, 1 << 20, FAKE, 1 << 20, FAKE, 16, FAKE, 16, None, 0, FAKE,
                           None, None, None)
        return lib.tcl_ssm_scan(ctypes.byref(a), None, n, None, FAKE, 1 << 20, FAKE, 1 << 40, None)

    for f in (conv, scan):
        assert f((1 << 18) + 1, (1 << 18) + 1, 4096, None) == -2
        assert f((1 << 24) + 1, (1 << 24) + 1, 1, None) == -2   # (64 channels at least)
        assert f(4, (1 << 22) + 1, 4096, FAKE) == -2
    for f, m in ((lib.tcl_logprobs, (FAKE, 4, FAKE, FAKE, FAKE, FAKE)),
                 (lib.tcl_distill_topk, (4, FAKE, FAKE, None, FAKE, None, 0))):
        args = dict(n=1 << 22, V=100, ld=100)
        assert f(0, args["n"], args["V"], FAKE, args["ld"], None, 1.0, *m, None, 0, None) == -2
        for temp in (1.1e30, 0.9e-30):
            assert f(0, 4, 100, FAKE, 100, None, temp, *m, None, 0, None) == -1
