"""Outputs that overlap what their call reads, or each other, are refused on the host, before any device work (pointers below
are never dereferenced)."""
import pytest

from paper_2604_12891_amd import binding as tb

BASE, STEP, BIG = 1 << 30, 1 << 24, 1 << 40


@pytest.fixture(scope="module")
def lib():
    return tb.lib()


def _call(f, ok, **kw):
    assert not set(kw) - set(ok)
    return f(*{**ok, **kw}.values())


G, W, V, K = 6, 4, 100, 8
SELECT = dict(dtype=0, G=G, W=W, V=V, x=BASE, ld=V, T=1.0, score=BASE + STEP, ended=BASE + 2 * STEP, K=K, parent=BASE + 3 * STEP,
              token=BASE + 4 * STEP, out=BASE + 5 * STEP, ws=BASE + 6 * STEP, n=BIG, stream=None)
BYTES = dict(score=4 * G * W, ended=4 * G * W, parent=4 * G * K, token=4 * G * K, out=4 * G * K)


@pytest.mark.parametrize("out", ["parent", "token", "out"])
def test_select(lib, out):
    BYTES["ws"] = lib.tcl_beam_select_workspace_bytes(G, W, V, K)
    for other, n in BYTES.items():
        if other == out:
            continue
        # its first and its last bytes, and all around it
        for at in (0, n - 4, 4 - BYTES[out], -16):
            assert _call(lib.tcl_beam_select, SELECT, **{out: SELECT[other] + at}) == -1, (other, at)


# ------------------------------------------------------------------ layer norm

R, C = 20, 100  # fp32
NORM = dict(dtype=0, rows=R, C=C, x=BASE, ldx=C, w=BASE + STEP, b=BASE + 2 * STEP, eps=1e-5, y=BASE + 3 * STEP, ldy=C, stream=None)


@pytest.mark.parametrize("other,n", [("x", 4 * R * C), ("w", 4 * C), ("b", 4 * C)])
def test_norm(lib, other, n):
    for at in (0, n - 4, 4 - 4 * R * C):
        assert _call(lib.tcl_layer_norm, NORM, y=NORM[other] + at) == -1


def test_norm_of_strided_rows(lib):
    """One leading dimension: columns that meet in a row or in the next one; two: rows that meet somewhere; only the last
    rows; every other row."""
    x = NORM["x"]
    for ldx, ldy, at in ((300, 300, 99), (300, 300, 201), (300, 300, -99), (300, 300, 19 * 300 + 99), (300, 300, -19 * 300),
                         (300, 200, 100), (300, 700, 150), (300, 701, 150), (250, 500, 99), (500, 250, 1), (101, 103, 2000), (300, 200, -50),
                         (100, 1 << 30, 100), (1 << 30, 100, (1 << 30) - 1)):
        assert _call(lib.tcl_layer_norm, NORM, ldx=ldx, ldy=ldy, y=x + 4 * at) == -1, (ldx, ldy, at)
        assert _call(lib.tcl_layer_norm, NORM, ldx=ldy, ldy=ldx, x=x + 4 * at, y=x) == -1, (ldx, ldy, at)


def test_norm_gradients(lib):
    ws = lib.tcl_layer_norm_workspace_bytes(0, R, C)
    ok = dict(dtype=0, rows=R, C=C, x=BASE, ldx=C, w=BASE + STEP, eps=1e-5, dy=BASE + 2 * STEP, lddy=C, dx=BASE + 3 * STEP, lddx=C,
              dw=BASE + 4 * STEP, db=BASE + 5 * STEP, ws=BASE + 6 * STEP, n=ws, stream=None)
    size = dict(x=4 * R * C, w=4 * C, dy=4 * R * C, dx=4 * R * C, dw=4 * C, db=4 * C, ws=ws)
    for out, others in (("dx", ("x", "w", "dy", "dw", "db", "ws")), ("dw", ("dx", "db", "ws")), ("db", ("dx", "dw", "ws"))):
        for other in others:
            for at in (0, size[other] - 4, 4 - size[out]):
                assert _call(lib.tcl_layer_norm_backward, ok, **{out: ok[other] + at}) == -1, (out, other, at)
