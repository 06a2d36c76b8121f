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
