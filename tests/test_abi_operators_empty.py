"""Batches of no sequences: nothing to do forwards, refused backwards, as the header says."""
import ctypes

import pytest

from paper_2604_12891_amd import binding as tb

FAKE = 1 << 20


@pytest.mark.parametrize("offs", [FAKE, None])
def test_no_sequences(offs):
    lib = tb.lib()
    c = tb.SsmConvArgs(0, 0, 0, 64, 4, offs, None, 64, FAKE, None, None)
    assert lib.tcl_ssm_conv(ctypes.byref(c), None, 0, None, None, 64, None) == 0
    assert lib.tcl_ssm_conv_workspace_bytes(0, 0, 64, 4) == 0
    assert lib.tcl_ssm_conv_backward(ctypes.byref(c), None, 64, None, None, 64, FAKE, FAKE, None, FAKE, 1 << 30,
                                     None) == -1
    assert b"no sequences" in lib.tcl_last_error()
    s = tb.SsmScanArgs(0, 0, 0, 64, 16, 1, offs, None, 64, None, 64, None, 16, None, 16, None, 64, FAKE, None, None,
                       None)
    assert lib.tcl_ssm_scan(ctypes.byref(s), None, 0, None, None, 64, None, 0, None) == 0
    assert lib.tcl_ssm_scan_backward_workspace_bytes(0, 0, 64, 16, 1) == 0
    g = tb.SsmScanGrads(None, 64, None, 64, None, 16, None, 16, None, 64, FAKE, None, None, None)
    assert lib.tcl_ssm_scan_backward(ctypes.byref(s), None, 64, None, ctypes.byref(g), FAKE, 1 << 30, None) == -1
    assert b"no sequences" in lib.tcl_last_error()
