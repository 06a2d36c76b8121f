"""Thin ctypes binding of libtcl (include/tcl.h): argument marshalling only.

Every step of the cost model runs in libtcl's HIP kernels; this module only
converts torch tensors to device pointers and the caller's current HIP
stream, and raises on a non-OK status. Loading fails loudly if the library
has not been built: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import Optional

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libtcl.so")
_lib = None

TCL_F32, TCL_BF16 = 0, 1
TCL_F32_MATMUL_SPLIT, TCL_F32_MATMUL_NATIVE, TCL_F32_MATMUL_SPLIT_BF16 = 0, 1, 2
F32_MATMUL = {"split": TCL_F32_MATMUL_SPLIT, "native": TCL_F32_MATMUL_NATIVE,
              "split_bf16": TCL_F32_MATMUL_SPLIT_BF16}
STATUS = {0: "TCL_OK", -1: "TCL_ERR_INVALID_ARG", -2: "TCL_ERR_UNSUPPORTED", -3: "TCL_ERR_WORKSPACE",
          -4: "TCL_ERR_OOM", -5: "TCL_ERR_HIP"}


class TclError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS.get(status, status)}: {msg}")
        self.status = status


class Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("F", "d_model", "d_inner", "d_state", "d_conv", "dt_rank", "n_layers", "head_hidden",
                 "final_norm")] + [("norm_eps", ctypes.c_float), ("dtype", ctypes.c_int32),
                                   ("f32_matmul", ctypes.c_int32), ("enc_hidden", ctypes.c_int32 * 2),
                                   ("dec_hidden2", ctypes.c_int32)]


class KDLoss(ctypes.Structure):
    """tcl_kd_loss: the Eq. (9) distillation objective."""
    _fields_ = [("beta", ctypes.c_float), ("phi", ctypes.c_float), ("sigma", ctypes.c_float),
                ("ewc_lambda", ctypes.c_float), ("d_fisher", ctypes.c_void_p), ("d_theta_prev", ctypes.c_void_p),
                ("d_phi", ctypes.c_void_p)]


class SsmConvArgs(ctypes.Structure):
    """tcl_ssm_conv_args."""
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "n_seq", "rows", "E", "K")] + [
        ("d_offs", ctypes.c_void_p), ("d_x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("d_w", ctypes.c_void_p),
        ("d_b", ctypes.c_void_p), ("d_state", ctypes.c_void_p)]


class SsmScanArgs(ctypes.Structure):
    """tcl_ssm_scan_args."""
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "n_seq", "rows", "E", "N", "L")] + [
        ("d_offs", ctypes.c_void_p), ("d_u", ctypes.c_void_p), ("ldu", ctypes.c_int64), ("d_dt", ctypes.c_void_p),
        ("lddt", ctypes.c_int64), ("d_B", ctypes.c_void_p), ("ldB", ctypes.c_int64), ("d_C", ctypes.c_void_p),
        ("ldC", ctypes.c_int64), ("d_z", ctypes.c_void_p), ("ldz", ctypes.c_int64), ("d_A_log", ctypes.c_void_p),
        ("d_D", ctypes.c_void_p), ("d_b_dt", ctypes.c_void_p), ("d_state", ctypes.c_void_p)]


class SsmScanGrads(ctypes.Structure):
    """tcl_ssm_scan_grads."""
    _fields_ = [("d_du", ctypes.c_void_p), ("lddu", ctypes.c_int64), ("d_ddt", ctypes.c_void_p),
                ("ldddt", ctypes.c_int64), ("d_dB", ctypes.c_void_p), ("lddB", ctypes.c_int64),
                ("d_dC", ctypes.c_void_p), ("lddC", ctypes.c_int64), ("d_dz", ctypes.c_void_p),
                ("lddz", ctypes.c_int64), ("d_dA_log", ctypes.c_void_p), ("d_dD", ctypes.c_void_p),
                ("d_db_dt", ctypes.c_void_p), ("d_dstate", ctypes.c_void_p)]


class DeltaRuleArgs(ctypes.Structure):
    """tcl_delta_rule_args."""
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "n_seq", "rows", "Hk", "H", "Dk", "Dv")] + [
        ("scale", ctypes.c_float), ("d_offs", ctypes.c_void_p), ("d_q", ctypes.c_void_p), ("ldq", ctypes.c_int64),
        ("d_k", ctypes.c_void_p), ("ldk", ctypes.c_int64), ("d_v", ctypes.c_void_p), ("ldv", ctypes.c_int64),
        ("d_g", ctypes.c_void_p), ("ldg", ctypes.c_int64), ("d_beta", ctypes.c_void_p), ("ldbeta", ctypes.c_int64),
        ("d_state", ctypes.c_void_p)]


class DeltaRuleGrads(ctypes.Structure):
    """tcl_delta_rule_grads."""
    _fields_ = [("d_dq", ctypes.c_void_p), ("lddq", ctypes.c_int64), ("d_dk", ctypes.c_void_p),
                ("lddk", ctypes.c_int64), ("d_dv", ctypes.c_void_p), ("lddv", ctypes.c_int64),
                ("d_dg", ctypes.c_void_p), ("lddg", ctypes.c_int64), ("d_dbeta", ctypes.c_void_p),
                ("lddbeta", ctypes.c_int64), ("d_dstate", ctypes.c_void_p)]


class BeamPool(ctypes.Structure):
    """tcl_beam_pool."""
    _fields_ = [("d_states", ctypes.c_void_p), ("bytes", ctypes.c_int64)]


# The same layouts as bytes: packing them takes a fraction of a ctypes structure's time, which
# a single token's call would notice.
_PACK_CONV = struct.Struct("@5iPPqPPP")
_PACK_SCAN = struct.Struct("@6iPPqPqPqPqPqPPPP")
_PACK_GRADS = struct.Struct("@PqPqPqPqPqPPPP")
_PACK_DELTA = struct.Struct("@7ifPPqPqPqPqPqP")
_PACK_DELTA_GRADS = struct.Struct("@PqPqPqPqPqP")

_vp, _i32, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
_i64, _f32 = ctypes.c_int64, ctypes.c_float
_SIGS = {
    "tcl_param_count": (_sz, [ctypes.POINTER(Config)]),
    "tcl_cost_model_create": (_i32, [ctypes.POINTER(Config), _vp, _sz, ctypes.POINTER(_vp)]),
    "tcl_cost_model_destroy": (_i32, [_vp]),
    "tcl_score_workspace_bytes": (_sz, [_vp, _i32, _i32]),
    "tcl_set_score_streams": (_i32, [_vp, _i32]),
    "tcl_score": (_i32, [_vp, _i32, _i32, _vp, _vp, _vp, _vp, _sz, _vp]),
    "tcl_score_noalloc_max_bytes": (_sz, []),
    "tcl_score_noalloc": (_i32, [_vp, _i32, _i32, _vp, _vp, _vp, _vp]),
    "tcl_get_params": (_i32, [_vp, _vp, _sz]),
    "tcl_set_params": (_i32, [_vp, _vp, _sz]),
    "tcl_last_error": (ctypes.c_char_p, []),
    "tcl_timing_enable": (_i32, [_vp, _i32]),
    "tcl_timing_count": (_i32, [_vp]),
    "tcl_timing_get": (_i32, [_vp, _i32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_double),
                              ctypes.POINTER(ctypes.c_int64)]),
    "tcl_timing_reset": (_i32, [_vp]),
    "tcl_trainer_create": (_i32, [_vp, _vp, ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_float,
                                  _i32, _i32, ctypes.POINTER(_vp)]),
    "tcl_trainer_destroy": (_i32, [_vp]),
    "tcl_distill_workspace_bytes": (_sz, [_vp, _i32, _i32]),
    "tcl_distill_step": (_i32, [_vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "tcl_trainer_get_grads": (_i32, [_vp, _vp, _sz]),
    "tcl_distill_step_kd": (_i32, [_vp, _i32, _i32, _vp, _vp, _vp, ctypes.POINTER(KDLoss), _vp, _vp, _sz, _vp]),
    "tcl_lambdarank_workspace_bytes": (_sz, [_i32]),
    "tcl_teacher_gate": (_i32, [_i32, _vp, _vp, _vp]),
    "tcl_test_distill_step_kd_ranked": (_i32, [_vp, _i32, _i32, _vp, _vp, _vp, ctypes.POINTER(KDLoss), _vp, _vp,
                                               _vp, _vp, _sz, _vp]),
    "tcl_topk": (_i32, [_i32, _vp, _vp, _i32, _vp, _vp]),
    "tcl_lateral_param_count": (_sz, [ctypes.POINTER(Config), _i32]),
    "tcl_lateral_create": (_i32, [_vp, _vp, _i32, _vp, _sz, ctypes.POINTER(_vp)]),
    "tcl_lateral_destroy": (_i32, [_vp]),
    "tcl_progressive_workspace_bytes": (_sz, [_vp, _i32, _i32]),
    "tcl_progressive_score": (_i32, [_vp, _i32, _i32, _vp, _vp, _vp, _vp, _sz, _vp]),
    "tcl_topk_score_workspace_bytes": (_sz, [_i32, _i32]),
    "tcl_topk_score": (_i32, [_i32, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _sz, _vp]),
    "tcl_rdu_workspace_bytes": (_sz, [_i32, _i32]),
    "tcl_rdu_select": (_i32, [_i32, _vp, _vp, _i32, _vp, _i32, _i32, _vp, _vp, _vp, _sz, _vp]),
    "tcl_lambdarank": (_i32, [_i32, _vp, _vp, ctypes.c_float, _vp, _vp, _vp, _sz, _vp]),
    "tcl_ssm_conv": (_i32, [_vp, _vp, _i32, _vp, _vp, _i64, _vp]),
    "tcl_ssm_conv_workspace_bytes": (_sz, [_i32] * 4),
    "tcl_ssm_conv_backward": (_i32, [_vp, _vp, _i64, _vp, _vp, _i64, _vp, _vp, _vp, _vp, _sz,
                                     _vp]),
    "tcl_ssm_scan_workspace_bytes": (_sz, [_i32] * 5),
    "tcl_ssm_scan": (_i32, [_vp, _vp, _i32, _vp, _vp, _i64, _vp, _sz, _vp]),
    "tcl_ssm_scan_backward_workspace_bytes": (_sz, [_i32] * 5),
    "tcl_ssm_scan_backward": (_i32, [_vp, _vp, _i64, _vp, _vp, _vp,
                                     _sz, _vp]),
    "tcl_logits_workspace_bytes": (_sz, [_i32] * 3),
    "tcl_logprobs": (_i32, [_i32, _i32, _i32, _vp, _i64, _vp, _f32, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _sz, _vp]),
    "tcl_distill_topk": (_i32, [_i32, _i32, _i32, _vp, _i64, _vp, _f32, _i32, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _sz,
                                _vp]),
    "tcl_delta_rule_workspace_bytes": (_sz, [_i32] * 7),
    "tcl_delta_rule": (_i32, [_vp, _vp, _i32, _vp, _vp, _i64, _vp, _sz, _vp]),
    "tcl_delta_rule_backward_workspace_bytes": (_sz, [_i32] * 7),
    "tcl_delta_rule_backward": (_i32, [_vp, _vp, _i64, _vp, _vp, _vp, _sz, _vp]),
    "tcl_layer_norm": (_i32, [_i32, _i32, _i32, _vp, _i64, _vp, _vp, _f32, _vp, _i64, _vp]),
    "tcl_layer_norm_workspace_bytes": (_sz, [_i32] * 3),
    "tcl_layer_norm_backward": (_i32, [_i32, _i32, _i32, _vp, _i64, _vp, _f32, _vp, _i64, _vp, _i64, _vp, _vp, _vp,
                                       _sz, _vp]),
    "tcl_beam_select_workspace_bytes": (_sz, [_i32] * 4),
    "tcl_beam_select": (_i32, [_i32, _i32, _i32, _i32, _vp, _i64, _f32, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _sz, _vp]),
    "tcl_beam_reorder": (_i32, [_i32, _i32, _vp, _vp, _i32, _vp, _i32, _vp, _vp]),
    "tcl_trainer_timing_enable": (_i32, [_vp, _i32]),
    "tcl_trainer_timing_count": (_i32, [_vp]),
    "tcl_trainer_timing_get": (_i32, [_vp, _i32, ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_double),
                                      ctypes.POINTER(ctypes.c_int64)]),
    "tcl_trainer_timing_reset": (_i32, [_vp]),
    "tcl_test_gemm_f32": (_i32, [_i32, _i32, _i32, _vp, _vp, _vp, _vp, _i32, _i32, _vp]),
    "tcl_test_gemm_split": (_i32, [_i32, _i32, _i32, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _i32, _i32, _vp, _vp]),
    "tcl_test_gemm_bf16": (_i32, [_i32, _i32, _i32, _i32, _i32, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _vp]),
    "tcl_test_conv_silu_f32": (_i32, [_i32, _i32, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp]),
    "tcl_test_xproj_conv_f32": (_i32, [_i32, _i32, _i32, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp,
                                       _vp, _vp]),
    "tcl_test_xproj_conv_bf16": (_i32, [_i32, _i32, _i32, _i32, _vp, _vp, _i32, _vp, _vp, _vp, _vp, _vp, _vp,
                                        _vp]),
    "tcl_test_offsets": (_i32, [_i32, _i32, _vp, _vp, _vp, _vp]),
    "tcl_test_scan_f32": (_i32, [_i32, _i32, _i32, _i32, _i32, _vp, _vp, _vp, _vp, _i32, _vp, _vp, _vp,
                                 _vp, _vp, _vp]),
}


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """Load libtcl.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with `python -m paper_2604_12891_amd.build`")
        L = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def check(status: int):
    if status != 0:
        raise TclError(status, lib().tcl_last_error().decode())


def make_config(F, d_model, d_inner, d_state, d_conv, dt_rank, n_layers, head_hidden,
                final_norm=1, norm_eps=1e-5, dtype="f32", f32_matmul="split", enc_hidden=(), dec_hidden2=0) -> Config:
    """f32_matmul ("split", "split_bf16" or "native") selects how an fp32 model runs its
    dense projections (tcl_f32_matmul); enc_hidden (up to two widths) and
    dec_hidden2 select the multi-layer encoder and three-layer decoder."""
    enc = list(enc_hidden) + [0] * (2 - len(enc_hidden))
    return Config(F, d_model, d_inner, d_state, d_conv, dt_rank, n_layers, head_hidden, final_norm,
                  norm_eps, TCL_BF16 if dtype == "bf16" else TCL_F32, F32_MATMUL[f32_matmul],
                  (ctypes.c_int32 * 2)(*enc), dec_hidden2)


def config_from_shape(shape, dtype="f32", f32_matmul="split") -> Config:
    return make_config(shape.F, shape.d_model, shape.d_inner, shape.d_state, shape.d_conv, shape.dt_rank,
                       shape.n_layers, shape.head_hidden, shape.final_norm, shape.norm_eps, dtype, f32_matmul,
                       tuple(getattr(shape, "enc_hidden", ())), getattr(shape, "dec_hidden2", 0))


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream=None) -> int:
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


class CostModel:
    """A device-resident cost model (tcl_cost_model_create / tcl_score)."""

    def __init__(self, cfg: Config, params: np.ndarray):
        L = lib()
        self.cfg = cfg
        self._n = L.tcl_param_count(ctypes.byref(cfg))
        blob = np.ascontiguousarray(params, dtype=np.float32)
        h = _vp()
        check(L.tcl_cost_model_create(ctypes.byref(cfg), blob.ctypes.data, blob.size, ctypes.byref(h)))
        self._h = h
        self._ws = None

    def close(self):
        if getattr(self, "_h", None):
            check(lib().tcl_cost_model_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def handle(self):
        return self._h

    def workspace_bytes(self, B: int, L: int) -> int:
        return lib().tcl_score_workspace_bytes(self._h, B, L)

    def workspace(self, B: int, L: int):
        import torch
        need = self.workspace_bytes(B, L)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self._ws

    def score(self, feats, lengths, out=None, workspace=None, stream=None):
        """feats [B,L,F] fp32 cuda, lengths [B] int32 cuda -> scores [B] fp32 cuda."""
        import torch
        B, L, _ = feats.shape
        if out is None:
            out = torch.empty(B, dtype=torch.float32, device=feats.device)
        ws = self.workspace(B, L) if workspace is None else workspace
        check(lib().tcl_score(self._h, B, L, feats.data_ptr(), lengths.data_ptr(), out.data_ptr(),
                              ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)))
        return out

    def score_noalloc(self, feats, lengths, out, stream=None):
        """tcl_score_noalloc: the scores into `out` with the library's own
        scratch buffer (no workspace, nothing allocated)."""
        B, L, _ = feats.shape
        check(lib().tcl_score_noalloc(self._h, B, L, feats.data_ptr(), lengths.data_ptr(), out.data_ptr(),
                                      _stream(stream)))
        return out

    def set_score_streams(self, n: int):
        """1: one pass per batch; 2 (default): batches of >= 2048 programs as
        two concurrent halves (tcl_set_score_streams)."""
        check(lib().tcl_set_score_streams(self._h, n))

    def timing(self, enable: bool):
        check(lib().tcl_timing_enable(self._h, int(enable)))

    def timing_reset(self):
        check(lib().tcl_timing_reset(self._h))

    def timing_report(self) -> dict:
        """{kernel name: (total_ms, launches)} of the launches timed so far."""
        L = lib()
        out = {}
        for i in range(L.tcl_timing_count(self._h)):
            name, ms, n = ctypes.c_char_p(), ctypes.c_double(), ctypes.c_int64()
            check(L.tcl_timing_get(self._h, i, ctypes.byref(name), ctypes.byref(ms), ctypes.byref(n)))
            out[name.value.decode()] = (ms.value, n.value)
        return out

    def get_params(self) -> np.ndarray:
        out = np.empty(self._n, dtype=np.float32)
        check(lib().tcl_get_params(self._h, out.ctypes.data, out.size))
        return out

    def set_params(self, params: np.ndarray):
        blob = np.ascontiguousarray(params, dtype=np.float32)
        check(lib().tcl_set_params(self._h, blob.ctypes.data, blob.size))


class Progressive:
    """A frozen KB and an active column joined by lateral adapters of width
    `adapter` (tcl_lateral_create / tcl_progressive_score). Keeps both models
    alive."""

    def __init__(self, kb: CostModel, ac: CostModel, adapter: int, params: np.ndarray):
        L = lib()
        self.kb, self.ac, self.adapter = kb, ac, adapter
        blob = np.ascontiguousarray(params, dtype=np.float32)
        h = _vp()
        check(L.tcl_lateral_create(kb.handle, ac.handle, adapter, blob.ctypes.data, blob.size, ctypes.byref(h)))
        self._h = h
        self._ws = None

    def close(self):
        if getattr(self, "_h", None):
            check(lib().tcl_lateral_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace(self, B: int, L: int):
        import torch
        need = lib().tcl_progressive_workspace_bytes(self._h, B, L)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self._ws

    def score(self, feats, lengths, out=None, workspace=None, stream=None):
        """The AC's scores with the KB read through Eq. (7): feats [B,L,F]
        fp32 cuda, lengths [B] int32 cuda -> [B] fp32 cuda."""
        import torch
        B, L, _ = feats.shape
        if out is None:
            out = torch.empty(B, dtype=torch.float32, device=feats.device)
        ws = self.workspace(B, L) if workspace is None else workspace
        check(lib().tcl_progressive_score(self._h, B, L, feats.data_ptr(), lengths.data_ptr(), out.data_ptr(),
                                          ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream)))
        return out


class Trainer:
    """Teacher -> student distillation (tcl_trainer_create / tcl_distill_step)."""

    def __init__(self, teacher: CostModel, student: CostModel, lr=1e-3, betas=(0.9, 0.999), eps=1e-8,
                 max_B=1024, max_L=25):
        h = _vp()
        check(lib().tcl_trainer_create(teacher.handle, student.handle, lr, betas[0], betas[1], eps, max_B,
                                       max_L, ctypes.byref(h)))
        self._h = h
        self._n = student._n
        self._keep = (teacher, student)  # the trainer must not outlive its models
        self._ws = None

    def close(self):
        if getattr(self, "_h", None):
            check(lib().tcl_trainer_destroy(self._h))
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_bytes(self, B: int, L: int) -> int:
        return lib().tcl_distill_workspace_bytes(self._h, B, L)

    def workspace(self, B: int, L: int):
        import torch
        need = self.workspace_bytes(B, L)
        if need == 0:
            raise ValueError(f"B={B}, L={L} exceed the trainer's bounds")
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self._ws

    def step(self, feats, lengths, labels, loss=None, workspace=None, stream=None):
        """One step; returns the device tensor [total, mse_teacher, mse_label]."""
        import torch
        B, L, _ = feats.shape
        if loss is None:
            loss = torch.empty(3, dtype=torch.float32, device=feats.device)
        ws = self.workspace(B, L) if workspace is None else workspace
        check(lib().tcl_distill_step(self._h, B, L, feats.data_ptr(), lengths.data_ptr(), labels.data_ptr(),
                                     loss.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(),
                                     _stream(stream)))
        return loss

    def step_kd(self, feats, lengths, labels, beta=0.5, phi=1.0, sigma=1.0, ewc_lambda=0.0, fisher=None,
                theta_prev=None, loss=None, workspace=None, stream=None, phi_dev=None, rank_keys=None,
                scores_out=None):
        """One step on the Eq. (9) objective (tcl_distill_step_kd); fisher and
        theta_prev are device fp32 tensors of the parameter count; phi_dev
        (a device fp32 tensor of one element, optional) replaces phi. Returns
        the device tensor [total, rank(s; teacher), rank(s; label), ewc].
        rank_keys / scores_out (device fp32 [B] / [2B]) go through the test
        entry tcl_test_distill_step_kd_ranked."""
        import torch
        B, L, _ = feats.shape
        if loss is None:
            loss = torch.empty(4, dtype=torch.float32, device=feats.device)
        ws = self.workspace(B, L) if workspace is None else workspace
        kd = KDLoss(beta, phi, sigma, ewc_lambda, _ptr(fisher), _ptr(theta_prev), _ptr(phi_dev))
        if rank_keys is None and scores_out is None:
            check(lib().tcl_distill_step_kd(self._h, B, L, feats.data_ptr(), lengths.data_ptr(),
                                            labels.data_ptr(), ctypes.byref(kd), loss.data_ptr(), ws.data_ptr(),
                                            ws.numel() * ws.element_size(), _stream(stream)))
        else:
            check(lib().tcl_test_distill_step_kd_ranked(
                self._h, B, L, feats.data_ptr(), lengths.data_ptr(), labels.data_ptr(), ctypes.byref(kd),
                _ptr(rank_keys), _ptr(scores_out), loss.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(),
                _stream(stream)))
        return loss

    def grads(self) -> np.ndarray:
        out = np.empty(self._n, dtype=np.float32)
        check(lib().tcl_trainer_get_grads(self._h, out.ctypes.data, out.size))
        return out

    def timing(self, enable: bool):
        check(lib().tcl_trainer_timing_enable(self._h, int(enable)))

    def timing_reset(self):
        check(lib().tcl_trainer_timing_reset(self._h))

    def timing_report(self) -> dict:
        L = lib()
        out = {}
        for i in range(L.tcl_trainer_timing_count(self._h)):
            name, ms, n = ctypes.c_char_p(), ctypes.c_double(), ctypes.c_int64()
            check(L.tcl_trainer_timing_get(self._h, i, ctypes.byref(name), ctypes.byref(ms), ctypes.byref(n)))
            out[name.value.decode()] = (ms.value, n.value)
        return out


def gemm_f32(A, W, bias=None, out=None, stream=None, tile=-1, epilogue=0):
    """epilogue 0: A W^T (+ bias); 1: out += A W^T; 2: rstd(A) * A W^T."""
    import torch
    M, K = A.shape
    N = W.shape[0]
    if out is None:
        out = torch.empty(M, N, dtype=torch.float32, device=A.device)
    check(lib().tcl_test_gemm_f32(M, N, K, A.data_ptr(), W.data_ptr(), _ptr(bias), out.data_ptr(), tile,
                                  epilogue, _stream(stream)))
    return out


def topk(scores, seg_offsets, K, stream=None):
    """Per-segment top-K (tcl_topk): scores fp32 [n], seg_offsets int32
    [n_seg + 1] (device); returns int32 [n_seg, K] global indices."""
    import torch
    n_seg = seg_offsets.numel() - 1
    out = torch.empty(n_seg, K, dtype=torch.int32, device=scores.device)
    check(lib().tcl_topk(n_seg, seg_offsets.data_ptr(), scores.data_ptr(), K, out.data_ptr(), _stream(stream)))
    return out


def topk_score(scores, latency, weight, seg_offsets, k, stream=None):
    """The Top-k score of Eq. (12) (tcl_topk_score): scores and latency fp32
    [n], weight fp32 [n_seg], seg_offsets int32 [n_seg + 1] (device).
    Returns a device fp64 tensor [3]: Top-k, numerator, denominator."""
    import torch
    n_seg = seg_offsets.numel() - 1
    out = torch.empty(3, dtype=torch.float64, device=scores.device)
    need = lib().tcl_topk_score_workspace_bytes(n_seg, k)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device=scores.device)
    check(lib().tcl_topk_score(n_seg, seg_offsets.data_ptr(), scores.data_ptr(), latency.data_ptr(),
                               weight.data_ptr(), k, out.data_ptr(), ws.data_ptr(), ws.numel(), _stream(stream)))
    return out


def rdu_select(scores, op, n_ops, initial, n_select, workspace=None, stream=None):
    """RDU selection (tcl_rdu_select): scores fp32 [N], op int32 [N], initial
    int32 [M0] (device). Returns (selected int32 [n_select], count int32 [1])."""
    import torch
    N = scores.numel()
    sel = torch.empty(max(n_select, 1), dtype=torch.int32, device=scores.device)
    cnt = torch.empty(1, dtype=torch.int32, device=scores.device)

    def call(ws):
        return lib().tcl_rdu_select(N, scores.data_ptr(), op.data_ptr(), n_ops, initial.data_ptr(), initial.numel(),
                                    n_select, sel.data_ptr(), cnt.data_ptr(), ws.data_ptr(),
                                    ws.numel() * ws.element_size(), _stream(stream))

    status = -3 if workspace is None else call(workspace)
    if status == -3:  # TCL_ERR_WORKSPACE: none, or one that is too small
        need = lib().tcl_rdu_workspace_bytes(N, n_ops)
        status = call(torch.empty(max(need, 256), dtype=torch.uint8, device=scores.device))
    check(status)
    return sel[:n_select], cnt


def lambdarank(scores, labels, sigma=1.0, grad=True, stream=None):
    """The LambdaRank loss of Eq. (6) (tcl_lambdarank) on device fp32 [B]
    tensors: returns (loss [1], grad [B] or None) as device tensors."""
    import torch
    B = scores.numel()
    loss = torch.empty(1, dtype=torch.float32, device=scores.device)
    g = torch.empty(B, dtype=torch.float32, device=scores.device) if grad else None
    nbytes = lib().tcl_lambdarank_workspace_bytes(B)
    ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=scores.device)
    check(lib().tcl_lambdarank(B, scores.data_ptr(), labels.data_ptr(), sigma, loss.data_ptr(), _ptr(g),
                               ws.data_ptr(), ws.numel(), _stream(stream)))
    return loss, g


# ---------------------------------------------------------------------------
# sequence and logit operators
# ---------------------------------------------------------------------------

def _dtype(t) -> int:
    import torch
    if t.dtype == torch.float32:
        return TCL_F32
    if t.dtype == torch.bfloat16:
        return TCL_BF16
    raise ValueError(f"fp32 or bf16 expected, not {t.dtype}")


def _expect(name, t, dtype, shape, like, rows=False):
    """t, when given, is a tensor of this type, shape and device; contiguous,
    or (rows) with unit stride within its rows."""
    if t is None:
        return
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name}: {dtype} {tuple(shape)} expected, not {t.dtype} {tuple(t.shape)}")
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")
    if t.is_contiguous():
        return
    if not rows or (shape[1] != 1 and t.stride(1) != 1) or (shape[0] != 1 and t.stride(0) < shape[1]):
        raise ValueError(f"{name}: {'rows' if rows else 'tensor'} not contiguous (strides {t.stride()})")


def _ld(t) -> int:
    """Leading dimension of a matrix of rows (one row, or none, has any)."""
    return t.shape[1] if t.is_contiguous() else t.stride(0)


def _row_ld(name, t, dtype, shape, like) -> int:
    """_expect's check of a matrix of rows, and its leading dimension."""
    if t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == like.get_device():
        return shape[1]
    _expect(name, t, dtype, shape, like, rows=True)
    return _ld(t)


def _adr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _stream_of(t) -> int:
    """The current stream of t's device (the current device); by torch's way to the bare handle where
    it has one, as a Stream object takes 1 us, a tenth of a token's call."""
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(t.get_device()) if raw else torch.cuda.current_stream(t.get_device()).cuda_stream


def _under(stream, call, *args, **kw):
    """call under another stream than the current one: what it allocates (results, a workspace)
    then belongs to that stream and is not given to others while its kernels run."""
    import torch
    with torch.cuda.stream(stream):
        return call(*args, **kw)


def _results(new, out, like):
    """new's tensors (name: shape, type, rows of a leading dimension or not), out's where it has them."""
    r = {}
    for name, spec in new.items():
        t = None if out is None else out.get(name)
        if spec is None:
            r[name] = None
        elif t is None:
            r[name] = like.new_empty(spec[0], dtype=spec[1])
        else:
            _expect(name, t, spec[1], spec[0], like, rows=spec[2])
            r[name] = t
    return r


def _on_device(t):
    import torch
    if not t.is_cuda or t.get_device() != torch.cuda.current_device():
        raise ValueError(f"tensors on {t.device}, which is not the current device")


def _workspace(workspace, like, size, *args):
    """The caller's workspace, or one of size(*args) bytes."""
    import torch
    if workspace is not None:
        if workspace.get_device() != like.get_device() or not workspace.is_contiguous():
            raise ValueError(f"workspace: contiguous memory on {like.device} expected")
        return workspace
    need = size(*args)
    return like.new_empty(need, dtype=torch.uint8) if need else None


def _ws_args(ws):
    return (None, 0) if ws is None else (ws.data_ptr(), ws.numel() * ws.element_size())


def _pools(state, state_out, slots, n_seq, shape, dtype, like):
    """Checks a call's state pools; returns the number of places in them."""
    import torch
    for name, t in (("state", state), ("state_out", state_out)):
        if t is not None:
            if t.dim() != 1 + len(shape):
                raise ValueError(f"{name}: {1 + len(shape)} dimensions expected, not {t.dim()}")
            _expect(name, t, dtype, (t.shape[0], *shape), like)
    if state is not None and state_out is not None and state.shape[0] != state_out.shape[0]:
        raise ValueError(f"pools of {state.shape[0]} and {state_out.shape[0]} states")
    _expect("slots", slots, torch.int32, (n_seq,), like)
    pool = state if state is not None else state_out
    return n_seq if pool is None else pool.shape[0]


def _sequences(x, offs):
    import torch
    if x.dim() != 2:
        raise ValueError(f"[rows, channels] expected, not {tuple(x.shape)}")
    _on_device(x)
    if offs is None:
        return x.shape[0]
    if offs.dim() != 1 or offs.numel() < 1:
        raise ValueError("offs: [n_seq + 1] expected")
    _expect("offs", offs, torch.int32, offs.shape, x)
    return offs.numel() - 1


def _conv_args(x, w, b, offs, n_seq, state):
    import torch
    rows, E = x.shape
    if w.dim() != 2:
        raise ValueError(f"w: [E, K] expected, not {tuple(w.shape)}")
    ldx = _row_ld("x", x, x.dtype, x.shape, x)
    _expect("w", w, torch.float32, (E, w.shape[1]), x)
    _expect("b", b, torch.float32, (E,), x)
    return _PACK_CONV.pack(_dtype(x), n_seq, rows, E, w.shape[1], _adr(offs), x.data_ptr(), ldx, w.data_ptr(),
                           _adr(b), _adr(state))


def ssm_conv(x, w, b=None, offs=None, state=None, state_out=None, slots=None, out=None, stream=None):
    """u = SiLU(b + causal depthwise conv(x; w)) with carried states
    (tcl_ssm_conv): x fp32 or bf16 [rows, E], w fp32 [E, K], b fp32 [E].
    offs int32 [n_seq + 1]: packed sequences; None: each row is one token of its own
    sequence. state / state_out [n, K-1, E] of x's type (may be the same tensor)
    with slots int32 [n_seq] into them. Returns u [rows, E]."""
    if stream is not None:
        return _under(stream, ssm_conv, x, w, b, offs, state, state_out, slots, out)
    import torch
    n_seq = _sequences(x, offs)
    n_slots = _pools(state, state_out, slots, n_seq, (w.shape[1] - 1, x.shape[1]), x.dtype, x)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    else:
        _expect("out", out, x.dtype, x.shape, x, rows=True)
    a = _conv_args(x, w, b, offs, n_seq, state)
    check(lib().tcl_ssm_conv(a, _ptr(slots), n_slots, _ptr(state_out), out.data_ptr(), _ld(out),
                             _stream_of(x)))
    return out


def ssm_conv_workspace(n_seq, rows, E, K):
    """A workspace for ssm_conv_backward, on the current device."""
    import torch
    return torch.empty(lib().tcl_ssm_conv_workspace_bytes(n_seq, rows, E, K), dtype=torch.uint8, device="cuda")


def ssm_conv_backward(x, w, b, du, offs=None, state=None, state_grad=None, workspace=None, out=None, stream=None):
    """Gradients of ssm_conv (tcl_ssm_conv_backward) from du [rows, E] and, for carried
    states [n_seq, K-1, E], the gradient state_grad of the end states. Returns a
    dict of dx, dw, db and dstate (None without a state); out: tensors of those names to write to.
    Rows of dx that no sequence owns are left as they are (in a new tensor: undefined). A batch
    of no sequences at all is refused."""
    if stream is not None:
        return _under(stream, ssm_conv_backward, x, w, b, du, offs, state, state_grad, workspace, out)
    import torch
    n_seq = _sequences(x, offs)
    K = w.shape[1]
    for name, t in (("state", state), ("state_grad", state_grad)):
        _expect(name, t, x.dtype, (n_seq, K - 1, x.shape[1]), x)
    _expect("du", du, x.dtype, x.shape, x, rows=True)
    a = _conv_args(x, w, b, offs, n_seq, state)
    r = _results(dict(dx=(x.shape, x.dtype, True), dw=(w.shape, w.dtype, False), db=(x.shape[1:], w.dtype, False),
                      dstate=None if state is None else (state.shape, x.dtype, False)), out, x)
    ws = _workspace(workspace, x, lib().tcl_ssm_conv_workspace_bytes, n_seq, *x.shape, K)
    check(lib().tcl_ssm_conv_backward(a, du.data_ptr(), _ld(du), _ptr(state_grad), r["dx"].data_ptr(),
                                      _ld(r["dx"]), r["dw"].data_ptr(), r["db"].data_ptr(), _ptr(r["dstate"]),
                                      *_ws_args(ws), _stream_of(x)))
    return r


def _scan_args(u, dt, A_log, B, C, D, z, b_dt, offs, n_seq, L, state):
    """(L, the packed tcl_ssm_scan_args)"""
    import torch
    rows, E = u.shape
    if A_log.dim() != 2:
        raise ValueError(f"A_log: [E, N] expected, not {tuple(A_log.shape)}")
    N = A_log.shape[1]
    act, bc = u.shape, (rows, N)
    ldu, lddt = _row_ld("u", u, u.dtype, act, u), _row_ld("dt", dt, u.dtype, act, u)
    ldB, ldC = _row_ld("B", B, u.dtype, bc, u), _row_ld("C", C, u.dtype, bc, u)
    ldz = 0 if z is None else _row_ld("z", z, u.dtype, act, u)
    _expect("A_log", A_log, torch.float32, (E, N), u)
    _expect("D", D, torch.float32, (E,), u)
    _expect("b_dt", b_dt, torch.float32, (E,), u)
    if L is None:
        L = max(rows, 1) if offs is not None else 1
    return L, _PACK_SCAN.pack(_dtype(u), n_seq, rows, E, N, L, _adr(offs), u.data_ptr(), ldu, dt.data_ptr(), lddt,
                              B.data_ptr(), ldB, C.data_ptr(), ldC, _adr(z), ldz, A_log.data_ptr(), _adr(D),
                              _adr(b_dt), _adr(state))


def ssm_scan_workspace(n_seq, rows, E, N, L, backward=False):
    """A workspace for ssm_scan (or ssm_scan_backward) with these sizes, on the
    current device."""
    import torch
    f = lib().tcl_ssm_scan_backward_workspace_bytes if backward else lib().tcl_ssm_scan_workspace_bytes
    return torch.empty(f(n_seq, rows, E, N, L), dtype=torch.uint8, device="cuda")


def ssm_scan(u, dt, A_log, B, C, D=None, z=None, b_dt=None, offs=None, L=None, state=None, state_out=None, slots=None,
             out=None, workspace=None, stream=None):
    """The selective scan with carried states (tcl_ssm_scan): u, dt, z [rows, E]
    and B, C [rows, N] fp32 or bf16, A_log [E, N], D, b_dt [E] and the states
    [n, E, N] fp32. offs, slots as for ssm_conv; L bounds the sequences' lengths (None:
    rows). Returns y [rows, E]."""
    if stream is not None:
        return _under(stream, ssm_scan, u, dt, A_log, B, C, D, z, b_dt, offs, L, state, state_out, slots, out, workspace)
    import torch
    n_seq = _sequences(u, offs)
    n_slots = _pools(state, state_out, slots, n_seq, A_log.shape, torch.float32, u)
    L, a = _scan_args(u, dt, A_log, B, C, D, z, b_dt, offs, n_seq, L, state)
    if out is None:
        out = torch.empty(u.shape, dtype=u.dtype, device=u.device)
    else:
        _expect("out", out, u.dtype, u.shape, u, rows=True)
    ws = None if offs is None else _workspace(workspace, u, lib().tcl_ssm_scan_workspace_bytes, n_seq, *u.shape,
                                              A_log.shape[1], L)
    check(lib().tcl_ssm_scan(a, _ptr(slots), n_slots, _ptr(state_out), out.data_ptr(), _ld(out),
                             *_ws_args(ws), _stream_of(u)))
    return out


def ssm_scan_backward(u, dt, A_log, B, C, dy, D=None, z=None, b_dt=None, offs=None, L=None, state=None,
                      state_grad=None, workspace=None, out=None, stream=None):
    """Gradients of ssm_scan (tcl_ssm_scan_backward) from dy [rows, E] and, for carried
    states [n_seq, E, N], the gradient state_grad of the end states. Returns a dict of
    du, ddt, dB, dC, dz (None without z), dA_log, dD, db_dt and dstate (None without a
    state); out: tensors of those names to write to. Rows of the activations' gradients that no sequence
    owns are left as they are (in a new tensor: undefined). A batch of no sequences at all is refused."""
    if stream is not None:
        return _under(stream, ssm_scan_backward, u, dt, A_log, B, C, dy, D, z, b_dt, offs, L, state, state_grad,
                      workspace, out)
    import torch
    n_seq = _sequences(u, offs)
    for name, t in (("state", state), ("state_grad", state_grad)):
        _expect(name, t, torch.float32, (n_seq, *A_log.shape), u)
    _expect("dy", dy, u.dtype, u.shape, u, rows=True)
    L, a = _scan_args(u, dt, A_log, B, C, D, z, b_dt, offs, n_seq, L, state)

    (rows, E), N, dt_, f32 = u.shape, A_log.shape[1], u.dtype, torch.float32
    act, vec = ((rows, E), dt_, True), ((E,), f32, False)
    r = _results(dict(du=act, ddt=act, dz=None if z is None else act, dB=((rows, N), dt_, True),
                      dC=((rows, N), dt_, True), dA_log=((E, N), f32, False), dD=vec, db_dt=vec,
                      dstate=None if state is None else ((n_seq, E, N), f32, False)), out, u)
    g = _PACK_GRADS.pack(r["du"].data_ptr(), _ld(r["du"]), r["ddt"].data_ptr(), _ld(r["ddt"]), r["dB"].data_ptr(),
                         _ld(r["dB"]), r["dC"].data_ptr(), _ld(r["dC"]), _adr(r["dz"]),
                         0 if z is None else _ld(r["dz"]), r["dA_log"].data_ptr(), r["dD"].data_ptr(),
                         r["db_dt"].data_ptr(), _adr(r["dstate"]))
    ws = _workspace(workspace, u, lib().tcl_ssm_scan_backward_workspace_bytes, n_seq, rows, E, N, L)
    check(lib().tcl_ssm_scan_backward(a, dy.data_ptr(), _ld(dy), _ptr(state_grad), g,
                                      *_ws_args(ws), _stream_of(u)))
    return r


def _heads_ld(name, t, dtype, shape, like) -> int:
    """Checks a tensor [rows, heads, width] whose rows are contiguous; its leading dimension."""
    width = shape[1] * shape[2]
    if t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == like.get_device():
        return width
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name}: {dtype} {tuple(shape)} expected, not {t.dtype} {tuple(t.shape)}")
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} is on {t.device}, not on {like.device}")
    if (shape[2] != 1 and t.stride(2) != 1) or (shape[1] != 1 and t.stride(1) != shape[2]) or (
            shape[0] != 1 and t.stride(0) < width):
        raise ValueError(f"{name}: rows not contiguous (strides {t.stride()})")
    return max(t.stride(0), width)


def _delta_args(q, k, v, g, beta, scale, offs, state):
    """(number of sequences, a state's shape, the packed tcl_delta_rule_args)"""
    import torch
    sq, sv, dt, f32 = q.shape, v.shape, q.dtype, torch.float32
    if len(sq) != 3 or len(sv) != 3:
        raise ValueError(f"q, v: [rows, heads, width] expected, not {tuple(sq)}, {tuple(sv)}")
    _on_device(q)
    (rows, Hk, Dk), (_, H, Dv) = sq, sv
    n_seq = rows
    if offs is not None:
        if offs.dim() != 1 or offs.numel() < 1:
            raise ValueError("offs: [n_seq + 1] expected")
        _expect("offs", offs, torch.int32, offs.shape, q)
        n_seq = offs.numel() - 1
    ldq, ldk = _heads_ld("q", q, dt, sq, q), _heads_ld("k", k, dt, sq, q)
    ldv = _heads_ld("v", v, dt, (rows, H, Dv), q)
    ldg, ldb = _row_ld("g", g, f32, (rows, H), q), _row_ld("beta", beta, f32, (rows, H), q)
    return n_seq, (H, Dk, Dv), _PACK_DELTA.pack(_dtype(q), n_seq, rows, Hk, H, Dk, Dv, Dk ** -0.5 if scale is None else scale,
                                   _adr(offs), q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv, g.data_ptr(),
                                   ldg, beta.data_ptr(), ldb, _adr(state))


def delta_rule_workspace(dtype, n_seq, rows, Hk, H, Dk, Dv, backward=False):
    """A workspace for delta_rule (or delta_rule_backward) with these sizes and torch type, on the
    current device."""
    import torch
    f = lib().tcl_delta_rule_backward_workspace_bytes if backward else lib().tcl_delta_rule_workspace_bytes
    size = f(TCL_BF16 if dtype is torch.bfloat16 else TCL_F32, n_seq, rows, Hk, H, Dk, Dv)
    return torch.empty(size, dtype=torch.uint8, device="cuda")


def delta_rule(q, k, v, g, beta, scale=None, offs=None, state=None, state_out=None, slots=None, out=None,
               workspace=None, stream=None):
    """The gated delta rule with carried states (tcl_delta_rule): q, k [rows, Hk, Dk] and v [rows, H, Dv]
    fp32 or bf16, g (logarithms of the decays) and beta [rows, H] and the states [n, H, Dk, Dv]
    fp32; scale None: Dk ** -0.5. offs int32 [n_seq + 1]: packed sequences; None: each row is one token of its own
    sequence. state / state_out (may be the same tensor) with slots int32 [n_seq] into them. Returns o
    [rows, H, Dv]."""
    if stream is not None:
        return _under(stream, delta_rule, q, k, v, g, beta, scale, offs, state, state_out, slots, out, workspace)
    import torch
    n_seq, shape, a = _delta_args(q, k, v, g, beta, scale, offs, state)
    n_slots = _pools(state, state_out, slots, n_seq, shape, torch.float32, q)
    if out is None:
        out, ldo = v.new_empty(v.shape), shape[0] * shape[2]
    else:
        ldo = _heads_ld("out", out, q.dtype, v.shape, q)
    ws = None if offs is None else _workspace(workspace, q, lib().tcl_delta_rule_workspace_bytes, _dtype(q), n_seq,
                                              q.shape[0], q.shape[1], *shape)
    check(lib().tcl_delta_rule(a, _ptr(slots), n_slots, _ptr(state_out), out.data_ptr(), ldo, *_ws_args(ws),
                               _stream_of(q)))
    return out


def delta_rule_backward(q, k, v, g, beta, do, scale=None, offs=None, state=None, state_grad=None, workspace=None,
                        out=None, stream=None):
    """Gradients of delta_rule (tcl_delta_rule_backward) from do [rows, H, Dv] and, for carried states
    [n_seq, H, Dk, Dv], the gradient state_grad of the end states. Returns a dict of dq, dk, dv, dg, dbeta and
    dstate (None without a state); out: contiguous tensors of those names to write to. Rows that no sequence owns
    are left as they are (in a new tensor: undefined). A batch of no sequences at all is refused."""
    if stream is not None:
        return _under(stream, delta_rule_backward, q, k, v, g, beta, do, scale, offs, state, state_grad, workspace, out)
    import torch
    n_seq, shape, a = _delta_args(q, k, v, g, beta, scale, offs, state)
    lddo = _heads_ld("do", do, q.dtype, v.shape, q)
    f32, full = torch.float32, (n_seq, *shape)
    for name, t in (("state", state), ("state_grad", state_grad)):
        _expect(name, t, f32, full, q)
    r = _results(dict(dq=(q.shape, q.dtype, False), dk=(q.shape, q.dtype, False), dv=(v.shape, q.dtype, False),
                      dg=(v.shape[:2], f32, False), dbeta=(v.shape[:2], f32, False),
                      dstate=None if state is None else (full, f32, False)), out, q)
    qk, H = q.shape[1] * q.shape[2], v.shape[1]
    gr = _PACK_DELTA_GRADS.pack(r["dq"].data_ptr(), qk, r["dk"].data_ptr(), qk, r["dv"].data_ptr(), H * v.shape[2],
                                r["dg"].data_ptr(), H, r["dbeta"].data_ptr(), H, _adr(r["dstate"]))
    ws = _workspace(workspace, q, lib().tcl_delta_rule_backward_workspace_bytes, _dtype(q), n_seq, q.shape[0],
                    q.shape[1], H, q.shape[2], v.shape[2])
    check(lib().tcl_delta_rule_backward(a, do.data_ptr(), lddo, _ptr(state_grad), gr, *_ws_args(ws), _stream_of(q)))
    return r


def _row_matrix(x):
    if x.dim() != 2:
        raise ValueError(f"[rows, channels] expected, not {tuple(x.shape)}")
    _on_device(x)
    return x.shape


def layer_norm(x, w=None, b=None, eps=1e-5, out=None, stream=None):
    """Layer norm over the columns of x [rows, C] fp32 or bf16 (tcl_layer_norm); w, b [C] fp32
    (None: ones, zeros). Returns y [rows, C]; out: a matrix to write it to, which must not overlap x."""
    if stream is not None:
        return _under(stream, layer_norm, x, w, b, eps, out)
    import torch
    shape = _row_matrix(x)
    rows, C = shape
    ldx = _row_ld("x", x, x.dtype, shape, x)
    _expect("w", w, torch.float32, (C,), x)
    _expect("b", b, torch.float32, (C,), x)
    if out is None:
        out, ldy = x.new_empty(shape), C
    else:
        ldy = _row_ld("out", out, x.dtype, shape, x)
    check(lib().tcl_layer_norm(_dtype(x), rows, C, x.data_ptr(), ldx, _ptr(w), _ptr(b), eps, out.data_ptr(), ldy,
                               _stream_of(x)))
    return out


def layer_norm_workspace(dtype, rows, C):
    """A workspace for layer_norm_backward of this torch type, on the current device."""
    import torch
    size = lib().tcl_layer_norm_workspace_bytes(TCL_BF16 if dtype is torch.bfloat16 else TCL_F32, rows, C)
    return torch.empty(size, dtype=torch.uint8, device="cuda")


def layer_norm_backward(x, w, dy, eps=1e-5, workspace=None, out=None, stream=None):
    """Gradients of layer_norm (tcl_layer_norm_backward) from dy [rows, C]; w as there. Returns a dict of
    dx, dw and db; out: tensors of those names to write to."""
    if stream is not None:
        return _under(stream, layer_norm_backward, x, w, dy, eps, workspace, out)
    import torch
    rows, C = _row_matrix(x)
    ldx, lddy = _row_ld("x", x, x.dtype, x.shape, x), _row_ld("dy", dy, x.dtype, x.shape, x)
    _expect("w", w, torch.float32, (C,), x)
    vec = ((C,), torch.float32, False)
    r = _results(dict(dx=(x.shape, x.dtype, True), dw=vec, db=vec), out, x)
    ws = _workspace(workspace, x, lib().tcl_layer_norm_workspace_bytes, _dtype(x), rows, C)
    check(lib().tcl_layer_norm_backward(_dtype(x), rows, C, x.data_ptr(), ldx, _ptr(w), eps, dy.data_ptr(), lddy,
                                        r["dx"].data_ptr(), _ld(r["dx"]), r["dw"].data_ptr(), r["db"].data_ptr(),
                                        *_ws_args(ws), _stream_of(x)))
    return r


def logits_workspace(n_rows, V, K):
    """A workspace for logprobs and distill_topk with these sizes, on the
    current device."""
    import torch
    return torch.empty(lib().tcl_logits_workspace_bytes(n_rows, V, K), dtype=torch.uint8, device="cuda")


def _logit_rows(logits, seg_offsets, max_len):
    """(rows, V, leading dimension) of rows [n, V], or of ragged segments of a
    one-dimensional array."""
    import torch
    _on_device(logits)
    if seg_offsets is None:
        if logits.dim() != 2:
            raise ValueError(f"[rows, V] logits expected, not {tuple(logits.shape)}")
        return *logits.shape, _row_ld("logits", logits, logits.dtype, logits.shape, logits)
    if logits.dim() != 1 or seg_offsets.dim() != 1 or seg_offsets.numel() < 1:
        raise ValueError("segments: logits [n] and seg_offsets [n_seg + 1] expected")
    _expect("logits", logits, logits.dtype, logits.shape, logits)
    _expect("seg_offsets", seg_offsets, torch.int32, seg_offsets.shape, logits)
    return seg_offsets.numel() - 1, max(logits.numel(), 1) if max_len is None else max_len, 0


def logprobs(logits, tokens=None, K=0, temperature=1.0, seg_offsets=None, max_len=None, workspace=None, stream=None):
    """Log probabilities of the given tokens, entropy and the K top alternatives
    (tcl_logprobs): logits fp32 or bf16 [rows, V], or [n] with seg_offsets int32 [rows + 1]
    (segments of max_len entries at most; indices then count from the array's start, as
    topk's do); tokens int32 [rows]. Returns a dict of logp (None without tokens), entropy,
    top [rows, K] int32 and top_logp [rows, K] (None for K = 0)."""
    if stream is not None:
        return _under(stream, logprobs, logits, tokens, K, temperature, seg_offsets, max_len, workspace)
    import torch
    n, V, ld = _logit_rows(logits, seg_offsets, max_len)
    _expect("tokens", tokens, torch.int32, (n,), logits)

    def new(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=logits.device)

    r = dict(logp=None if tokens is None else new(n), entropy=new(n), top=new(n, K, dtype=torch.int32) if K else None,
             top_logp=new(n, K) if K else None)
    ws = _workspace(workspace, logits, lib().tcl_logits_workspace_bytes, n, V, K)
    check(lib().tcl_logprobs(_dtype(logits), n, V, logits.data_ptr(), ld, _ptr(seg_offsets), temperature,
                             _ptr(tokens), K, _ptr(r["logp"]), r["entropy"].data_ptr(), _ptr(r["top"]),
                             _ptr(r["top_logp"]), *_ws_args(ws), _stream_of(logits)))
    return r


def distill_topk(logits, top, teacher, weight=None, temperature=1.0, seg_offsets=None, max_len=None, grad=True,
                 workspace=None, stream=None):
    """Distillation from a teacher's top logits (tcl_distill_topk): the student's
    logits as for logprobs, top int32 and teacher fp32 [rows, K], weight fp32 [rows] (the
    gradient's factor of each row). grad: True (a new tensor), False (the loss
    alone), or the tensor that takes it, which may be logits itself. Returns a dict
    of loss [rows] fp32 and grad (None if not wanted)."""
    if stream is not None:
        return _under(stream, distill_topk, logits, top, teacher, weight, temperature, seg_offsets, max_len, grad,
                      workspace)
    import torch
    n, V, ld = _logit_rows(logits, seg_offsets, max_len)
    if top.dim() != 2:
        raise ValueError(f"top: [rows, K] expected, not {tuple(top.shape)}")
    K = top.shape[1]
    _expect("top", top, torch.int32, (n, K), logits)
    _expect("teacher", teacher, torch.float32, (n, K), logits)
    _expect("weight", weight, torch.float32, (n,), logits)
    if grad is True:
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    elif grad is False:
        grad = None
    _expect("grad", grad, logits.dtype, logits.shape, logits, rows=seg_offsets is None)
    ldg = _ld(grad) if grad is not None and seg_offsets is None else 0
    loss = torch.empty(n, dtype=torch.float32, device=logits.device)
    ws = _workspace(workspace, logits, lib().tcl_logits_workspace_bytes, n, V, K)
    check(lib().tcl_distill_topk(_dtype(logits), n, V, logits.data_ptr(), ld, _ptr(seg_offsets), temperature, K,
                                 top.data_ptr(), teacher.data_ptr(), _ptr(weight), loss.data_ptr(), _ptr(grad), ldg,
                                 *_ws_args(ws), _stream_of(logits)))
    return dict(loss=loss, grad=grad)


def beam_select_workspace(groups, W, V, K):
    """A workspace for beam_select with these sizes, on the current device."""
    import torch
    return torch.empty(lib().tcl_beam_select_workspace_bytes(groups, W, V, K), dtype=torch.uint8, device="cuda")


def beam_select(logits, score, K=None, ended=None, temperature=1.0, workspace=None, stream=None):
    """The K (None: W) best continuations of each group's W beams (tcl_beam_select): logits fp32 or bf16
    [groups * W, V], score fp32 [groups, W] (-inf: a dead beam), ended int32 [groups, W] (>= 0: the beam has ended,
    with that token). Returns a dict of parent (rows of logits), token int32 and score fp32, all [groups, K]."""
    if stream is not None:
        return _under(stream, beam_select, logits, score, K, ended, temperature, workspace)
    import torch
    n, V, ld = _logit_rows(logits, None, None)
    if score.dim() != 2 or score.numel() != n:
        raise ValueError(f"score: [groups, W] with {n} beams expected, not {tuple(score.shape)}")
    G, W = score.shape
    _expect("score", score, torch.float32, (G, W), logits)
    _expect("ended", ended, torch.int32, (G, W), logits)
    K = W if K is None else K
    places = (G, max(K, 0))
    r = dict(parent=logits.new_empty(places, dtype=torch.int32), token=logits.new_empty(places, dtype=torch.int32),
             score=score.new_empty(places))
    ws = _workspace(workspace, logits, lib().tcl_beam_select_workspace_bytes, G, W, V, K)
    check(lib().tcl_beam_select(_dtype(logits), G, W, V, logits.data_ptr(), ld, temperature, score.data_ptr(),
                                _ptr(ended), K, r["parent"].data_ptr(), r["token"].data_ptr(), r["score"].data_ptr(),
                                *_ws_args(ws), _stream_of(logits)))
    return r


def beam_reorder(parent, slots, pools, out=None, stream=None):
    """The beams' states after a selection (tcl_beam_reorder): parent int32 [groups, W], the rows that the new
    beams continue; slots int32 [groups, W], the old beams' places in every one of pools (contiguous tensors
    [n_slots, ...] of any type, changed in place). Returns the new beams' places [groups, W]."""
    if stream is not None:
        return _under(stream, beam_reorder, parent, slots, pools, out)
    import torch
    if parent.dim() != 2:
        raise ValueError(f"parent: [groups, W] expected, not {tuple(parent.shape)}")
    _on_device(parent)
    G, W = parent.shape
    for name, t in (("parent", parent), ("slots", slots), ("out", out)):
        _expect(name, t, torch.int32, (G, W), parent)
    n_slots = 0
    array = (BeamPool * max(len(pools), 1))()
    for i, t in enumerate(pools):
        if t.dim() < 1 or not t.is_contiguous() or t.get_device() != parent.get_device():
            raise ValueError(f"pools[{i}]: contiguous states on {parent.device} expected")
        if i and t.shape[0] != n_slots:
            raise ValueError(f"pools of {n_slots} and {t.shape[0]} states")
        n_slots = t.shape[0]
        array[i].d_states = t.data_ptr()
        array[i].bytes = t.numel() // max(n_slots, 1) * t.element_size() if n_slots else 1
    if out is None:
        out = parent.new_empty((G, W))
    check(lib().tcl_beam_reorder(G, W, parent.data_ptr(), slots.data_ptr(), n_slots, out.data_ptr(), len(pools), array,
                                 _stream_of(parent)))
    return out


def teacher_gate(e, out=None, stream=None):
    """The teacher-loss gate of Eq. (10)-(11) (tcl_teacher_gate) over device
    fp32 batch losses e [n]; returns phi [n] (device)."""
    import torch
    if out is None:
        out = torch.empty_like(e)
    check(lib().tcl_teacher_gate(e.numel(), e.data_ptr(), out.data_ptr(), _stream(stream)))
    return out


def gemm_split(A, W, bias=None, out=None, stream=None, variant=-1, epilogue=0, offs=None):
    """The split-path fp32 GEMM (tcl_test_gemm_split). epilogue 0: A W^T
    (+ bias); 1: out += A W^T; 2: rstd(A) * A W^T; 3: A fp32 [B, L, K]
    gathered by offs [B+1], + bias, out [B*L, N]. variant 1 (32-row panels),
    2 (16-row panels), 3 (32-row panels, all N in registers), 4 (32-row
    panels, K in two halves on two wavefronts per SIMD) or -1."""
    import torch
    N, K = W.shape
    if epilogue == 3:
        Bp, L, _ = A.shape
        M = Bp * L
    else:
        M, Bp, L = A.shape[0], 0, 0
    if out is None:
        if epilogue == 1:
            raise ValueError("epilogue 1 accumulates into out")
        out = torch.empty(M, N, dtype=torch.float32, device=A.device)
    Kw = (K + 7) // 8 * 8
    scratch = torch.empty(3 * N * Kw, dtype=torch.int16, device=A.device)
    check(lib().tcl_test_gemm_split(M, N, K, A.data_ptr(), _ptr(offs), Bp, L, W.data_ptr(), _ptr(bias),
                                    out.data_ptr(), variant, epilogue, scratch.data_ptr(), _stream(stream)))
    return out


(GEMM_BF16_F32, GEMM_BF16_BF16, GEMM_BF16_NORM, GEMM_BF16_RESID, GEMM_BF16_GATHER, GEMM_BF16_F32A,
 GEMM_BF16_F32A_RESID) = range(7)


def gemm_bf16(A, W, bias=None, out=None, stream=None, kind=GEMM_BF16_F32, tile=-1, gain=None, offs=None):
    """The bf16 GEMM variants (see tcl_test_gemm_bf16): W [N, round_up(K, 8)]
    torch.bfloat16, zero-padded in K.
    GEMM_BF16_F32: A bf16 [M,K] -> fp32 (+ bias); GEMM_BF16_BF16: -> bf16;
    GEMM_BF16_NORM: A fp32 -> RMSNorm(gain) -> bf16; GEMM_BF16_RESID: out
    (fp32, required) += A W^T; GEMM_BF16_GATHER: A fp32 [B, L, K] gathered
    by offs [B+1] -> fp32 + bias, out [B*L, N]; GEMM_BF16_F32A: A fp32
    (rounded to bf16) -> fp32; GEMM_BF16_F32A_RESID: out (fp32, required)
    += bf16(A) W^T."""
    import torch
    N = W.shape[0]
    if kind == GEMM_BF16_GATHER:
        Bp, L, K = A.shape
        M = Bp * L
    else:
        (M, K), Bp, L = A.shape, 0, 0
    if W.shape[1] != (K + 7) // 8 * 8:
        raise ValueError(f"W must be [N, {(K + 7) // 8 * 8}] (K zero-padded to a multiple of 8)")
    if out is None:
        if kind in (GEMM_BF16_RESID, GEMM_BF16_F32A_RESID):
            raise ValueError("the residual kinds accumulate into out")
        bf16_out = kind in (GEMM_BF16_BF16, GEMM_BF16_NORM)
        out = torch.empty(M, N, dtype=torch.bfloat16 if bf16_out else torch.float32, device=A.device)
    check(lib().tcl_test_gemm_bf16(kind, tile, M, N, K, A.data_ptr(), _ptr(offs), Bp, L, W.data_ptr(),
                                   _ptr(bias), _ptr(gain), out.data_ptr(), _stream(stream)))
    return out


def conv_silu_f32(offs, x, w, b, E, out, ldx=None, stream=None):
    B = offs.numel() - 1
    check(lib().tcl_test_conv_silu_f32(B, E, w.shape[1], offs.data_ptr(), x.data_ptr(),
                                       x.shape[1] if ldx is None else ldx, w.data_ptr(), b.data_ptr(),
                                       out.data_ptr(), _stream(stream)))
    return out


def xproj_conv_f32(offs, x, w, b, W, rows, E, ldx=None, stream=None):
    """The fused conv + SiLU + x_proj kernel (tcl_test_xproj_conv_f32):
    returns (u [rows, E], xdbl [rows, N]); rows past offs[B] are NaN."""
    import torch
    B = offs.numel() - 1
    N = W.shape[0]
    u = torch.full((rows, E), float("nan"), dtype=torch.float32, device=x.device)
    xdbl = torch.full((rows, N), float("nan"), dtype=torch.float32, device=x.device)
    wsplit = torch.empty(3 * N * E, dtype=torch.int16, device=x.device)
    tpos = torch.empty(rows, dtype=torch.uint8, device=x.device)
    check(lib().tcl_test_xproj_conv_f32(B, rows, E, N, offs.data_ptr(), x.data_ptr(),
                                        x.shape[1] if ldx is None else ldx, w.data_ptr(), b.data_ptr(),
                                        W.data_ptr(), wsplit.data_ptr(), tpos.data_ptr(), u.data_ptr(),
                                        xdbl.data_ptr(), _stream(stream)))
    return u, xdbl


def xproj_conv_bf16(offs, x, w, b, W, rows, E, ldx=None, stream=None):
    """The bf16 fused conv + SiLU + x_proj kernel (tcl_test_xproj_conv_bf16):
    x torch.bfloat16 [rows, ldx], W torch.bfloat16 [N, E]; returns (u bf16
    [rows, E], xdbl fp32 [rows, N]); rows past offs[B] are left as they were
    (u zero, xdbl NaN)."""
    import torch
    B = offs.numel() - 1
    N = W.shape[0]
    u = torch.zeros((rows, E), dtype=torch.bfloat16, device=x.device)
    xdbl = torch.full((rows, N), float("nan"), dtype=torch.float32, device=x.device)
    tpos = torch.empty(rows, dtype=torch.uint8, device=x.device)
    check(lib().tcl_test_xproj_conv_bf16(B, rows, E, N, offs.data_ptr(), x.data_ptr(),
                                         x.shape[1] if ldx is None else ldx, w.data_ptr(), b.data_ptr(),
                                         W.data_ptr(), tpos.data_ptr(), u.data_ptr(), xdbl.data_ptr(),
                                         _stream(stream)))
    return u, xdbl


def offsets(lengths, L, ord=None, stream=None):
    """tcl_test_offsets: returns the device int32 offsets [B+1]; ord (a
    device int32 [B] tensor, optional) receives the longest-first order."""
    import torch
    B = lengths.numel()
    offs = torch.empty(B + 1, dtype=torch.int32, device=lengths.device)
    check(lib().tcl_test_offsets(B, L, lengths.data_ptr(), offs.data_ptr(), _ptr(ord), _stream(stream)))
    return offs


def scan_f32(offs, u, xdbl, z, W_dt, b_dt, A_log, D, out, ldz=None, stream=None, chunks=0):
    """chunks = 0: the sequential or the small-batch scan, as tcl_score chooses;
    1..8: chunked two-level scan."""
    B = offs.numel() - 1
    E = u.shape[1]
    N = A_log.shape[1]
    R = W_dt.shape[1]
    check(lib().tcl_test_scan_f32(B, E, N, R, chunks, offs.data_ptr(), u.data_ptr(), xdbl.data_ptr(), z.data_ptr(),
                                  z.shape[1] if ldz is None else ldz, W_dt.data_ptr(), b_dt.data_ptr(),
                                  A_log.data_ptr(), D.data_ptr(), out.data_ptr(), _stream(stream)))
    return out
