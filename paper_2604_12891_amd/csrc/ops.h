// Sequence and logit operators (internal to libtcl): the launchers behind
// tcl_ssm_* / tcl_logprobs / tcl_distill_topk, and their workspace sizes.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tcl {

// ---------------------------------------------------------------- causal conv + SiLU
struct ConvOp {
  bool bf16 = false;
  int n_seq = 0, rows = 0, E = 0, K = 0;
  const int* offs = nullptr;  // [n_seq + 1]; null: one row per sequence
  const void* x = nullptr;
  int64_t ldx = 0;
  const float* w = nullptr;   // [E, K]
  const float* b = nullptr;   // [E] or null
  const void* state = nullptr;  // [slots, K - 1, E] or null (zeros)
  const int* slots = nullptr;   // [n_seq] or null (the sequence's own index)
  int n_slots = 0;
};
hipError_t launch_ssm_conv(const ConvOp& a, void* state_out, void* u, int64_t ldu, hipStream_t s);
size_t ssm_conv_workspace_bytes(int n_seq, int rows, int E, int K);
hipError_t launch_ssm_conv_bwd(const ConvOp& a, const void* du, int64_t lddu, const void* dstate_out, void* dx,
                               int64_t lddx, float* dw, float* db, void* dstate, float* ws, hipStream_t s);

// ---------------------------------------------------------------- selective scan
struct ScanOp {
  bool bf16 = false;
  int n_seq = 0, rows = 0, E = 0, N = 0, L = 0;
  const int* offs = nullptr;  // [n_seq + 1]; null: one row per sequence
  const void *u = nullptr, *dt = nullptr, *B = nullptr, *C = nullptr, *z = nullptr;  // z may be null
  int64_t ldu = 0, lddt = 0, ldB = 0, ldC = 0, ldz = 0;
  const float *A_log = nullptr, *D = nullptr, *b_dt = nullptr;  // [E, N]; [E] or null
  const float* state = nullptr;  // [slots, E, N] or null (zeros)
  const int* slots = nullptr;
  int n_slots = 0;
};
struct ScanGrads {
  void *du = nullptr, *ddt = nullptr, *dB = nullptr, *dC = nullptr, *dz = nullptr;
  int64_t lddu = 0, ldddt = 0, lddB = 0, lddC = 0, lddz = 0;
  float *dA_log = nullptr, *dD = nullptr, *db_dt = nullptr;
  float* dstate = nullptr;
};
size_t ssm_scan_workspace_bytes(int n_seq, int rows, int E, int N, int L);
hipError_t launch_ssm_scan(const ScanOp& a, float* state_out, void* y, int64_t ldy, float* ws, hipStream_t s);
size_t ssm_scan_bwd_workspace_bytes(int n_seq, int rows, int E, int N, int L);
hipError_t launch_ssm_scan_bwd(const ScanOp& a, const void* dy, int64_t lddy, const float* dstate_out,
                               const ScanGrads& g, float* ws, hipStream_t s);

// ---------------------------------------------------------------- logits
// Rows of V entries with leading dimension ld, or (offs non-null) ragged
// segments offs[r] .. offs[r + 1] - 1 of one array, V entries at most.
struct LogitRows {
  bool bf16 = false;
  int n = 0, V = 0;
  const void* x = nullptr;
  int64_t ld = 0;
  const int* offs = nullptr;
  float inv_temp = 1.f;
};
size_t logits_workspace_bytes(int n, int V, int K);
hipError_t launch_logprobs(const LogitRows& a, const int* tokens, int K, float* logp, float* entropy, int* top,
                           float* top_logp, void* ws, hipStream_t s);
hipError_t launch_distill_topk(const LogitRows& a, int K, const int* top, const float* teacher, const float* weight,
                               float* loss, void* grad, int64_t ldg, void* ws, hipStream_t s);

}  // namespace tcl
