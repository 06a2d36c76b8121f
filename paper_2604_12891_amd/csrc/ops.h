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
// Sums of `parts` partial vectors part[p][total][E], M of them laid out as o0 [E, M], the next
// two (null: not wanted) as o1 [E] and o2 [E]; in a fixed order.
void sum_parts(const float* part, int parts, int M, int total, int E, float* o0, float* o1, float* o2, hipStream_t s);
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

// ---------------------------------------------------------------- layer norm
struct NormOp {
  bool bf16 = false;
  int rows = 0, C = 0;
  const void* x = nullptr;
  int64_t ldx = 0;
  const float *w = nullptr, *b = nullptr;  // [C] or null (ones, zeros)
  float eps = 1e-5f;
};
constexpr int kMaxNormC = 16384;
hipError_t launch_layer_norm(const NormOp& a, void* y, int64_t ldy, hipStream_t s);
size_t layer_norm_workspace_bytes(bool bf16, int rows, int C);
hipError_t launch_layer_norm_bwd(const NormOp& a, const void* dy, int64_t lddy, void* dx, int64_t lddx, float* dw,
                                 float* db, float* ws, hipStream_t s);

// ---------------------------------------------------------------- gated delta rule
struct DeltaOp {
  bool bf16 = false;
  int n_seq = 0, rows = 0, Hk = 0, H = 0, Dk = 0, Dv = 0;
  const int* offs = nullptr;  // [n_seq + 1]; null: one row per sequence
  const void *q = nullptr, *k = nullptr, *v = nullptr;
  int64_t ldq = 0, ldk = 0, ldv = 0;
  const float *g = nullptr, *beta = nullptr;
  int64_t ldg = 0, ldb = 0;
  float scale = 1.f;
  const float* state = nullptr;  // [slots, H, Dk, Dv] or null (zeros)
  const int* slots = nullptr;
  int n_slots = 0;
};
struct DeltaGrads {
  void *dq = nullptr, *dk = nullptr, *dv = nullptr;
  int64_t lddq = 0, lddk = 0, lddv = 0;
  float *dg = nullptr, *dbeta = nullptr;
  int64_t lddg = 0, lddb = 0;
  float* dstate = nullptr;
};
size_t delta_rule_workspace_bytes(bool bf16, int n_seq, int rows, int Hk, int H, int Dk, int Dv);
hipError_t launch_delta_rule(const DeltaOp& a, float* state_out, void* o, int64_t ldo, float* ws, hipStream_t s);
size_t delta_rule_bwd_workspace_bytes(bool bf16, int n_seq, int rows, int Hk, int H, int Dk, int Dv);
hipError_t launch_delta_rule_bwd(const DeltaOp& a, const void* d_o, int64_t lddo, const float* dstate_out,
                                 const DeltaGrads& g, float* ws, hipStream_t s);

// ---------------------------------------------------------------- beam search
// Row g W + b holds beam b of group g.
size_t beam_select_workspace_bytes(int groups, int W, int V, int K);
hipError_t launch_beam_select(const LogitRows& a, int W, int K, const float* score, const int* ended, int* parent,
                              int* token, float* out_score, void* ws, hipStream_t s);
constexpr int kPoolsPerLaunch = 64;
struct BeamPool {
  void* data;
  int64_t bytes;  // of one state
};
hipError_t launch_beam_reorder(int groups, int W, const int* parent, const int* slots, int n_slots, int* slots_out,
                               int n_pools, const BeamPool* pools, hipStream_t s);

}  // namespace tcl
