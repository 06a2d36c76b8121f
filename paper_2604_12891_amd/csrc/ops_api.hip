// C entry points of the sequence and logit operators (include/tcl.h): argument
// checks, then the launchers of ssm.hip and logits.hip.
#include <cmath>

#include "model.h"
#include "ops.h"

using namespace tcl;

namespace {

bool misaligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

// A launch has fewer than 2^32 threads. A scan's tiles hold 30 rows or more, besides one per sequence, and
// their channels are rounded up to 64, in the gradients (wavefronts in fours) to less than twice that: with these
// bounds 2 (2^34 / 30 + 2^30) threads at most, and row and tile indices far inside 31 bits. The convolution's
// tiles hold 8 to 16 rows only where 32 would give fewer than 2^17 threads, 32 or more else, and a thread takes
// one channel or more of a tile: 2^34 / 32 + 2^30 threads at most.
constexpr int kMaxRows = 1 << 30;
constexpr int64_t kMaxRowWork = (int64_t)1 << 34, kMaxSeqWork = (int64_t)1 << 30;
// Rows of logits take a workgroup of up to 1,024 threads each.
constexpr int kMaxLogitRows = (1 << 22) - 1;
constexpr float kMinTemp = 1e-30f, kMaxTemp = 1e30f;

tcl_status check_workspace(const void* d_ws, size_t have, size_t need) {
  if (need == 0) return TCL_OK;
  if (!d_ws) return fail(TCL_ERR_INVALID_ARG, "NULL workspace (needs %zu bytes)", need);
  if (misaligned(d_ws, 256)) return fail(TCL_ERR_INVALID_ARG, "d_workspace must be 256-byte aligned");
  if (have < need) return fail(TCL_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", have, need);
  return TCL_OK;
}

tcl_status check_sequences(int32_t dtype, int32_t n_seq, int32_t rows, int32_t E, const int32_t* d_offs) {
  if (dtype != TCL_F32 && dtype != TCL_BF16) return fail(TCL_ERR_INVALID_ARG, "bad dtype %d", dtype);
  if (n_seq < 0 || rows < 0) return fail(TCL_ERR_INVALID_ARG, "negative size (n_seq=%d rows=%d)", n_seq, rows);
  if (!d_offs && rows != n_seq)
    return fail(TCL_ERR_INVALID_ARG, "without d_offs every sequence is one row (n_seq=%d rows=%d)", n_seq, rows);
  if (E < 1 || E > 65536) return fail(TCL_ERR_UNSUPPORTED, "E must be in [1, 65536] (got %d)", E);
  const int64_t C = ((int64_t)E + 63) / 64 * 64;
  if (n_seq > kMaxRows || rows > kMaxRows || rows * C > kMaxRowWork || n_seq * C > kMaxSeqWork)
    return fail(TCL_ERR_UNSUPPORTED, "too many rows or sequences x channels (n_seq=%d rows=%d E=%d)", n_seq, rows, E);
  return TCL_OK;
}

tcl_status check_slots(const int32_t* d_slots, int32_t n_slots, int32_t n_seq, bool pools) {
  if (n_slots < 0) return fail(TCL_ERR_INVALID_ARG, "n_slots must not be negative");
  if (!d_slots && pools && n_slots < n_seq)
    return fail(TCL_ERR_INVALID_ARG, "without d_slots the pool needs a state per sequence (n_slots=%d n_seq=%d)",
                n_slots, n_seq);
  return TCL_OK;
}

tcl_status conv_op(const tcl_ssm_conv_args* a, ConvOp* op) {
  if (!a) return fail(TCL_ERR_INVALID_ARG, "args is NULL");
  if (tcl_status st = check_sequences(a->dtype, a->n_seq, a->rows, a->E, a->d_offs)) return st;
  if (a->K < 1 || a->K > 4) return fail(TCL_ERR_UNSUPPORTED, "K must be in [1, 4] (got %d)", a->K);
  if (a->ldx < a->E) return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than E");
  if (!a->d_w || (!a->d_x && a->rows > 0)) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  op->bf16 = a->dtype == TCL_BF16;
  op->n_seq = a->n_seq; op->rows = a->rows; op->E = a->E; op->K = a->K;
  op->offs = a->d_offs; op->x = a->d_x; op->ldx = a->ldx; op->w = a->d_w; op->b = a->d_b;
  op->state = a->d_state;
  return TCL_OK;
}

tcl_status scan_op(const tcl_ssm_scan_args* a, ScanOp* op) {
  if (!a) return fail(TCL_ERR_INVALID_ARG, "args is NULL");
  if (tcl_status st = check_sequences(a->dtype, a->n_seq, a->rows, a->E, a->d_offs)) return st;
  if (a->N != 8 && a->N != 16) return fail(TCL_ERR_UNSUPPORTED, "N must be 8 or 16 (got %d)", a->N);
  if (a->d_offs && a->L < 1) return fail(TCL_ERR_INVALID_ARG, "L must be positive (got %d)", a->L);
  if (a->ldu < a->E || a->lddt < a->E || a->ldB < a->N || a->ldC < a->N || (a->d_z && a->ldz < a->E))
    return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than the row");
  if (!a->d_A_log || (a->rows > 0 && (!a->d_u || !a->d_dt || !a->d_B || !a->d_C)))
    return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  if (misaligned(a->d_A_log, 16) || misaligned(a->d_state, 16))
    return fail(TCL_ERR_INVALID_ARG, "A_log and the states must be 16-byte aligned");
  op->bf16 = a->dtype == TCL_BF16;
  op->n_seq = a->n_seq; op->rows = a->rows; op->E = a->E; op->N = a->N; op->L = a->d_offs ? a->L : 1;
  op->offs = a->d_offs;
  op->u = a->d_u; op->dt = a->d_dt; op->B = a->d_B; op->C = a->d_C; op->z = a->d_z;
  op->ldu = a->ldu; op->lddt = a->lddt; op->ldB = a->ldB; op->ldC = a->ldC; op->ldz = a->ldz;
  op->A_log = a->d_A_log; op->D = a->d_D; op->b_dt = a->d_b_dt; op->state = a->d_state;
  return TCL_OK;
}

tcl_status logit_rows(int32_t dtype, int32_t n_rows, int32_t V, const void* d_logits, int64_t ld,
                      const int32_t* d_seg_offsets, float temperature, LogitRows* a) {
  if (dtype != TCL_F32 && dtype != TCL_BF16) return fail(TCL_ERR_INVALID_ARG, "bad dtype %d", dtype);
  if (n_rows < 0 || V < 1) return fail(TCL_ERR_INVALID_ARG, "need n_rows >= 0, V > 0 (got %d, %d)", n_rows, V);
  if (V > (1 << 30)) return fail(TCL_ERR_UNSUPPORTED, "V must be at most 2^30 (got %d)", V);
  if (n_rows > kMaxLogitRows) return fail(TCL_ERR_UNSUPPORTED, "n_rows must be below 2^22 (got %d)", n_rows);
  if (!d_seg_offsets && ld < V) return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than V");
  if (!(temperature >= kMinTemp && temperature <= kMaxTemp))
    return fail(TCL_ERR_INVALID_ARG, "temperature must be in [1e-30, 1e30]");
  if (!d_logits && !d_seg_offsets && n_rows > 0) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  if (misaligned(d_logits, dtype == TCL_BF16 ? 2 : 4))
    return fail(TCL_ERR_INVALID_ARG, "logits are not aligned to their type");
  a->bf16 = dtype == TCL_BF16;
  a->n = n_rows; a->V = V; a->x = d_logits; a->ld = ld; a->offs = d_seg_offsets;
  a->inv_temp = 1.0f / temperature;
  return TCL_OK;
}

}  // namespace

// ------------------------------------------------------------------ convolution

TCL_API tcl_status tcl_ssm_conv(const tcl_ssm_conv_args* args, const int32_t* d_slots, int32_t n_slots,
                                void* d_state_out, void* d_u, int64_t ldu, void* stream) {
  ConvOp op;
  if (tcl_status st = conv_op(args, &op)) return st;
  if (tcl_status st = check_slots(d_slots, n_slots, op.n_seq, op.K > 1 && (op.state || d_state_out))) return st;
  if (ldu < op.E) return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than E");
  if (!d_u && op.rows > 0) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  if (op.n_seq == 0) return TCL_OK;
  op.slots = d_slots;
  op.n_slots = n_slots;
  TCL_HIP(launch_ssm_conv(op, d_state_out, d_u, ldu, static_cast<hipStream_t>(stream)));
  return TCL_OK;
}

TCL_API size_t tcl_ssm_conv_workspace_bytes(int32_t n_seq, int32_t rows, int32_t E, int32_t K) {
  if (n_seq <= 0 || n_seq > kMaxRows || rows < 0 || E < 1 || E > 65536 || K < 1 || K > 4) return 0;
  return ssm_conv_workspace_bytes(n_seq, rows, E, K);
}

TCL_API tcl_status tcl_ssm_conv_backward(const tcl_ssm_conv_args* args, const void* d_du, int64_t lddu,
                                         const void* d_dstate_out, void* d_dx, int64_t lddx, float* d_dw,
                                         float* d_db, void* d_dstate, void* d_workspace, size_t ws_bytes,
                                         void* stream) {
  ConvOp op;
  if (tcl_status st = conv_op(args, &op)) return st;
  if (lddu < op.E || lddx < op.E) return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than E");
  if (!d_dw || (op.rows > 0 && (!d_du || !d_dx))) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  if (op.n_seq == 0) return fail(TCL_ERR_INVALID_ARG, "no sequences to take gradients of");
  op.n_slots = op.n_seq;
  if (tcl_status st = check_workspace(d_workspace, ws_bytes, ssm_conv_workspace_bytes(op.n_seq, op.rows, op.E, op.K)))
    return st;
  TCL_HIP(launch_ssm_conv_bwd(op, d_du, lddu, d_dstate_out, d_dx, lddx, d_dw, d_db, d_dstate,
                              static_cast<float*>(d_workspace), static_cast<hipStream_t>(stream)));
  return TCL_OK;
}

// ------------------------------------------------------------------ selective scan

TCL_API size_t tcl_ssm_scan_workspace_bytes(int32_t n_seq, int32_t rows, int32_t E, int32_t N, int32_t L) {
  if (n_seq <= 0 || n_seq > kMaxRows || rows < 0 || E < 1 || E > 65536 || (N != 8 && N != 16) || L < 1) return 0;
  return ssm_scan_workspace_bytes(n_seq, rows, E, N, L);
}

TCL_API tcl_status tcl_ssm_scan(const tcl_ssm_scan_args* args, const int32_t* d_slots, int32_t n_slots,
                                float* d_state_out, void* d_y, int64_t ldy, void* d_workspace, size_t ws_bytes,
                                void* stream) {
  ScanOp op;
  if (tcl_status st = scan_op(args, &op)) return st;
  if (tcl_status st = check_slots(d_slots, n_slots, op.n_seq, op.state || d_state_out)) return st;
  if (ldy < op.E) return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than E");
  if (!d_y && op.rows > 0) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  if (misaligned(d_state_out, 16)) return fail(TCL_ERR_INVALID_ARG, "the states must be 16-byte aligned");
  if (op.n_seq == 0) return TCL_OK;
  op.slots = d_slots;
  op.n_slots = n_slots;
  const size_t need = op.offs ? ssm_scan_workspace_bytes(op.n_seq, op.rows, op.E, op.N, op.L) : 0;
  if (tcl_status st = check_workspace(d_workspace, ws_bytes, need)) return st;
  TCL_HIP(launch_ssm_scan(op, d_state_out, d_y, ldy, static_cast<float*>(d_workspace),
                          static_cast<hipStream_t>(stream)));
  return TCL_OK;
}

TCL_API size_t tcl_ssm_scan_backward_workspace_bytes(int32_t n_seq, int32_t rows, int32_t E, int32_t N, int32_t L) {
  if (n_seq <= 0 || n_seq > kMaxRows || rows < 0 || E < 1 || E > 65536 || (N != 8 && N != 16) || L < 1) return 0;
  return ssm_scan_bwd_workspace_bytes(n_seq, rows, E, N, L);
}

TCL_API tcl_status tcl_ssm_scan_backward(const tcl_ssm_scan_args* args, const void* d_dy, int64_t lddy,
                                         const float* d_dstate_out, const tcl_ssm_scan_grads* g, void* d_workspace,
                                         size_t ws_bytes, void* stream) {
  ScanOp op;
  if (tcl_status st = scan_op(args, &op)) return st;
  if (!g) return fail(TCL_ERR_INVALID_ARG, "grads is NULL");
  if (lddy < op.E || g->lddu < op.E || g->ldddt < op.E || g->lddB < op.N || g->lddC < op.N ||
      (g->d_dz && g->lddz < op.E))
    return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than the row");
  if (!g->d_dA_log || (op.rows > 0 && (!d_dy || !g->d_du || !g->d_ddt || !g->d_dB || !g->d_dC)))
    return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  if (op.rows > 0 && (op.z != nullptr) != (g->d_dz != nullptr))
    return fail(TCL_ERR_INVALID_ARG, "d_dz goes with d_z");
  if (misaligned(d_dstate_out, 16) || misaligned(g->d_dstate, 16))
    return fail(TCL_ERR_INVALID_ARG, "the states' gradients must be 16-byte aligned");
  if (op.n_seq == 0) return fail(TCL_ERR_INVALID_ARG, "no sequences to take gradients of");
  op.n_slots = op.n_seq;
  const size_t need = ssm_scan_bwd_workspace_bytes(op.n_seq, op.rows, op.E, op.N, op.L);
  if (tcl_status st = check_workspace(d_workspace, ws_bytes, need)) return st;
  ScanGrads o;
  o.du = g->d_du; o.ddt = g->d_ddt; o.dB = g->d_dB; o.dC = g->d_dC; o.dz = g->d_dz;
  o.lddu = g->lddu; o.ldddt = g->ldddt; o.lddB = g->lddB; o.lddC = g->lddC; o.lddz = g->lddz;
  o.dA_log = g->d_dA_log; o.dD = g->d_dD; o.db_dt = g->d_db_dt; o.dstate = g->d_dstate;
  TCL_HIP(launch_ssm_scan_bwd(op, d_dy, lddy, d_dstate_out, o, static_cast<float*>(d_workspace),
                              static_cast<hipStream_t>(stream)));
  return TCL_OK;
}

// ------------------------------------------------------------------ logits

TCL_API size_t tcl_logits_workspace_bytes(int32_t n_rows, int32_t V, int32_t K) {
  if (n_rows <= 0 || V < 1 || V > (1 << 30) || K < 0 || K > 1024) return 0;
  return logits_workspace_bytes(n_rows, V, K);
}

TCL_API tcl_status tcl_logprobs(int32_t dtype, int32_t n_rows, int32_t V, const void* d_logits, int64_t ld,
                                const int32_t* d_seg_offsets, float temperature, const int32_t* d_tokens, int32_t K,
                                float* d_logp, float* d_entropy, int32_t* d_top, float* d_top_logp,
                                void* d_workspace, size_t ws_bytes, void* stream) {
  LogitRows a;
  if (tcl_status st = logit_rows(dtype, n_rows, V, d_logits, ld, d_seg_offsets, temperature, &a)) return st;
  if (K < 0 || K > 64) return fail(TCL_ERR_UNSUPPORTED, "K must be in [0, 64] (got %d)", K);
  if (n_rows == 0) return TCL_OK;
  if ((d_logp && !d_tokens) || (K > 0 && !d_top)) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  if (tcl_status st = check_workspace(d_workspace, ws_bytes, logits_workspace_bytes(n_rows, V, K))) return st;
  TCL_HIP(launch_logprobs(a, d_tokens, K, d_logp, d_entropy, d_top, d_top_logp, d_workspace,
                          static_cast<hipStream_t>(stream)));
  return TCL_OK;
}

TCL_API tcl_status tcl_distill_topk(int32_t dtype, int32_t n_rows, int32_t V, const void* d_logits, int64_t ld,
                                    const int32_t* d_seg_offsets, float temperature, int32_t K,
                                    const int32_t* d_top, const float* d_teacher, const float* d_weight,
                                    float* d_loss, void* d_grad, int64_t ldg, void* d_workspace, size_t ws_bytes,
                                    void* stream) {
  LogitRows a;
  if (tcl_status st = logit_rows(dtype, n_rows, V, d_logits, ld, d_seg_offsets, temperature, &a)) return st;
  if (K < 1 || K > 1024) return fail(TCL_ERR_UNSUPPORTED, "K must be in [1, 1024] (got %d)", K);
  if (n_rows == 0) return TCL_OK;
  if (!d_top || !d_teacher || !d_loss) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  if (d_grad && !d_seg_offsets && ldg < V) return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than V");
  if (d_grad == d_logits && !d_seg_offsets && ldg != ld)
    return fail(TCL_ERR_INVALID_ARG, "a gradient in place of the logits needs their leading dimension");
  if (misaligned(d_grad, dtype == TCL_BF16 ? 2 : 4))
    return fail(TCL_ERR_INVALID_ARG, "the gradient is not aligned to its type");
  if (tcl_status st = check_workspace(d_workspace, ws_bytes, logits_workspace_bytes(n_rows, V, K))) return st;
  TCL_HIP(launch_distill_topk(a, K, d_top, d_teacher, d_weight, d_loss, d_grad, ldg, d_workspace,
                              static_cast<hipStream_t>(stream)));
  return TCL_OK;
}
