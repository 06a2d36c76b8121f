// C entry points of the sequence and logit operators (include/tcl.h): argument
// checks, then the launchers of ssm.hip, delta.hip, norm.hip, logits.hip and beam.hip.
#include <algorithm>
#include <cmath>
#include <numeric>

#include "model.h"
#include "ops.h"

using namespace tcl;

namespace {

bool misaligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

// Matrices of n rows of w bytes, ld apart, that share a byte; columns beside each other in one buffer, or rows between each
// other's, do not.
struct Rows {
  const void* p;
  int64_t n, w, ld;
};
Rows flat(const void* p, size_t bytes) { return {p, bytes > 0, (int64_t)bytes, (int64_t)bytes}; }
bool overlap(Rows a, Rows b) {
  if (!a.p || !b.p || a.n < 1 || b.n < 1) return false;
  const int64_t x = reinterpret_cast<int64_t>(a.p), y = reinterpret_cast<int64_t>(b.p);
  const int64_t x_end = x + (a.n - 1) * a.ld + a.w, y_end = y + (b.n - 1) * b.ld + b.w;
  if (x >= y_end || y >= x_end) return false;
  // where rows of b begin behind rows of a: always the same, modulo what both strides are multiples of
  const int64_t g = std::gcd(a.ld, b.ld), d = ((y - x) % g + g) % g;
  if (d >= a.w && g - d >= b.w) return false;
  for (int64_t i = std::max<int64_t>(0, (y - a.w - x) / a.ld); i < a.n && x + i * a.ld < y_end; ++i) {
    const int64_t at = x + i * a.ld, last = at + a.w - 1 - y;  // b's last row that begins in front of the row's end
    if (last >= 0 && y + std::min(b.n - 1, last / b.ld) * b.ld + b.w > at) return true;
  }
  return false;
}

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

// ------------------------------------------------------------------ layer norm

namespace {

tcl_status norm_op(int32_t dtype, int32_t rows, int32_t C, const void* d_x, int64_t ldx, const float* d_w,
                   const float* d_b, float eps, NormOp* op) {
  if (dtype != TCL_F32 && dtype != TCL_BF16) return fail(TCL_ERR_INVALID_ARG, "bad dtype %d", dtype);
  if (rows < 0 || C < 1) return fail(TCL_ERR_INVALID_ARG, "need rows >= 0, C > 0 (got %d, %d)", rows, C);
  if (C > kMaxNormC) return fail(TCL_ERR_UNSUPPORTED, "C must be at most %d (got %d)", kMaxNormC, C);
  if (rows > kMaxRows) return fail(TCL_ERR_UNSUPPORTED, "rows must be at most 2^30 (got %d)", rows);
  if (ldx < C) return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than C");
  if (!(eps >= 0.f && eps < INFINITY)) return fail(TCL_ERR_INVALID_ARG, "eps must be finite and not negative");
  if (!d_x && rows > 0) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  if (misaligned(d_x, dtype == TCL_BF16 ? 2 : 4)) return fail(TCL_ERR_INVALID_ARG, "x is not aligned to its type");
  op->bf16 = dtype == TCL_BF16;
  op->rows = rows; op->C = C; op->x = d_x; op->ldx = ldx; op->w = d_w; op->b = d_b; op->eps = eps;
  return TCL_OK;
}

}  // namespace

TCL_API tcl_status tcl_layer_norm(int32_t dtype, int32_t rows, int32_t C, const void* d_x, int64_t ldx,
                                  const float* d_w, const float* d_b, float eps, void* d_y, int64_t ldy,
                                  void* stream) {
  NormOp op;
  if (tcl_status st = norm_op(dtype, rows, C, d_x, ldx, d_w, d_b, eps, &op)) return st;
  if (ldy < C) return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than C");
  if (rows == 0) return TCL_OK;
  if (!d_y) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  const int64_t el = op.bf16 ? 2 : 4;
  if (misaligned(d_y, el)) return fail(TCL_ERR_INVALID_ARG, "y is not aligned to its type");
  const Rows y = {d_y, rows, C * el, ldy * el};
  if (overlap(y, {d_x, rows, C * el, ldx * el}) || overlap(y, flat(d_w, C * 4)) || overlap(y, flat(d_b, C * 4)))
    return fail(TCL_ERR_INVALID_ARG, "y overlaps an input");
  TCL_HIP(launch_layer_norm(op, d_y, ldy, static_cast<hipStream_t>(stream)));
  return TCL_OK;
}

TCL_API size_t tcl_layer_norm_workspace_bytes(int32_t dtype, int32_t rows, int32_t C) {
  if ((dtype != TCL_F32 && dtype != TCL_BF16) || rows <= 0 || rows > kMaxRows || C < 1 || C > kMaxNormC) return 0;
  return layer_norm_workspace_bytes(dtype == TCL_BF16, rows, C);
}

TCL_API tcl_status tcl_layer_norm_backward(int32_t dtype, int32_t rows, int32_t C, const void* d_x, int64_t ldx,
                                           const float* d_w, float eps, const void* d_dy, int64_t lddy, void* d_dx,
                                           int64_t lddx, float* d_dw, float* d_db, void* d_workspace,
                                           size_t ws_bytes, void* stream) {
  NormOp op;
  if (tcl_status st = norm_op(dtype, rows, C, d_x, ldx, d_w, nullptr, eps, &op)) return st;
  if (lddy < C || lddx < C) return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than C");
  if (!d_dw || (rows > 0 && (!d_dy || !d_dx))) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  const int64_t el = op.bf16 ? 2 : 4;
  if (misaligned(d_dy, el) || misaligned(d_dx, el))
    return fail(TCL_ERR_INVALID_ARG, "dy and dx have to be aligned to their type");
  const size_t need = rows > 0 ? layer_norm_workspace_bytes(op.bf16, rows, C) : 0;
  if (tcl_status st = check_workspace(d_workspace, ws_bytes, need)) return st;
  const Rows dx = {d_dx, rows, C * el, lddx * el}, dw = flat(d_dw, C * 4), db = flat(d_db, C * 4), ws = flat(d_workspace, need);
  if (overlap(dx, {d_x, rows, C * el, ldx * el}) || overlap(dx, {d_dy, rows, C * el, lddy * el}) ||
      overlap(dx, flat(d_w, C * 4)) || overlap(dx, ws) || overlap(dw, ws) || overlap(db, ws))
    return fail(TCL_ERR_INVALID_ARG, "an output overlaps an input or the workspace");
  if (overlap(dw, db) || overlap(dw, dx) || overlap(db, dx))
    return fail(TCL_ERR_INVALID_ARG, "outputs overlap each other");
  TCL_HIP(launch_layer_norm_bwd(op, d_dy, lddy, d_dx, lddx, d_dw, d_db, static_cast<float*>(d_workspace),
                                static_cast<hipStream_t>(stream)));
  return TCL_OK;
}

// ------------------------------------------------------------------ gated delta rule

namespace {

// Fewer than 2^32 threads a launch: of packed sequences a head takes 16 workgroups of 512 at most (kMaxSeqHeads),
// of single tokens 8 of 64 (kMaxTokenHeads); a chunk's key head, of 64 rows or the rest of a sequence, one of 512.
constexpr int64_t kMaxSeqHeads = ((int64_t)1 << 19) - 1, kMaxTokenHeads = ((int64_t)1 << 22) - 1;
constexpr int kMaxHeads = 1024, kMaxDk = 128, kMaxDv = 256;
// (a chunk's rows are addressed in 31 bits)
constexpr int64_t kMaxLd = (int64_t)1 << 22;

bool delta_sizes(int32_t n_seq, int32_t rows, int32_t Hk, int32_t H, int32_t Dk, int32_t Dv) {
  return n_seq >= 0 && rows >= 0 && n_seq <= kMaxRows && rows <= kMaxRows && Hk >= 1 && H >= Hk && H <= kMaxHeads &&
         H % Hk == 0 && Dk >= 8 && Dk <= kMaxDk && Dk % 8 == 0 && Dv >= 8 && Dv <= kMaxDv && Dv % 8 == 0 &&
         (int64_t)rows * H <= ((int64_t)1 << 28) && (int64_t)n_seq * H <= kMaxTokenHeads;
}

tcl_status delta_op(const tcl_delta_rule_args* a, DeltaOp* op) {
  if (!a) return fail(TCL_ERR_INVALID_ARG, "args is NULL");
  if (a->dtype != TCL_F32 && a->dtype != TCL_BF16) return fail(TCL_ERR_INVALID_ARG, "bad dtype %d", a->dtype);
  if (a->n_seq < 0 || a->rows < 0)
    return fail(TCL_ERR_INVALID_ARG, "negative size (n_seq=%d rows=%d)", a->n_seq, a->rows);
  if (!a->d_offs && a->rows != a->n_seq)
    return fail(TCL_ERR_INVALID_ARG, "without d_offs every sequence is one row (n_seq=%d rows=%d)", a->n_seq, a->rows);
  if (a->Hk < 1 || a->H < a->Hk || a->H > kMaxHeads || a->H % a->Hk)
    return fail(TCL_ERR_UNSUPPORTED, "H must be a multiple of Hk, at most %d (got %d, %d)", kMaxHeads, a->H, a->Hk);
  if (a->Dk < 8 || a->Dk > kMaxDk || a->Dk % 8 || a->Dv < 8 || a->Dv > kMaxDv || a->Dv % 8)
    return fail(TCL_ERR_UNSUPPORTED, "Dk and Dv must be multiples of 8, at most %d and %d (got %d, %d)", kMaxDk, kMaxDv,
                a->Dk, a->Dv);
  if (!delta_sizes(a->n_seq, a->rows, a->Hk, a->H, a->Dk, a->Dv) ||
      (a->d_offs && (int64_t)a->n_seq * a->H > kMaxSeqHeads))
    return fail(TCL_ERR_UNSUPPORTED, "too many rows or sequences x heads (n_seq=%d rows=%d H=%d)", a->n_seq, a->rows,
                a->H);
  const int64_t qk = (int64_t)a->Hk * a->Dk, v = (int64_t)a->H * a->Dv;
  if (a->ldq < qk || a->ldk < qk || a->ldv < v || a->ldg < a->H || a->ldbeta < a->H)
    return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than the row");
  if (a->ldq > kMaxLd || a->ldk > kMaxLd || a->ldv > kMaxLd)
    return fail(TCL_ERR_UNSUPPORTED, "leading dimensions must be at most %lld", (long long)kMaxLd);
  if (a->rows > 0 && (!a->d_q || !a->d_k || !a->d_v || !a->d_g || !a->d_beta))
    return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  const uintptr_t el = a->dtype == TCL_BF16 ? 2 : 4;
  if (misaligned(a->d_q, el) || misaligned(a->d_k, el) || misaligned(a->d_v, el))
    return fail(TCL_ERR_INVALID_ARG, "activations are not aligned to their type");
  if (misaligned(a->d_state, 16)) return fail(TCL_ERR_INVALID_ARG, "the states must be 16-byte aligned");
  op->bf16 = a->dtype == TCL_BF16;
  op->n_seq = a->n_seq; op->rows = a->rows; op->Hk = a->Hk; op->H = a->H; op->Dk = a->Dk; op->Dv = a->Dv;
  op->offs = a->d_offs;
  op->q = a->d_q; op->k = a->d_k; op->v = a->d_v; op->ldq = a->ldq; op->ldk = a->ldk; op->ldv = a->ldv;
  op->g = a->d_g; op->beta = a->d_beta; op->ldg = a->ldg; op->ldb = a->ldbeta;
  op->scale = a->scale; op->state = a->d_state;
  return TCL_OK;
}

}  // namespace

TCL_API size_t tcl_delta_rule_workspace_bytes(int32_t dtype, int32_t n_seq, int32_t rows, int32_t Hk, int32_t H,
                                              int32_t Dk, int32_t Dv) {
  if ((dtype != TCL_F32 && dtype != TCL_BF16) || n_seq == 0 || !delta_sizes(n_seq, rows, Hk, H, Dk, Dv)) return 0;
  return delta_rule_workspace_bytes(dtype == TCL_BF16, n_seq, rows, Hk, H, Dk, Dv);
}

TCL_API tcl_status tcl_delta_rule(const tcl_delta_rule_args* args, const int32_t* d_slots, int32_t n_slots,
                                  float* d_state_out, void* d_o, int64_t ldo, void* d_workspace, size_t ws_bytes,
                                  void* stream) {
  DeltaOp op;
  if (tcl_status st = delta_op(args, &op)) return st;
  if (tcl_status st = check_slots(d_slots, n_slots, op.n_seq, op.state || d_state_out)) return st;
  if (ldo < (int64_t)op.H * op.Dv) return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than the row");
  if (ldo > kMaxLd) return fail(TCL_ERR_UNSUPPORTED, "leading dimensions must be at most %lld", (long long)kMaxLd);
  if (!d_o && op.rows > 0) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  if (misaligned(d_o, op.bf16 ? 2 : 4)) return fail(TCL_ERR_INVALID_ARG, "o is not aligned to its type");
  if (misaligned(d_state_out, 16)) return fail(TCL_ERR_INVALID_ARG, "the states must be 16-byte aligned");
  if (op.n_seq == 0) return TCL_OK;
  op.slots = d_slots;
  op.n_slots = n_slots;
  const size_t need =
      op.offs ? delta_rule_workspace_bytes(op.bf16, op.n_seq, op.rows, op.Hk, op.H, op.Dk, op.Dv) : 0;
  if (tcl_status st = check_workspace(d_workspace, ws_bytes, need)) return st;
  TCL_HIP(launch_delta_rule(op, d_state_out, d_o, ldo, static_cast<float*>(d_workspace),
                            static_cast<hipStream_t>(stream)));
  return TCL_OK;
}

TCL_API size_t tcl_delta_rule_backward_workspace_bytes(int32_t dtype, int32_t n_seq, int32_t rows, int32_t Hk,
                                                       int32_t H, int32_t Dk, int32_t Dv) {
  if ((dtype != TCL_F32 && dtype != TCL_BF16) || n_seq == 0 || !delta_sizes(n_seq, rows, Hk, H, Dk, Dv)) return 0;
  return delta_rule_bwd_workspace_bytes(dtype == TCL_BF16, n_seq, rows, Hk, H, Dk, Dv);
}

TCL_API tcl_status tcl_delta_rule_backward(const tcl_delta_rule_args* args, const void* d_do, int64_t lddo,
                                           const float* d_dstate_out, const tcl_delta_rule_grads* g,
                                           void* d_workspace, size_t ws_bytes, void* stream) {
  DeltaOp op;
  if (tcl_status st = delta_op(args, &op)) return st;
  if (!g) return fail(TCL_ERR_INVALID_ARG, "grads is NULL");
  const int64_t qk = (int64_t)op.Hk * op.Dk, v = (int64_t)op.H * op.Dv;
  if (lddo < v || g->lddq < qk || g->lddk < qk || g->lddv < v || g->lddg < op.H || g->lddbeta < op.H)
    return fail(TCL_ERR_INVALID_ARG, "leading dimension smaller than the row");
  if (lddo > kMaxLd || g->lddq > kMaxLd || g->lddk > kMaxLd || g->lddv > kMaxLd)
    return fail(TCL_ERR_UNSUPPORTED, "leading dimensions must be at most %lld", (long long)kMaxLd);
  if (op.rows > 0 && (!d_do || !g->d_dq || !g->d_dk || !g->d_dv || !g->d_dg || !g->d_dbeta))
    return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  const uintptr_t el = op.bf16 ? 2 : 4;
  if (misaligned(d_do, el) || misaligned(g->d_dq, el) || misaligned(g->d_dk, el) || misaligned(g->d_dv, el))
    return fail(TCL_ERR_INVALID_ARG, "activations are not aligned to their type");
  if (misaligned(d_dstate_out, 16) || misaligned(g->d_dstate, 16))
    return fail(TCL_ERR_INVALID_ARG, "the states' gradients must be 16-byte aligned");
  if ((int64_t)op.n_seq * op.H > kMaxSeqHeads)
    return fail(TCL_ERR_UNSUPPORTED, "too many sequences x heads (n_seq=%d H=%d)", op.n_seq, op.H);
  if (op.n_seq == 0) return fail(TCL_ERR_INVALID_ARG, "no sequences to take gradients of");
  op.n_slots = op.n_seq;
  const size_t need = delta_rule_bwd_workspace_bytes(op.bf16, op.n_seq, op.rows, op.Hk, op.H, op.Dk, op.Dv);
  if (tcl_status st = check_workspace(d_workspace, ws_bytes, need)) return st;
  DeltaGrads o;
  o.dq = g->d_dq; o.dk = g->d_dk; o.dv = g->d_dv; o.lddq = g->lddq; o.lddk = g->lddk; o.lddv = g->lddv;
  o.dg = g->d_dg; o.dbeta = g->d_dbeta; o.lddg = g->lddg; o.lddb = g->lddbeta; o.dstate = g->d_dstate;
  TCL_HIP(launch_delta_rule_bwd(op, d_do, lddo, d_dstate_out, o, static_cast<float*>(d_workspace),
                                static_cast<hipStream_t>(stream)));
  return TCL_OK;
}

// ------------------------------------------------------------------ beam search

namespace {

constexpr int kMaxBeams = 64, kMaxCandidates = 64;

bool beam_sizes(int32_t groups, int32_t W, int32_t V, int32_t K) {
  return groups >= 0 && W >= 1 && W <= kMaxBeams && (int64_t)groups * W <= kMaxLogitRows && V >= 1 && V <= (1 << 30) &&
         K >= 1 && K <= kMaxCandidates;
}

}  // namespace

TCL_API size_t tcl_beam_select_workspace_bytes(int32_t n_groups, int32_t W, int32_t V, int32_t K) {
  if (n_groups == 0 || !beam_sizes(n_groups, W, V, K)) return 0;
  return beam_select_workspace_bytes(n_groups, W, V, K);
}

TCL_API tcl_status tcl_beam_select(int32_t dtype, int32_t n_groups, int32_t W, int32_t V, const void* d_logits,
                                   int64_t ld, float temperature, const float* d_score, const int32_t* d_ended,
                                   int32_t K, int32_t* d_parent, int32_t* d_token, float* d_out_score,
                                   void* d_workspace, size_t ws_bytes, void* stream) {
  if (n_groups < 0 || W < 1) return fail(TCL_ERR_INVALID_ARG, "need n_groups >= 0, W > 0 (got %d, %d)", n_groups, W);
  if (W > kMaxBeams || K < 1 || K > kMaxCandidates)
    return fail(TCL_ERR_UNSUPPORTED, "W and K must be in [1, %d] and [1, %d] (got %d, %d)", kMaxBeams, kMaxCandidates, W,
                K);
  if ((int64_t)n_groups * W > kMaxLogitRows)
    return fail(TCL_ERR_UNSUPPORTED, "there must be fewer than 2^22 beams (got %d x %d)", n_groups, W);
  LogitRows a;
  if (tcl_status st = logit_rows(dtype, n_groups * W, V, d_logits, ld, nullptr, temperature, &a)) return st;
  if (n_groups == 0) return TCL_OK;
  if (!d_score || !d_parent || !d_token || !d_out_score) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  const size_t need = beam_select_workspace_bytes(n_groups, W, V, K);
  if (tcl_status st = check_workspace(d_workspace, ws_bytes, need)) return st;
  const size_t out = (size_t)n_groups * K * 4, in = (size_t)n_groups * W * 4;
  const Rows outs[] = {flat(d_parent, out), flat(d_token, out), flat(d_out_score, out)};
  const Rows ins[] = {flat(d_score, in), flat(d_ended, in), flat(d_workspace, need)};  // (what a group reads while others write)
  for (int i = 0; i < 3; ++i) {
    for (const Rows& b : ins)
      if (overlap(outs[i], b)) return fail(TCL_ERR_INVALID_ARG, "an output overlaps the scores, d_ended or the workspace");
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], outs[j])) return fail(TCL_ERR_INVALID_ARG, "outputs overlap each other");
  }
  TCL_HIP(launch_beam_select(a, W, K, d_score, d_ended, d_parent, d_token, d_out_score, d_workspace,
                             static_cast<hipStream_t>(stream)));
  return TCL_OK;
}

TCL_API tcl_status tcl_beam_reorder(int32_t n_groups, int32_t W, const int32_t* d_parent, const int32_t* d_slots,
                                    int32_t n_slots, int32_t* d_slots_out, int32_t n_pools,
                                    const tcl_beam_pool* pools, void* stream) {
  if (n_groups < 0 || W < 1 || n_slots < 0 || n_pools < 0)
    return fail(TCL_ERR_INVALID_ARG, "negative size (n_groups=%d W=%d n_slots=%d n_pools=%d)", n_groups, W, n_slots,
                n_pools);
  if (W > kMaxBeams) return fail(TCL_ERR_UNSUPPORTED, "W must be in [1, %d] (got %d)", kMaxBeams, W);
  if ((int64_t)n_groups * W > kMaxLogitRows)
    return fail(TCL_ERR_UNSUPPORTED, "there must be fewer than 2^22 beams (got %d x %d)", n_groups, W);
  if (n_pools > 0 && !pools) return fail(TCL_ERR_INVALID_ARG, "pools is NULL");
  for (int i = 0; i < n_pools; ++i) {
    if (pools[i].bytes < 1 || pools[i].bytes > ((int64_t)1 << 31))
      return fail(TCL_ERR_UNSUPPORTED, "pool %d: a state has 1 to 2^31 bytes (got %lld)", i, (long long)pools[i].bytes);
    if (!pools[i].d_states && n_slots > 0) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  }
  if (n_groups == 0) return TCL_OK;
  if (!d_parent || !d_slots || !d_slots_out) return fail(TCL_ERR_INVALID_ARG, "NULL device pointer");
  const size_t len = (size_t)n_groups * W * sizeof(int32_t);
  if (overlap(flat(d_slots_out, len), flat(d_slots, len)) || overlap(flat(d_slots_out, len), flat(d_parent, len)))
    return fail(TCL_ERR_INVALID_ARG, "d_slots_out overlaps an input");
  static_assert(sizeof(tcl_beam_pool) == sizeof(BeamPool), "one layout");
  TCL_HIP(launch_beam_reorder(n_groups, W, d_parent, d_slots, n_slots, d_slots_out, n_pools,
                              reinterpret_cast<const BeamPool*>(pools), static_cast<hipStream_t>(stream)));
  return TCL_OK;
}
