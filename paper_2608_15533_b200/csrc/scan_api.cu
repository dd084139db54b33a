// C ABI of the scan over packed sequences: argument checks, workspace layout, launches in order.
// Declarations and the contract of every entry point are in include/deltalog.h.
#include "scan_launch.cuh"

using namespace deltalog;

namespace {

// The checks that every scan entry point shares; nothing is launched before they pass.
int validate_scan(const deltalog_desc *d, const deltalog_plan *plan, const void *q, const void *k, const void *v, const float *g, const float *beta,
                  const float *u_bonus, const void *workspace, size_t workspace_bytes, bool train) {
    if (int rc = validate_desc(d)) return rc;
    if (int rc = validate_plan(plan)) return rc;
    if (int rc = validate_token(d, q, k, v, g, beta, u_bonus, plan->n, q)) return rc;
    if ((long long)plan->n * d->H > 0x7fffffffll || d->H > 65535) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    if (plan->n == 0) return DELTALOG_OK;
    const ScanLayout l = scan_layout(d, plan->n, plan->max_tokens, train);
    if (!workspace || !aligned16(workspace) || workspace_bytes < l.total) return DELTALOG_ERR_INVALID_ARG;
    return DELTALOG_OK;
}

ScanArgs scan_args(const deltalog_desc *d, const deltalog_plan *plan, const void *q, const void *k, const void *v, const float *g, const float *beta,
                   const float *u_bonus, void *workspace, const ScanLayout &l) {
    ScanArgs a = {};
    a.starts = plan->starts, a.chunk_starts = plan->chunk_starts, a.chunk_seq = plan->chunk_seq;
    a.n = plan->n, a.max_chunks = scan_max_chunks(plan->n, plan->max_tokens), a.max_tokens = plan->max_tokens, a.num_slots = d->num_slots, a.status = plan->status;
    a.H = d->H, a.Hq = d->H_qk > 0 ? d->H_qk : d->H, a.dv = d->d_v;
    a.scale = d->op == DELTALOG_RWKV6 ? 1.f : d->scale;
    a.q = q, a.k = k, a.v = v;
    a.g = op_has_gate(d->op) ? g : nullptr, a.beta = beta, a.bonus = u_bonus;
    char *w = static_cast<char *>(workspace);
    auto plane = [&](size_t off) { return reinterpret_cast<__nv_bfloat16 *>(w + off); };
    a.A = plane(l.A), a.T = plane(l.T), a.qt = plane(l.qt), a.kt = plane(l.kt), a.kh = plane(l.kh);
    auto floats = [&](size_t off) { return reinterpret_cast<float *>(w + off); };
    a.U = floats(l.U), a.S = floats(l.S), a.dV = floats(l.dV), a.dS = floats(l.dS), a.decay = floats(l.decay);
    a.dq_part = floats(l.dq_part), a.dk_part = floats(l.dk_part), a.dbonus_part = floats(l.dbonus_part);
    a.order = reinterpret_cast<int32_t *>(w + l.order);
    a.qi = plane(l.qi), a.ki = plane(l.ki);
    a.split = l.split, a.pieces = floats(l.pieces);
    return a;
}

// The chunks' matrices and operands, then the chain.
int run_forward(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s) {
    if (int rc = launch_scan_prep(d, a, s)) return rc;
    return launch_scan_forward(d, a, s);
}

}  // namespace

extern "C" {

size_t deltalog_scan_workspace_bytes(const deltalog_desc *desc, int32_t n, int32_t max_tokens, int32_t train) {
    if (validate_desc(desc) || n < 0 || max_tokens < 0) return 0;
    return scan_layout(desc, n, max_tokens, train != 0).total;
}

int deltalog_prefill(const deltalog_desc *desc, const deltalog_state *state, const deltalog_plan *plan, const void *q, const void *k, const void *v,
                     const float *g, const float *beta, const float *u_bonus, const int32_t *fresh, void *out, void *workspace,
                     size_t workspace_bytes, void *stream) {
    if (int rc = validate_scan(desc, plan, q, k, v, g, beta, u_bonus, workspace, workspace_bytes, false)) return rc;
    if (int rc = validate_state(state)) return rc;
    if (!out || !aligned16(out)) return DELTALOG_ERR_INVALID_ARG;
    if (plan->n == 0) return DELTALOG_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // entries that are pending in the logs of the listed slots belong in front of the new tokens
    if (int rc = deltalog_merge(desc, state, plan->scan_slots, plan->n, 0, stream)) return rc;
    ScanArgs a = scan_args(desc, plan, q, k, v, g, beta, u_bonus, workspace, scan_layout(desc, plan->n, plan->max_tokens, false));
    a.slots = plan->scan_slots, a.status = state->status;
    a.S_in = a.S_out = state->S_base;
    a.in_bf16 = a.out_bf16 = desc->base_dtype == DELTALOG_BF16;
    a.fresh = fresh, a.log_len = state->log_len, a.out = out;
    a.clear = (desc->hints & DELTALOG_HINT_ZERO_UNWRITTEN) != 0;
    return run_forward(desc, a, s);
}

int deltalog_scan_forward(const deltalog_desc *desc, const deltalog_plan *plan, const float *S_init, const void *q, const void *k, const void *v,
                          const float *g, const float *beta, const float *u_bonus, void *out, float *S_final, int32_t save, void *workspace,
                          size_t workspace_bytes, void *stream) {
    if (int rc = validate_scan(desc, plan, q, k, v, g, beta, u_bonus, workspace, workspace_bytes, save != 0)) return rc;
    if (!out || !aligned16(out)) return DELTALOG_ERR_INVALID_ARG;
    if (plan->n == 0) return DELTALOG_OK;
    ScanArgs a = scan_args(desc, plan, q, k, v, g, beta, u_bonus, workspace, scan_layout(desc, plan->n, plan->max_tokens, save != 0));
    a.S_in = S_init, a.S_out = S_final, a.out = out, a.keep = save != 0;
    a.clear = (desc->hints & DELTALOG_HINT_ZERO_UNWRITTEN) != 0;
    return run_forward(desc, a, static_cast<cudaStream_t>(stream));
}

int deltalog_scan_backward(const deltalog_desc *desc, const deltalog_plan *plan, const float *S_init, const void *q, const void *k, const void *v,
                           const float *g, const float *beta, const float *u_bonus, const void *dout, const float *dS_final, int32_t saved,
                           const deltalog_scan_grads *grads, int32_t rows, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = validate_scan(desc, plan, q, k, v, g, beta, u_bonus, workspace, workspace_bytes, true)) return rc;
    if (!dout || !aligned16(dout) || !grads || !grads->q || !grads->k || !grads->v || rows < plan->max_tokens) return DELTALOG_ERR_INVALID_ARG;
    if (!aligned16(grads->q) || !aligned16(grads->k) || !aligned16(grads->v)) return DELTALOG_ERR_INVALID_ARG;
    if ((op_has_gate(desc->op) && !grads->g) || (op_delta_rule(desc->op) && !grads->beta) || (desc->op == DELTALOG_RWKV6 && !grads->u_bonus))
        return DELTALOG_ERR_INVALID_ARG;
    if (plan->n == 0) return DELTALOG_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    ScanArgs a = scan_args(desc, plan, q, k, v, g, beta, u_bonus, workspace, scan_layout(desc, plan->n, plan->max_tokens, true));
    if (!saved) {
        a.S_in = S_init, a.keep = 1;
        if (int rc = run_forward(desc, a, s)) return rc;
    }
    a.dout = dout;
    a.dS_final = dS_final, a.dS_init = grads->S_init;
    a.dq = grads->q, a.dk = grads->k, a.dv_out = grads->v;
    a.dg = op_has_gate(desc->op) ? grads->g : nullptr;
    a.dbeta = op_delta_rule(desc->op) ? grads->beta : nullptr;
    if (int rc = launch_scan_backward(desc, a, s)) return rc;
    return launch_scan_grad(desc, a, rows, grads->u_bonus, s);
}

}  // extern "C"
