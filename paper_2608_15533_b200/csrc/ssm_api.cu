// C ABI of the selective state space scan: argument checks, workspace layout, launches in order.
#include "ssm_launch.cuh"

using namespace deltalog;

namespace {

int validate_ssm_desc(const deltalog_ssm_desc *d) {
    if (!d || d->channels <= 0 || d->groups <= 0 || (d->io_dtype != DELTALOG_F32 && d->io_dtype != DELTALOG_BF16)) return DELTALOG_ERR_INVALID_ARG;
    if (d->d_state != 8 && d->d_state != 16 && d->d_state != 32 && d->d_state != 64) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    if (d->channels % d->groups || (d->channels / d->groups) % 8) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    if ((long long)d->channels * d->d_state > 0x3fffffffll) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    return DELTALOG_OK;
}

int validate_ssm(const deltalog_ssm_desc *d, const deltalog_ssm_inputs *in) {
    if (int rc = validate_ssm_desc(d)) return rc;
    if (!in || !in->x || !in->dt || !in->A || !in->B || !in->C) return DELTALOG_ERR_INVALID_ARG;
    const int vec = d->io_dtype == DELTALOG_F32 ? 4 : 8;
    const long long states = (long long)d->groups * d->d_state;
    auto tokens_ok = [&](const void *p, long long stride, long long width) { return aligned16(p) && stride >= width && stride % vec == 0; };
    auto too_wide = [](long long stride) { return stride > (1 << 25); };  // a tile's offsets are kept in 32 bits
    if (!tokens_ok(in->x, in->x_stride, d->channels) || !tokens_ok(in->dt, in->dt_stride, d->channels) ||
        !tokens_ok(in->B, in->B_stride, states) || !tokens_ok(in->C, in->C_stride, states) || (in->z && !tokens_ok(in->z, in->z_stride, d->channels)))
        return DELTALOG_ERR_INVALID_ARG;
    if (too_wide(in->x_stride) || too_wide(in->dt_stride) || too_wide(in->B_stride) || too_wide(in->C_stride) || (in->z && too_wide(in->z_stride)))
        return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    if (!aligned16(in->A) || !aligned16(in->D) || !aligned16(in->dt_bias)) return DELTALOG_ERR_INVALID_ARG;
    return DELTALOG_OK;
}

constexpr int32_t kMostTokens = 1 << 30;  // (a stretch is rounded up, and its end has to fit an int)

int validate_room(const deltalog_ssm_desc *d, int32_t tokens, bool train, const void *workspace, size_t bytes) {
    if (tokens > kMostTokens) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    if (!workspace || !aligned16(workspace) || bytes < ssm_layout(d, tokens, train).total) return DELTALOG_ERR_INVALID_ARG;
    return DELTALOG_OK;
}

SsmArgs ssm_args(const deltalog_ssm_desc *d, const deltalog_ssm_inputs *in) {
    SsmArgs a = {};
    a.x = in->x, a.dt = in->dt, a.B = in->B, a.C = in->C, a.z = in->z;
    a.x_stride = in->x_stride, a.dt_stride = in->dt_stride, a.B_stride = in->B_stride, a.C_stride = in->C_stride, a.z_stride = in->z_stride;
    a.A = in->A, a.D = in->D, a.bias = in->dt_bias;
    a.D_ = d->channels, a.G = d->groups, a.num_slots = d->num_slots, a.softplus = d->softplus != 0;
    return a;
}

// The forward pass over a plan's tokens, its workspace laid out for `room` tokens.
void ssm_forward_args(const deltalog_ssm_desc *d, const deltalog_plan *p, int32_t room, bool train, void *workspace, SsmArgs &a) {
    a.rows = Rows{p->starts, p->token_seq, p->n};
    a.max_tokens = p->max_tokens;
    const SsmForm form = ssm_forward_form(d, p->n, p->max_tokens);
    const SsmCut c = ssm_cut(d, p->n, p->max_tokens, form);
    a.span = c.span, a.spans = c.spans, a.part = c.part, a.parts = c.parts, a.blocks = c.blocks, a.wide = form == kSsmWide;
    const SsmLayout l = ssm_layout(d, room, train);
    char *w = static_cast<char *>(workspace);
    auto floats = [&](size_t off) { return reinterpret_cast<float *>(w + off); };
    a.local = floats(l.local), a.sums = floats(l.sums);
}

}  // namespace

extern "C" {

int deltalog_ssm_step(const deltalog_ssm_desc *desc, float *S, const deltalog_ssm_inputs *in, const int32_t *slot_idx, int32_t B, void *out,
                      int32_t *status, void *stream) {
    if (int rc = validate_ssm(desc, in)) return rc;
    if (desc->num_slots <= 0 || B < 0 || !S || !out || !aligned16(S) || !aligned16(out)) return DELTALOG_ERR_INVALID_ARG;
    if (!slot_idx && B > desc->num_slots) return DELTALOG_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(S) % 32 || reinterpret_cast<uintptr_t>(in->A) % 32) return DELTALOG_ERR_INVALID_ARG;  // 32-byte accesses
    if (B == 0) return DELTALOG_OK;
    SsmArgs a = ssm_args(desc, in);
    a.S_in = S, a.S_out = S, a.slots = slot_idx, a.out = out, a.status = status, a.total_rows = B;
    return launch_ssm_step(desc, a, static_cast<cudaStream_t>(stream));
}

size_t deltalog_ssm_workspace_bytes(const deltalog_ssm_desc *desc, int32_t n, int32_t max_tokens, int32_t train) {
    if (validate_ssm_desc(desc) || n < 0 || max_tokens < 0 || max_tokens > kMostTokens) return 0;
    return ssm_layout(desc, max_tokens, train != 0).total;
}

int deltalog_ssm_prefill(const deltalog_ssm_desc *desc, float *S, const deltalog_plan *plan, const deltalog_ssm_inputs *in, const int32_t *fresh,
                         void *out, int32_t *status, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = validate_ssm(desc, in)) return rc;
    if (int rc = validate_plan(plan)) return rc;
    if (desc->num_slots <= 0 || !S || !out || !aligned16(S) || !aligned16(out)) return DELTALOG_ERR_INVALID_ARG;
    if (int rc = validate_room(desc, plan->max_tokens, false, workspace, workspace_bytes)) return rc;
    if (plan->n == 0) return DELTALOG_OK;
    SsmArgs a = ssm_args(desc, in);
    ssm_forward_args(desc, plan, plan->max_tokens, false, workspace, a);
    if (a.spans > 1) a.front = reinterpret_cast<float *>(static_cast<char *>(workspace) + ssm_layout(desc, plan->max_tokens, false).front);
    a.S_in = S, a.S_out = S, a.slots = plan->scan_slots, a.fresh = fresh, a.out = out, a.status = status;
    a.clear = (desc->hints & DELTALOG_HINT_ZERO_UNWRITTEN) != 0;
    return launch_ssm_forward(desc, a, static_cast<cudaStream_t>(stream));
}

int deltalog_ssm_forward(const deltalog_ssm_desc *desc, const deltalog_plan *plan, const float *S_init, const deltalog_ssm_inputs *in, void *out,
                         float *S_final, int32_t save, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = validate_ssm(desc, in)) return rc;
    if (int rc = validate_plan(plan)) return rc;
    if (!out || !aligned16(out) || !aligned16(S_init) || !aligned16(S_final)) return DELTALOG_ERR_INVALID_ARG;
    if (int rc = validate_room(desc, plan->max_tokens, save != 0, workspace, workspace_bytes)) return rc;
    if (plan->n == 0) return DELTALOG_OK;
    SsmArgs a = ssm_args(desc, in);
    ssm_forward_args(desc, plan, plan->max_tokens, save != 0, workspace, a);
    if (save) a.kept = static_cast<float *>(workspace);  // in front of everything else, whatever the workspace has room for
    a.S_in = S_init, a.S_out = S_final, a.out = out;
    a.clear = (desc->hints & DELTALOG_HINT_ZERO_UNWRITTEN) != 0;
    return launch_ssm_forward(desc, a, static_cast<cudaStream_t>(stream));
}

int deltalog_ssm_backward(const deltalog_ssm_desc *desc, const deltalog_plan *plan, const float *S_init, const deltalog_ssm_inputs *in,
                          const void *dout, const float *dS_final, int32_t saved, const deltalog_ssm_grads *grads, int32_t rows, void *workspace,
                          size_t workspace_bytes, void *stream) {
    if (int rc = validate_ssm(desc, in)) return rc;
    if (int rc = validate_plan(plan)) return rc;
    if (!dout || !aligned16(dout) || !aligned16(S_init) || !aligned16(dS_final) || !grads || rows < plan->max_tokens) return DELTALOG_ERR_INVALID_ARG;
    if (!grads->x || !grads->dt || !grads->B || !grads->C || !grads->A || (in->z && !grads->z) || (in->D && !grads->D) || (in->dt_bias && !grads->dt_bias))
        return DELTALOG_ERR_INVALID_ARG;
    if (!aligned16(grads->x) || !aligned16(grads->dt) || !aligned16(grads->z) || !aligned16(grads->S_init)) return DELTALOG_ERR_INVALID_ARG;
    if (int rc = validate_room(desc, rows, true, workspace, workspace_bytes)) return rc;
    if (plan->n == 0) return DELTALOG_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    SsmArgs a = ssm_args(desc, in);
    // the forward pass's share is laid out behind the kept states of `rows` tokens, of which it writes plan->max_tokens' worth
    ssm_forward_args(desc, plan, rows, true, workspace, a);
    a.S_in = S_init;
    a.kept = static_cast<float *>(workspace);
    if (!saved)
        if (int rc = launch_ssm_forward(desc, a, s)) return rc;
    const SsmLayout l = ssm_layout(desc, rows, true);
    char *w = static_cast<char *>(workspace);
    auto floats = [&](size_t off) { return reinterpret_cast<float *>(w + off); };
    const SsmCut c = ssm_cut(desc, plan->n, rows, kSsmBack);
    a.span = c.span, a.spans = c.spans, a.part = c.part, a.parts = c.parts, a.blocks = c.blocks, a.total_rows = rows;
    a.part_bc = floats(l.part_bc), a.part_A = floats(l.part_A), a.part_cols = floats(l.part_cols);
    a.dout = dout, a.dS_final = dS_final;
    a.dx = grads->x, a.ddt = grads->dt, a.dB = grads->B, a.dC = grads->C, a.dz = in->z ? grads->z : nullptr;
    a.dA = grads->A, a.dD = in->D ? grads->D : nullptr, a.dbias = in->dt_bias ? grads->dt_bias : nullptr, a.dS_init = grads->S_init;
    return launch_ssm_backward(desc, a, s);
}

}  // extern "C"
