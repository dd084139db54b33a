// deltalog_head_norm_*: argument checks, grids, launches.
#include <cmath>

#include "headnorm_kernel.cuh"
#include "launch_common.cuh"
#include "validate.h"

using namespace deltalog;

namespace {

int validate_norm_desc(const deltalog_norm_desc *d) {
    if (!d || d->H_q <= 0 || d->H_k < 0 || (d->io_dtype != DELTALOG_F32 && d->io_dtype != DELTALOG_BF16)) return DELTALOG_ERR_INVALID_ARG;
    if (d->norm < DELTALOG_NORM_L2 || d->norm > DELTALOG_NORM_NONE || !(d->eps >= 0.f) || !std::isfinite(d->q_scale)) return DELTALOG_ERR_INVALID_ARG;
    if (d->d <= 0 || d->d % 8 || d->d > 256 || d->rot < 0 || d->rot > d->d || d->rot % 16) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    // (a head index times d has to fit an int)
    if ((long long)d->H_q * d->d > 0x3fffffffll || (long long)d->H_k * d->d > 0x3fffffffll) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    return DELTALOG_OK;
}

int validate_norm(const deltalog_norm_desc *d, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const float *w_q, const float *w_k,
                  const float *cos, const float *sin, const int32_t *positions, int32_t tokens) {
    if (int rc = validate_norm_desc(d)) return rc;
    const int vec = d->io_dtype == DELTALOG_F32 ? 4 : 8;
    if (tokens < 0 || !q || !aligned16(q) || q_stride < (long long)d->H_q * d->d || q_stride % vec) return DELTALOG_ERR_INVALID_ARG;
    if (d->H_k && (!k || !aligned16(k) || k_stride < (long long)d->H_k * d->d || k_stride % vec)) return DELTALOG_ERR_INVALID_ARG;
    if (w_q && d->norm != DELTALOG_NORM_RMS) return DELTALOG_ERR_INVALID_ARG;
    if (d->H_k ? !w_q != !w_k : w_k != nullptr) return DELTALOG_ERR_INVALID_ARG;
    if (!aligned16(w_q) || !aligned16(w_k)) return DELTALOG_ERR_INVALID_ARG;
    if (d->rot && (!cos || !sin || !positions || !aligned16(cos) || !aligned16(sin) || d->table_rows <= 0)) return DELTALOG_ERR_INVALID_ARG;
    return DELTALOG_OK;
}

NormArgs norm_args(const deltalog_norm_desc *d, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const float *w_q, const float *w_k,
                   const float *cos, const float *sin, const int32_t *positions, int32_t tokens) {
    NormArgs a = {};
    a.q = q, a.k = k, a.q_stride = q_stride, a.k_stride = k_stride, a.w_q = w_q, a.w_k = w_k, a.cos = cos, a.sin = sin, a.positions = positions;
    a.tokens = tokens, a.H_q = d->H_q, a.H_k = d->H_k, a.d = d->d, a.norm = d->norm, a.rot = d->rot, a.interleaved = d->interleaved != 0;
    a.table_rows = d->table_rows, a.eps = d->eps, a.q_scale = d->q_scale;
    return a;
}

int norm_lanes(int d) { return d <= 32 ? 2 : d <= 64 ? 4 : d <= 128 ? 8 : 16; }

template <int HEADS>
long long norm_blocks(const deltalog_norm_desc *d, int32_t tokens) {
    const int L = norm_lanes(d->d);
    auto items = [&](int heads) {
        return L == 2 ? norm_items<2, HEADS>(tokens, heads) : L == 4 ? norm_items<4, HEADS>(tokens, heads)
             : L == 8 ? norm_items<8, HEADS>(tokens, heads) : norm_items<16, HEADS>(tokens, heads);
    };
    return (items(d->H_q) + items(d->H_k) + kNormThreads / 32 - 1) / (kNormThreads / 32);
}

// One wave of blocks, which walk over the items (of 148 SMs, whichever device is current: with weights the backward pass keeps a
// block's sums, and the workspace's size depends on it).
long long norm_wave(long long blocks, int per_sm) { return blocks < 148 * per_sm ? blocks : 148 * per_sm; }
long long norm_kept_blocks(const deltalog_norm_desc *d, int32_t tokens) {
    return norm_wave(norm_blocks<kNormHeadsBack>(d, tokens), d->io_dtype == DELTALOG_F32 ? kNormBackCtas<float> : kNormBackCtas<__nv_bfloat16>);
}

#define NORM_DISPATCH(desc_, CALL)                                                                  \
    do {                                                                                            \
        const int l_ = norm_lanes((desc_)->d);                                                      \
        if ((desc_)->io_dtype == DELTALOG_F32) { NORM_LANES(float, l_, CALL); }                     \
        else { NORM_LANES(__nv_bfloat16, l_, CALL); }                                               \
    } while (0)
#define NORM_LANES(IO, l_, CALL) \
    if (l_ == 2) { CALL(IO, 2); } else if (l_ == 4) { CALL(IO, 4); } else if (l_ == 8) { CALL(IO, 8); } else { CALL(IO, 16); }

}  // namespace

extern "C" {

int deltalog_head_norm_forward(const deltalog_norm_desc *desc, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const float *w_q,
                               const float *w_k, const float *cos, const float *sin, const int32_t *positions, int32_t tokens, void *out_q,
                               void *out_k, int32_t *status, void *stream) {
    if (int rc = validate_norm(desc, q, q_stride, k, k_stride, w_q, w_k, cos, sin, positions, tokens)) return rc;
    if (!out_q || !aligned16(out_q) || (desc->H_k && (!out_k || !aligned16(out_k)))) return DELTALOG_ERR_INVALID_ARG;
    if (tokens == 0) return DELTALOG_OK;
    NormArgs a = norm_args(desc, q, q_stride, k, k_stride, w_q, w_k, cos, sin, positions, tokens);
    a.out_q = out_q, a.out_k = out_k, a.status = status;
    const long long blocks = norm_blocks<kNormHeads>(desc, tokens);
    const long long grid = norm_wave(blocks, desc->io_dtype == DELTALOG_F32 ? kNormCtas<float> : kNormCtas<__nv_bfloat16>);
    if (blocks > 0x1fffffffll) return DELTALOG_ERR_UNSUPPORTED_SHAPE;  // items are counted in 31 bits
    cudaStream_t s = static_cast<cudaStream_t>(stream);
#define CALL(IO, L) head_norm_forward_kernel<IO, L><<<(unsigned)grid, kNormThreads, 0, s>>>(a)
    NORM_DISPATCH(desc, CALL);
#undef CALL
    return finish_launch();
}

size_t deltalog_head_norm_workspace_bytes(const deltalog_norm_desc *desc, int32_t tokens) {
    if (validate_norm_desc(desc) || desc->norm != DELTALOG_NORM_RMS || tokens < 0) return 0;
    return (size_t)norm_kept_blocks(desc, tokens) * 2 * desc->d * sizeof(float);
}

int deltalog_head_norm_backward(const deltalog_norm_desc *desc, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const float *w_q,
                                const float *w_k, const float *cos, const float *sin, const int32_t *positions, int32_t tokens,
                                const void *dout_q, const void *dout_k, void *dq, void *dk, float *dw_q, float *dw_k, void *workspace,
                                size_t workspace_bytes, void *stream) {
    if (int rc = validate_norm(desc, q, q_stride, k, k_stride, w_q, w_k, cos, sin, positions, tokens)) return rc;
    if (!dout_q || !dq || !aligned16(dout_q) || !aligned16(dq)) return DELTALOG_ERR_INVALID_ARG;
    if (desc->H_k && (!dout_k || !dk || !aligned16(dout_k) || !aligned16(dk))) return DELTALOG_ERR_INVALID_ARG;
    const bool weighted = w_q != nullptr;
    if (weighted && (!dw_q || (desc->H_k && !dw_k))) return DELTALOG_ERR_INVALID_ARG;
    if (weighted && tokens && (!workspace || !aligned16(workspace) || workspace_bytes < deltalog_head_norm_workspace_bytes(desc, tokens)))
        return DELTALOG_ERR_INVALID_ARG;
    NormArgs a = norm_args(desc, q, q_stride, k, k_stride, w_q, w_k, cos, sin, positions, tokens);
    a.out_q = dq, a.out_k = dk, a.dout_q = dout_q, a.dout_k = dout_k, a.partial = static_cast<float *>(workspace);
    const long long grid = norm_kept_blocks(desc, tokens);
    if (norm_blocks<kNormHeadsBack>(desc, tokens) > 0x1fffffffll) return DELTALOG_ERR_UNSUPPORTED_SHAPE;  // items are counted in 31 bits
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (grid > 0) {
#define CALL(IO, L) head_norm_backward_kernel<IO, L><<<(unsigned)grid, kNormThreads, 0, s>>>(a)
        NORM_DISPATCH(desc, CALL);
#undef CALL
        if (int rc = finish_launch()) return rc;
    }
    if (!weighted) return DELTALOG_OK;
    head_norm_reduce_kernel<<<(2 * desc->d + 31) / 32, 256, 0, s>>>(a.partial, (int)grid, desc->d, dw_q, dw_k);
    return finish_launch();
}

}  // extern "C"
