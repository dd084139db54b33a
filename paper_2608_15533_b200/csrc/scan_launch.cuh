// Host-side pieces of the scan's entry points: which tensors live where in the workspace, and the launch functions of
// its kernels (one translation unit each).
#pragma once

#include "launch_common.cuh"
#include "scan_common.cuh"

namespace deltalog {

// Byte offsets into the caller's workspace.
struct ScanLayout {
    size_t order, A, T, decay, qt, kt, kh, qi, ki, U, S, dV, dS, dq_part, dk_part, dbonus_part, pieces, total;
    int split;
};

// Segments that a row may be cut into: as many as leave every chain of the first pass an SM of its own, none for rows that
// are short for it.  One GDN row in segments against one chain, us with preparation: 8 heads, 1536 tokens 97 / 116, 4096 tokens
// 127 / 280, 16k tokens 303 / 1079; 32 heads 116 / 127, 244 / 308, 859 / 1185; 48 heads 127 / 131, 271 / 328, 934 / 1256.
// (n counts the plan's rows, those that decode among them, since the host knows no lengths: the 16k row of 32 heads takes 874 us by
// itself and 1210 among 47 decoding rows, where it runs as one chain.)
inline int scan_split(const deltalog_desc *d, int32_t n, int32_t max_tokens) {
    const long long units = (long long)n * d->H;
    if (d->d_v != 128 || units < 1 || units * scan_pieces(3) > kSplitCtas) return 1;
    return scan_segments(scan_max_chunks(n, max_tokens), ((int)(kSplitCtas / units) + 3) / 2);
}

inline ScanLayout scan_layout(const deltalog_desc *d, int32_t n, int32_t max_tokens, bool train) {
    const size_t H = d->H, Hq = d->H_qk > 0 ? d->H_qk : d->H, dk = d->d_k, dv = d->d_v, tok = max_tokens;
    const size_t units = (size_t)scan_max_chunks(n, max_tokens) * H;
    const bool vec = op_vec_decay(d->op), delta = op_delta_rule(d->op), f32 = d->io_dtype == DELTALOG_F32;
    size_t at = 0;
    auto take = [&](bool wanted, size_t bytes) {
        const size_t off = at;
        if (wanted) at += (bytes + 255) / 256 * 256;
        return off;
    };
    ScanLayout l;
    const size_t mats = units * kPlanes * kChunk * kChunk * 2, vecs = units * kPlanes * kChunk * dk * 2, vals = units * kChunk * dv * 4;
    l.order = take(true, (size_t)n * 4);
    l.A = take(true, mats);
    l.T = take(delta, mats);
    l.decay = take(true, units * (vec ? dk : 2 * kChunk) * 4);
    l.qt = take(vec, vecs);
    l.kt = take(vec && delta, vecs);
    l.kh = take(vec, vecs);
    const size_t raw = (size_t)scan_max_chunks(n, max_tokens) * Hq * kPlanes * kChunk * dk * 2;
    l.qi = take(f32 && !vec, raw);
    l.ki = take(f32 && !vec, raw);
    l.U = take(train && delta, vals);
    l.S = take(train, units * dk * dv * 4);
    l.dV = take(train && delta, vals);
    l.dS = take(train, units * dk * dv * 4);
    l.dq_part = take(train && H != Hq, tok * H * dk * 4);
    l.dk_part = take(train && H != Hq, tok * H * dk * 4);
    l.dbonus_part = take(train && d->op == DELTALOG_RWKV6, units * dk * 4);
    l.split = scan_split(d, n, max_tokens);
    // (one tile per CTA of the first pass at most, whether or not these rows are cut: fewer rows might be, and a workspace
    // for more rows has to do for them)
    const bool may_cut = dv == 128 && (long long)H * scan_pieces(3) <= kSplitCtas && scan_max_chunks(n, max_tokens) >= 3 * kMinSegment;
    l.pieces = take(may_cut, (size_t)kSplitCtas * dk * dv * 4);
    l.total = at;
    return l;
}

// SCAN_SHAPES(desc, CALL): CALL(VEC, P, DK, DELTA, IO) for the chain kernels
#define DELTALOG_SCAN_DK(d, CALL, VEC, P, DELTA, IO)              \
    do {                                                          \
        if ((d)->d_k == 128) { CALL(VEC, P, 128, DELTA, IO); }    \
        else { CALL(VEC, P, 64, DELTA, IO); }                     \
    } while (0)
#define DELTALOG_SCAN_IO(d, CALL, VEC, DELTA)                                                                          \
    do {                                                                                                               \
        if ((d)->io_dtype == DELTALOG_F32) DELTALOG_SCAN_DK(d, CALL, VEC, 3, DELTA, float);                             \
        else DELTALOG_SCAN_DK(d, CALL, VEC, 1, DELTA, __nv_bfloat16);                                                  \
    } while (0)
#define DELTALOG_SCAN_DISPATCH(d, CALL)                                              \
    do {                                                                             \
        if (op_vec_decay((d)->op)) {                                                 \
            if (op_delta_rule((d)->op)) DELTALOG_SCAN_IO(d, CALL, true, true);        \
            else DELTALOG_SCAN_IO(d, CALL, true, false);                             \
        } else {                                                                     \
            if (op_delta_rule((d)->op)) DELTALOG_SCAN_IO(d, CALL, false, true);       \
            else DELTALOG_SCAN_IO(d, CALL, false, false);                            \
        }                                                                            \
    } while (0)

// Warps (16 columns of d_v = 64 each) of a CTA of the mma.sync chains.  The warps of a CTA share the loads of q, k, A and T; a
// unit spread over two CTAs reads them again, from L2.  While the units do not fill the device, smaller CTAs put it to work on
// more SMs.
inline int scan_chain_warps(int units) { return units < device_info().sms ? 2 : 4; }

int launch_scan_prep(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s);
int launch_scan_forward(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s);
int launch_scan_forward_tc(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s);
int launch_scan_backward(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s);
int launch_scan_backward_tc(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s);
int launch_scan_grad(const deltalog_desc *d, const ScanArgs &a, int rows, float *dbonus, cudaStream_t s);

}  // namespace deltalog
