// Host-side pieces of the state space scan's entry points: how the tokens are cut, which tensors live where in the workspace,
// and the launch functions of its kernels (one translation unit per direction).
#pragma once

#include "launch_common.cuh"
#include "ssm_join_kernel.cuh"

namespace deltalog {

inline long long ssm_ceil(long long a, long long b) { return (a + b - 1) / b; }

constexpr int kSsmSpanMin = 128;  // tokens of a stretch at least
constexpr int kSsmParts = 2;          // parts of a stretch in the first pass: the stretches alone would leave it a wave with gaps

// How the forward pass (`wide` or not) or the backward pass cuts channels into blocks and tokens into stretches.
enum SsmForm { kSsmWide, kSsmNarrow, kSsmBack };
inline int ssm_blocks(const deltalog_ssm_desc *d, SsmForm form) {
    const int n = d->d_state, wide = n == 8 ? 128 : n == 16 ? 64 : 32;  // channels of a CTA
    return (int)ssm_ceil(d->channels / d->groups, form == kSsmWide || (form == kSsmBack && n != 64) ? wide : wide / 2);
}

// CTAs of a form that an SM holds (the launches assert that it is what the kernels' shared memory and registers leave).  With four, and
// three backward, for all, a wave was one and a half of what fits with fp32 or 8 states.  fp32, 8k tokens in 4 rows x 4096 channels,
// then 4k in 9 rows x 2560, four for all / as here, us: 8 states 595 / 548, 202 / 118; 16 476 / 478, 185 / 198; 32 636 / 679, 288 / 236;
// 64 1326 / 927, 437 / 472; gradients 1019 / 986, 347 / 327; 1033 / 1071, 380 / 344; 1609 / 1609, 540 / 570; 3721 / 3333, 1222 / 1121.
constexpr int ssm_on_sm(bool fp32, int states, SsmForm form) {
    switch (states) {
    case 8: return form == kSsmNarrow ? (fp32 ? 3 : 4) : fp32 ? 1 : 2;
    case 16: return form == kSsmNarrow ? 4 : form == kSsmBack ? (fp32 ? 2 : 3) : fp32 ? 2 : 4;
    case 32: return form == kSsmNarrow ? 4 : form == kSsmBack ? 3 : fp32 ? 3 : 4;
    default: return form != kSsmNarrow && fp32 ? 2 : 3;
    }
}

// Stretches that the tokens are cut into at most: as many as one wave of CTAs has, or two or three waves where those are filled
// better by more than a twentieth (a cut makes the row that crosses it run twice behind its last border; of few blocks of
// channels one wave may leave an SM in seven idle).  (148 SMs whatever the device: workspaces depend on it.)
inline int ssm_most_spans(const deltalog_ssm_desc *d, SsmForm form) {
    const int blocks = ssm_blocks(d, form) * d->groups, wave = 148 * ssm_on_sm(d->io_dtype == DELTALOG_F32, d->d_state, form);
    if (blocks >= wave) return 1;
    int best = wave / blocks;
    double full = (double)best * blocks / wave;
    for (int waves = 2; waves <= 3; ++waves) {
        const int spans = waves * wave / blocks;
        if ((double)spans * blocks / (waves * wave) > 1.05 * full) best = spans, full = (double)spans * blocks / (waves * wave);
    }
    return best;
}
struct SsmCut { int span, spans, part, parts, blocks; };
inline SsmCut ssm_cut(const deltalog_ssm_desc *d, int32_t rows, int32_t tokens, SsmForm form) {
    long long span = ssm_ceil(tokens, ssm_most_spans(d, form)), round = kSsmSpanMin;
    // (documents of round lengths end where stretches of round lengths do, which then need no first pass: up to an eighth more)
    while (round < span) round *= 2;
    if (span < kSsmSpanMin || (rows > 1 && round - span <= span / 8)) span = round;
    const long long part = ssm_ceil(span, 32 * kSsmParts) * 32;
    SsmCut c;
    c.part = (int)part, c.span = (int)(part * kSsmParts);
    c.spans = (int)ssm_ceil(tokens, c.span), c.parts = (int)ssm_ceil(tokens, c.part), c.blocks = ssm_blocks(d, form);
    return c;
}
// Narrow where the wide form would leave SMs without a CTA.
inline SsmForm ssm_forward_form(const deltalog_ssm_desc *d, int32_t rows, int32_t tokens) {
    const SsmCut c = ssm_cut(d, rows, tokens, kSsmWide);
    return (long long)c.spans * c.blocks * d->groups < 148 ? kSsmNarrow : kSsmWide;
}
// What ssm_cut gives at most for this many tokens or fewer, in whichever form.
inline int ssm_room(const deltalog_ssm_desc *d, int32_t tokens, bool backward) {
    const long long wide = ssm_most_spans(d, backward ? kSsmBack : kSsmWide), narrow = backward ? 1 : ssm_most_spans(d, kSsmNarrow);
    const long long most = wide > narrow ? wide : narrow, spans = ssm_ceil(tokens, kSsmSpanMin);
    return (int)(spans < most ? spans : most);
}

// Byte offsets into the caller's workspace.
struct SsmLayout {
    size_t kept, local, front, sums, part_bc, part_A, part_cols, total;
};
inline SsmLayout ssm_layout(const deltalog_ssm_desc *d, int32_t tokens, bool train) {
    const size_t D = d->channels, N = d->d_state;
    size_t at = 0;
    auto take = [&](bool wanted, size_t bytes) {
        const size_t off = at;
        if (wanted) at += (bytes + 255) / 256 * 256;
        return off;
    };
    SsmLayout l;
    const int f = ssm_room(d, tokens, false), b = train ? ssm_room(d, tokens, true) : 0, joined = kSsmParts * (f > b ? f : b);
    l.kept = take(train, (size_t)ssm_ceil(tokens, kSsmBlock) * D * N * 4);
    l.local = take(f > 1 || b > 1, (size_t)joined * D * N * 4);
    l.front = take(f > 1 && !train, (size_t)kSsmParts * f * D * N * 4);
    l.sums = take(f > 1 || b > 1, (size_t)joined * D * 4);
    l.part_bc = take(train, (size_t)d->groups * ssm_blocks(d, kSsmBack) * tokens * 2 * N * 4);
    l.part_A = take(train, (size_t)b * D * N * 4);
    l.part_cols = take(train, (size_t)b * 2 * D * 4);
    l.total = at ? at : 256;
    return l;
}

// FN<io type, states>
#define SSM_DISPATCH(desc_, CALL)                                                                        \
    do {                                                                                                 \
        if ((desc_)->io_dtype == DELTALOG_F32) { SSM_STATES(float, (desc_)->d_state, CALL); }            \
        else { SSM_STATES(__nv_bfloat16, (desc_)->d_state, CALL); }                                      \
    } while (0)
#define SSM_STATES(IO, n_, CALL)                                                                         \
    if ((n_) == 8) { CALL(IO, 8); } else if ((n_) == 16) { CALL(IO, 16); } else if ((n_) == 32) { CALL(IO, 32); } else { CALL(IO, 64); }

template <bool BACK>
int launch_ssm_join(const SsmArgs &a, int states, cudaStream_t s) {
    const size_t smem = (size_t)a.parts;
    if (int rc = ensure_smem(ssm_join_kernel<BACK>, smem)) return rc;
    ssm_join_kernel<BACK><<<(unsigned)ssm_ceil((long long)a.D_ * states / 4, 128), 128, smem, s>>>(a, states);
    return finish_launch();
}

int launch_ssm_forward(const deltalog_ssm_desc *d, const SsmArgs &a, cudaStream_t s);   // both passes
int launch_ssm_step(const deltalog_ssm_desc *d, const SsmArgs &a, cudaStream_t s);
int launch_ssm_backward(const deltalog_ssm_desc *d, const SsmArgs &a, cudaStream_t s);  // both passes and the sums

}  // namespace deltalog
