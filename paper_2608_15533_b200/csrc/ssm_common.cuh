// The selective state space scan: arguments, shapes and pieces that its kernels share.
//     delta = softplus(dt + bias);  h_t = a_t h_(t-1) + delta x B,  a = exp(delta A);  y = C . h + D x;  out = y silu(z)
//
// A lane holds four neighbouring states of a channel (of two or four channels where the state is wide), d_state / 4 lanes a channel, and
// walks down the tokens.  The packed tokens are cut into flat stretches of `span` tokens, whatever rows they belong to, one
// CTA per stretch and block of channels, so that ragged rows load the SMs evenly.  A row that goes on behind the end of a
// stretch is joined by a first pass over the stretch (ssm_local_kernel): the state that the stretch alone leaves, and the sum
// of its step sizes, whose exponential with A is the decay across it.  The second pass starts from
//     h = exp(A sum_j) (.. exp(A sum_i) h_i + h_(i+1) ..) + h_j.
#pragma once

#include "layer_common.cuh"

namespace deltalog {

constexpr int kSsmThreads = 128, kSsmWarps = kSsmThreads / 32;
constexpr int kSsmBlock = 8;  // tokens between two kept states

struct SsmArgs {
    const void *x, *dt, *B, *C, *z;
    long long x_stride, dt_stride, B_stride, C_stride, z_stride;
    const float *A, *D, *bias;
    void *out;
    const float *S_in;  // states in front of the rows (the pool for prefill), or NULL
    float *S_out;
    const int32_t *slots, *fresh;  // per row; NULL: row i is state i, none starts afresh
    int32_t *status;
    Rows rows;
    int32_t D_, G, num_slots, softplus, clear;  // D_: channels
    int32_t max_tokens, total_rows;             // tokens that the plan reaches; rows of the token tensors
    int32_t span, spans, blocks;                // stretches and blocks of channels per group
    float *local, *front, *sums;                // [spans, D_, N] state a stretch leaves, its open row's first state; [spans, D_] step sizes
    float *kept;                                // [max_tokens / 8, D_, N], or NULL
    // backward
    const void *dout;
    const float *dS_final;
    void *dx, *ddt, *dB, *dC, *dz;
    float *dA, *dD, *dbias, *dS_init;
    float *part_bc, *part_A, *part_cols;        // [G * blocks, rows, 2 N], [spans, D_, N], [spans, 2, D_]
};

// Lanes of a channel, channels side by side in a warp.
template <int N> struct SsmLanes {
    static constexpr int kStates = N / 4, kChannels = 32 / kStates;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// softplus(v) = max(v, 0) + log(1 + e), e = exp(-|v|) <= 1, with log(1 + e) = 2 atanh(t), t = e / (2 + e) <= 1/3, by the
// series t + t^3/3 + ..: what is left out is below t^14 / 15 < 2e-8 of the sum, and small e keep their relative accuracy.
__device__ __forceinline__ float ssm_softplus(float v) {
    const float e = __expf(-fabsf(v)), t = __fdividef(e, 2.f + e), s = t * t;
    float p = 1.f / 13.f;
    p = fmaf(p, s, 1.f / 11.f);
    p = fmaf(p, s, 1.f / 9.f);
    p = fmaf(p, s, 1.f / 7.f);
    p = fmaf(p, s, 1.f / 5.f);
    p = fmaf(p, s, 1.f / 3.f);
    p = fmaf(p, s, 1.f);
    return fmaxf(v, 0.f) + 2.f * t * p;
}

// Sums over the LN neighbouring lanes of a group, of V values at once: every step halves the values that a lane answers
// for.  On return v[0 .. V / LN) hold the sums of the values from the returned index on.
template <int V, int LN, int STRIDE = 1>
__device__ __forceinline__ int lanes_reduce(float (&v)[V], int lane) {
    int first = 0, have = V;
#pragma unroll
    for (int o = LN / 2; o > 0; o >>= 1) {
        const bool up = lane & (o * STRIDE);
        if (have > 1) {
            have >>= 1;
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                if (j < have) {
                    const float send = up ? v[j] : v[j + have], stay = up ? v[j + have] : v[j];
                    v[j] = stay + __shfl_xor_sync(0xffffffffu, send, o * STRIDE);
                }
            }
            first += up ? have : 0;
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], o * STRIDE);
        }
    }
    return first;
}

// 16 bytes, or zeros where `there` is false (the address is not read then, but has to be a valid one).
__device__ __forceinline__ void ssm_copy16(void *dst, const void *src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(smem_addr(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// A tile of `rows` tokens x `cols` elements (16-byte multiples) into dense shared memory; tokens from `first` on are those
// of [lo, hi), columns those below `cols_there`; everything else becomes zero.
template <typename IO>
__device__ __forceinline__ void ssm_stage(IO *dst, const IO *src, long long stride, int first, int rows, int lo, int hi, int cols, int cols_there, int threads) {
    constexpr int V = 16 / sizeof(IO);
    const int per = cols / V;
    for (int i = threadIdx.x; i < rows * per; i += threads) {
        const int r = i / per, c = (i - r * per) * V, t = first + r;
        const bool there = t >= lo && t < hi && c < cols_there;
        ssm_copy16(dst + r * cols + c, there ? src + (size_t)t * stride + c : src, there);
    }
}

// What a token's row says: looked up by one lane per token of a tile.
struct SsmToken {
    int row, state;      // -1: a token that the call skips
    int begin, end;      // its row's tokens
};
__device__ __forceinline__ SsmToken ssm_token(const SsmArgs &a, int t, bool tell) {
    SsmToken k{-1, -1, 0, 0};
    if (t >= a.max_tokens) return k;
    const int row = a.rows.of(t);
    if (row < 0) return k;
    k.state = row;
    if (a.slots) {
        k.state = a.slots[row];
        if (k.state >= a.num_slots) {
            if (tell && a.status) atomicOr(a.status, DELTALOG_STATUS_BAD_SLOT);
            k.state = -1;
        }
        if (k.state < 0) return k;
    }
    k.row = row, k.begin = a.rows.starts[row], k.end = a.rows.starts[row + 1];
    return k;
}

}  // namespace deltalog
