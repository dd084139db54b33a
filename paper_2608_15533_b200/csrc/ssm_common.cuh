// The selective state space scan: arguments, shapes and pieces that its kernels share.
//     delta = softplus(dt + bias);  h_t = a_t h_(t-1) + delta x B,  a = exp(delta A);  y = C . h + D x;  out = y silu(z)
//
// A lane holds four neighbouring states of a channel (of two or four channels where the state is wide), d_state / 4 lanes a channel, and
// walks down the tokens.  The packed tokens are cut into flat stretches of `span` tokens, whatever rows they belong to, one
// CTA per stretch and block of channels, so that ragged rows load the SMs evenly.  A row that goes on behind the end of a
// stretch is joined by a first pass over parts of the stretch, so that it has more CTAs than the second: the state that a part alone
// leaves, and the sum of its step sizes, whose exponential with A is the decay across it.  ssm_join_kernel puts them together.
#pragma once

#include <type_traits>

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
    int32_t span, spans, blocks, wide;          // stretches, blocks of channels per group, the forward pass's form
    int32_t part, parts;                        // parts of stretches, in tokens and in all
    float *local, *front, *sums;                // [parts, D_, N] state a part leaves, its open row's first state; [parts, D_] step sizes
    float *kept;                                // [max_tokens / 8, D_, N], or NULL
    // backward
    const void *dout;
    const float *dS_final;
    void *dx, *ddt, *dB, *dC, *dz;
    float *dA, *dD, *dbias, *dS_init;
    float *part_bc, *part_A, *part_cols;        // [G * blocks, rows, 2 N], [spans, D_, N], [spans, 2, D_]
};

// CTAs of a kernel that an SM holds, by its registers and its shared memory: 228 KB, of which the system takes one for every CTA.
constexpr int ssm_ctas(int by_registers, size_t shared) {
    return by_registers < (int)(228 * 1024 / (shared + 1024)) ? by_registers : (int)(228 * 1024 / (shared + 1024));
}

// Lanes of a channel, channels side by side in a warp.
template <int N> struct SsmLanes {
    static constexpr int kStates = N / 4, kChannels = 32 / kStates;
};

__device__ __forceinline__ float2 exp2_fast(float2 x) { return make_float2(exp2_fast(x.x), exp2_fast(x.y)); }

// Decays of a token, 2^(A delta), lifted by what the hardware's 2^x is low on average (ssm_lift).
__device__ __forceinline__ float2 ssm_decay(float2 A, float delta, float lift) { return exp2_fast(__ffma2_rn(A, both(delta), both(lift))); }

// softplus(v) = max(v, 0) + log(1 + e), e = exp(-|v|) in [0, 1], of two values.  The exponent of two is rounded, by up to |v| / 2^24,
// and so is its constant: what both lost, m - x log 2 (Cody and Waite's reduction), goes into the result by the first-order term
// (without the constant's part step sizes were high by 1.3e-8 |v|).  |v| is cut off where e is long 0, since an infinite exponent
// (of a mask's -inf, or of the lowest values of a type) would have lost what is no number; a v that is none stays so.  log(1 + e) = e P(e)
// with P the polynomial of degree 9 of least relative error on [0, 1] (5e-9, by exchange of its extrema): small step sizes keep their
// relative accuracy, which the logarithm of a rounded 1 + e would lose.  Measured against 64 bits: 2.8e-7 at most, from -85 to 80.
// `e` comes back for the derivative.
__device__ __forceinline__ float ssm_minus_abs(float v) {  // max(-|v|, -150), or NaN
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(-fabsf(v)), "f"(-150.f));
    return m;
}
__device__ __forceinline__ float2 ssm_softplus(float2 v, float2 &e) {
    const float2 m = make_float2(ssm_minus_abs(v.x), ssm_minus_abs(v.y)), x = __fmul2_rn(m, both(1.4426950408889634f));
    const float2 lost = __ffma2_rn(x, both(1.9046542e-9f), __ffma2_rn(x, both(-0.6931471805599453f), m));  // m - x log 2, its constant in two words
    e = exp2_fast(x);
    e = __ffma2_rn(e, lost, e);
    constexpr float kP[10] = {1.f, -0.4999990165233612f, 0.3332996368408203f, -0.24954134225845337f, 0.1967593878507614f,
                              -0.15305592119693756f, 0.10603655129671097f, -0.05695953220129013f, 0.01985146291553974f, -0.0032440251670777798f};
    float2 p = both(kP[9]);
#pragma unroll
    for (int i = 8; i >= 0; --i) p = __ffma2_rn(p, e, both(kP[i]));
    return __ffma2_rn(p, e, make_float2(fmaxf(v.x, 0.f), fmaxf(v.y, 0.f)));
}
// softplus'(v) = 1 / (1 + exp(-v)) from that e.
__device__ __forceinline__ float ssm_sigmoid(float v, float e) {
    const float r = rcp_fast(1.f + e);
    return v >= 0.f ? r : e * r;
}

// What lifts the decays' exponents x = A delta (in powers of two).  Measured against 64 bits, the hardware's 2^x is low on average, by
// 5e-9 to 7e-9 for x in [-3e-3, -1e-4], by 2.4e-8 from -2^-8 to -1 and by 5e-8 below.  That is little in one decay, but the same in all of
// them: a state that remembers 1.4 / |x| tokens, and the gradients that go back over them, are off by as many times as much.  An addend
// of the product, which is free, takes it out, of one size on either side of -2^-8.  A lane's four states of a channel share one, by the
// slowest of them, in which it counts most: in the scans by the step size that the channel's bias stands for, one choice for all
// tokens, so that a row's bits do not depend on its neighbours; without a bias or a softplus by a value in between.
// (dA, dbias, dS_init of 4 x 2048 tokens x 4096 channels, distance from 64 bits: 8.8e-7, 5.8e-7, 9.4e-7; with 2.2e-8 for all 1.6e-6, 7.1e-7,
// 1.4e-6, and slow channels (|x| of 1e-3) 1.4e-5 off where they now are 2e-6; with 0.9e-8 for all 1.6e-6, 7.8e-7, 1.2e-6.)
__device__ __forceinline__ float ssm_lift(float x) { return x > -0.00390625f ? 0.9e-8f : 2.9e-8f; }
__device__ __forceinline__ float ssm_lift(const SsmArgs &a, const float2 (&A2)[2], float bias) {
    float2 unused;
    const float x = fmaxf(fmaxf(A2[0].x, A2[0].y), fmaxf(A2[1].x, A2[1].y)) * ssm_softplus(both(bias), unused).x;
    return a.softplus && a.bias ? ssm_lift(x) : 1.4e-8f;
}

// Sums over the LN lanes of a group (STRIDE apart) of V values at once: every step halves the values that a lane answers for, as
// long as their number is even.  On return v[0..] holds the sums of the values from the returned index on.
template <int V, int LN, int STRIDE = 1>
__device__ __forceinline__ int lanes_reduce(float (&v)[V], int lane) {
    int first = 0;
    auto step = [&](auto have_, auto o_) {
        constexpr int HAVE = decltype(have_)::value, O = decltype(o_)::value;
        const bool up = lane & (O * STRIDE);
        if constexpr (HAVE % 2 == 0) {
#pragma unroll
            for (int j = 0; j < HAVE / 2; ++j) {
                const float send = up ? v[j] : v[j + HAVE / 2], stay = up ? v[j + HAVE / 2] : v[j];
                v[j] = stay + __shfl_xor_sync(0xffffffffu, send, O * STRIDE);
            }
            first += up ? HAVE / 2 : 0;
        } else {
#pragma unroll
            for (int j = 0; j < HAVE; ++j) v[j] += __shfl_xor_sync(0xffffffffu, v[j], O * STRIDE);
        }
    };
    constexpr int H1 = V % 2 ? V : V / 2, H2 = H1 % 2 ? H1 : H1 / 2, H3 = H2 % 2 ? H2 : H2 / 2;
    if constexpr (LN >= 2) step(std::integral_constant<int, V>{}, std::integral_constant<int, LN / 2>{});
    if constexpr (LN >= 4) step(std::integral_constant<int, H1>{}, std::integral_constant<int, LN / 4>{});
    if constexpr (LN >= 8) step(std::integral_constant<int, H2>{}, std::integral_constant<int, LN / 8>{});
    if constexpr (LN >= 16) step(std::integral_constant<int, H3>{}, std::integral_constant<int, LN / 16>{});
    return first;
}

// 16 bytes, or zeros where `there` is false (the address is not read then, but has to be a valid one).
__device__ __forceinline__ void ssm_copy16(void *dst, const void *src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(smem_addr(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// A tile of ROWS tokens x COLS elements (multiples of 16 bytes) into dense shared memory; tokens from `first` on are those of
// [lo, hi), columns those below `there`; everything else becomes zero.  ALL: nothing is missing.
template <bool ALL, int ROWS, int COLS, typename IO>
__device__ __forceinline__ void ssm_stage(IO *dst, const IO *src, long long stride, int first, int lo, int hi, int there) {
    constexpr int V = 16 / sizeof(IO), PER = COLS / V, N = ROWS * PER;
    const IO *tile = src + first * stride;
#pragma unroll
    for (int i0 = 0; i0 < N; i0 += kSsmThreads) {
        const int i = i0 + threadIdx.x;
        if (N % kSsmThreads && i >= N) break;
        const int r = i / PER, c = (i % PER) * V, t = first + r, off = r * (int)stride + c;
        if (ALL) {
            cp_async16(dst + i * V, tile + off);
        } else {
            const bool ok = t >= lo && t < hi && c < there;
            ssm_copy16(dst + i * V, ok ? tile + off : src, ok);
        }
    }
}

// Four neighbouring states' values of a token as two pairs.
template <typename IO>
__device__ __forceinline__ void ssm_pairs(const IO *p, float2 (&v)[2]) {
    float f[4];
    load_vec<IO, 4>(p, f);
    v[0] = make_float2(f[0], f[1]), v[1] = make_float2(f[2], f[3]);
}
__device__ __forceinline__ void ssm_load(const float *p, float2 (&v)[2]) {
    const float4 f = *reinterpret_cast<const float4 *>(p);
    v[0] = make_float2(f.x, f.y), v[1] = make_float2(f.z, f.w);
}
__device__ __forceinline__ void ssm_store(float *p, const float2 (&v)[2]) { *reinterpret_cast<float4 *>(p) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y); }

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

// f(row) for the rows without tokens among the share of one CTA of a grid's last rows, by every thread.
constexpr int kSsmEmptyRows = 1024;
inline unsigned ssm_empty_ctas(int n) {
    const long long ctas = ((long long)n + kSsmEmptyRows - 1) / kSsmEmptyRows;
    return (unsigned)(ctas < 32768 ? ctas : 32768);
}
template <typename F>
__device__ __forceinline__ void ssm_empty_rows(const SsmArgs &a, int share, F f) {
    const int lane = threadIdx.x & 31, shares = gridDim.y - a.spans;
    const int each = ((a.rows.n + shares - 1) / shares + 31) & ~31;
    const long long first = (long long)share * each;
    const int end = (int)min((long long)a.rows.n, first + each);
    for (int row = (int)min(first, (long long)end); row < end; row += 32) {
        const int mine = min(row + lane, end - 1);
        unsigned empty = __ballot_sync(0xffffffffu, row + lane < end && a.rows.starts[mine] == a.rows.starts[mine + 1]);
        for (; empty; empty &= empty - 1) f(row + __ffs(empty) - 1);
    }
}

}  // namespace deltalog
