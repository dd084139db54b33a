// Short causal convolution over packed sequences and for single tokens:
//     pre[t] = bias + sum_j w[j] x[t - (W - 1) + j],   out = pre or pre sigmoid(pre)
// with a row's window (its last W - 1 inputs) in front of its first token.
//
// Bound by HBM: an input is read and an output written once, a dozen operations between them.  A lane holds the weights of four
// neighbouring channels in registers and walks down a run of tokens, so that an input is loaded once per run and the W - 1 inputs in
// front of it come out of registers; the arithmetic is packed, two channels an instruction.  The first W - 1 tokens of a row, which
// need its window, and the window itself are left to blocks of their own, one warp per row and vector of channels: a window is
// then read and written by the same threads, in that order, however many blocks work on the row.
// 36k x 8192 16-bit inputs 207 us (5.7 TB/s, 0.87 of a copy); 16k x 4096 52 us, their gradients 113 us (3.6 TB/s): 59 % of the issue
// slots, 33 instructions an element by the counters, nearly half of them outside of the loop over whole groups of tokens (runs of 56 tokens
// begin and end in the general form, look up their row and walk three tokens further), with the 16 warps an SM that 128 registers leave.
#pragma once

#include "layer_common.cuh"

namespace deltalog {

struct ConvArgs {
    const void *x, *init;  // init: windows in front of the rows (the pool for prefill), or NULL
    long long x_stride;
    const float *w, *bias;
    void *out, *final;
    const int32_t *slots, *fresh;  // per row; NULL: row i is window i, none starts afresh
    int32_t *status;
    Rows rows;
    int32_t C, silu, num_slots, max_tokens, total_rows, run, clear;
    // backward
    const void *dout, *dfinal;
    void *dx, *dinit;
    float *partial;
};

constexpr int kConvThreads = 128, kConvVec = 4;  // channels per lane: eight would need up to 200 registers

// Inputs on their way: a lane copies its own channels of U tokens a stage into shared memory and reads nothing but its own, so that a
// wait for its own copies is all it needs.  (Held in registers instead, eight tokens ahead: 257 us where this takes 207.)
template <typename IO>
__device__ __forceinline__ void conv_copy(Pack<IO, kConvVec> *dst, const IO *src) {
    if constexpr (sizeof(IO) * kConvVec == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(smem_addr(dst)), "l"(src) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;\n" ::"r"(smem_addr(dst)), "l"(src) : "memory");
}
template <int N>
__device__ __forceinline__ void conv_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }

// Window of a row: slot or row, -1 for a row that the call skips.
__device__ __forceinline__ int conv_slot(const ConvArgs &a, int row, bool tell) {
    if (!a.slots) return row;
    const int slot = a.slots[row];
    if (slot < a.num_slots) return slot;
    if (tell && a.status) atomicOr(a.status, DELTALOG_STATUS_BAD_SLOT);
    return -1;
}

// A lane's four channels as two pairs, for the packed arithmetic.
struct Quad { float2 a, b; };
__device__ __forceinline__ Quad quad(float4 f) { return {make_float2(f.x, f.y), make_float2(f.z, f.w)}; }
__device__ __forceinline__ Quad quad_zero() { return {both(0.f), both(0.f)}; }
template <typename IO>
__device__ __forceinline__ Quad quad(const Pack<IO, kConvVec> &v) { return {load2(v.e), load2(v.e + 2)}; }
__device__ __forceinline__ Quad quad_fma(const Quad &x, const Quad &y, const Quad &z) { return {__ffma2_rn(x.a, y.a, z.a), __ffma2_rn(x.b, y.b, z.b)}; }
template <typename IO>
__device__ __forceinline__ Pack<IO, kConvVec> quad_round(const Quad &q) {
    Pack<IO, kConvVec> v;
    store2(v.e, q.a), store2(v.e + 2, q.b);
    return v;
}

// Weights [channels, W]: 4 W consecutive floats.
template <int W>
__device__ __forceinline__ void conv_weights(const ConvArgs &a, int c, Quad (&w)[W], Quad &b) {
    float f[W * kConvVec];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const float4 v = __ldg(reinterpret_cast<const float4 *>(a.w + (size_t)c * W) + i);
        f[4 * i] = v.x, f[4 * i + 1] = v.y, f[4 * i + 2] = v.z, f[4 * i + 3] = v.w;
    }
    b = a.bias ? quad(__ldg(reinterpret_cast<const float4 *>(a.bias + c))) : quad_zero();
#pragma unroll
    for (int j = 0; j < W; ++j) w[j] = {make_float2(f[j], f[W + j]), make_float2(f[2 * W + j], f[3 * W + j])};
}

// Pre-activations from the window p (p[0] the oldest input).
template <int W>
__device__ __forceinline__ Quad conv_pre(const Quad (&p)[W], const Quad (&w)[W], const Quad &b) {
    Quad r = b;
#pragma unroll
    for (int j = 0; j < W; ++j) r = quad_fma(w[j], p[j], r);
    return r;
}
template <typename IO>
__device__ __forceinline__ Pack<IO, kConvVec> conv_act(Quad r, bool silu) {
    if (silu) {
        r.a = __fmul2_rn(r.a, make_float2(sigmoid(r.a.x), sigmoid(r.a.y)));
        r.b = __fmul2_rn(r.b, make_float2(sigmoid(r.b.x), sigmoid(r.b.y)));
    }
    return quad_round<IO>(r);
}
template <int W>
__device__ __forceinline__ void conv_shift(Quad (&p)[W]) {
#pragma unroll
    for (int j = 0; j < W - 1; ++j) p[j] = p[j + 1];
}

// ---- forward over packed rows ------------------------------------------------------------------------------------
// Blocks [0, head_blocks): the rows' first tokens and windows.  The others: runs of tokens.
template <typename IO, int W>
__global__ void __launch_bounds__(kConvThreads) conv_forward_kernel(const ConvArgs a, int col_blocks, long long head_blocks) {
    constexpr int V = kConvVec, U = 8;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = ((int)(blockIdx.x % col_blocks) * 32 + lane) * V;
    const bool live = c < a.C;  // C is a multiple of 8
    const int cc = live ? c : 0;
    const IO *x = static_cast<const IO *>(a.x) + cc;
    IO *out = static_cast<IO *>(a.out) + cc;
    Quad w[W], b, p[W];
    const long long block = blockIdx.x / col_blocks;
    auto input = [&](long long t) { return pack_load<IO, V>(x + t * a.x_stride); };
    if (block < head_blocks) {
        const long long row = block * (kConvThreads / 32) + warp;
        if (row >= a.rows.n) return;
        const int slot = conv_slot(a, (int)row, true);
        if (slot < 0) return;
        const int s = a.rows.starts[row], len = a.rows.starts[row + 1] - s;
        if (len == 0 && (a.slots || !a.final)) return;
        conv_weights<W>(a, cc, w, b);
        const bool old = a.init && !(a.fresh && a.fresh[row]);
        const size_t at = (size_t)slot * (W - 1) * a.C + cc;
        Pack<IO, V> keep[W - 1], win[W - 1];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            win[j] = old ? pack_load<IO, V>(static_cast<const IO *>(a.init) + at + (size_t)j * a.C) : pack_zero<IO, V>();
            p[j] = quad(win[j]);
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int t = len - (W - 1) + j;  // token t of the row; in front of it, input W - 1 + t of the window
            keep[j] = win[j];
            if (t >= 0) keep[j] = input(s + t);
#pragma unroll
            for (int i = 0; i < W - 1; ++i)
                if (t < 0 && W - 1 + t == i) keep[j] = win[i];
        }
#pragma unroll
        for (int t = 0; t < W - 1; ++t) {
            if (t >= len) break;
            p[W - 1] = quad(input(s + t));
            const Pack<IO, V> o = conv_act<IO>(conv_pre<W>(p, w, b), a.silu);
            if (live) pack_store(out + (size_t)(s + t) * a.C, o);
            conv_shift(p);
        }
        if (live && a.final)
#pragma unroll
            for (int j = 0; j < W - 1; ++j) pack_store(static_cast<IO *>(a.final) + at + (size_t)j * a.C, keep[j]);
        return;
    }
    const long long first = ((block - head_blocks) * (kConvThreads / 32) + warp) * a.run;
    if (first >= a.max_tokens) return;
    const int t0 = (int)first, t1 = (int)min((long long)a.max_tokens, first + a.run);
    // every load of the first tokens is on its way before the look-ups of the row, each of which waits for the one before
    constexpr int S = sizeof(IO) == 4 ? 2 : 3;
    __shared__ Pack<IO, V> ring[kConvThreads / 32][S][U][32];
    Pack<IO, V> win[W - 1];
    auto fetch = [&](int t, int stage) {
        if (t < t1)
#pragma unroll
            for (int u = 0; u < U; ++u) conv_copy(&ring[warp][stage][u][lane], x + min(t + u, t1 - 1) * a.x_stride);
        cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < S - 1; ++s) fetch(t0 + s * U, s);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) win[j] = input(max(t0 - (W - 1) + j, 0));  // (of a row in front, perhaps: then it is not used)
    conv_weights<W>(a, cc, w, b);
    int end = a.max_tokens, begin = 0;
    bool mine = false;
    auto enter = [&](int r) {  // r < 0: behind the last sequence
        mine = r >= 0 && conv_slot(a, r, false) >= 0;
        begin = r >= 0 ? a.rows.starts[r] : 0;
        end = r >= 0 ? a.rows.starts[r + 1] : a.max_tokens;
    };
    const int row0 = a.rows.of(t0);
    if (row0 < 0) {  // all of the run is behind the last sequence
        if (a.clear && live)
            for (int t = t0; t < t1; ++t) pack_store(out + (size_t)t * a.C, pack_zero<IO, V>());
        conv_wait<0>();
        return;
    }
    enter(row0);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) p[j] = quad(win[j]);
    for (int t = t0, stage = 0; t < t1; t += U, stage = stage == S - 1 ? 0 : stage + 1) {
        fetch(t + (S - 1) * U, stage == 0 ? S - 1 : stage - 1);
        conv_wait<S - 1>();
        const Pack<IO, V> (*cur)[32] = ring[warp][stage];
        IO *to = out + (size_t)t * a.C;
        auto token = [&](int u) {
            p[W - 1] = quad(cur[u][lane]);
            const Pack<IO, V> o = conv_act<IO>(conv_pre<W>(p, w, b), a.silu);
            conv_shift(p);
            return o;
        };
        if (mine && t - begin >= W - 1 && t + U <= min(t1, end)) {  // one row, none of its first tokens
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const Pack<IO, V> o = token(u);
                if (live) pack_store(to + (size_t)u * a.C, o);
            }
            continue;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = t + u;
            if (at >= t1) break;
            if (at >= end) enter(a.rows.of(at));
            const Pack<IO, V> o = token(u);
            if (mine) {
                if (live && at - begin >= W - 1) pack_store(to + (size_t)u * a.C, o);
            } else if (a.clear && live) {
                pack_store(to + (size_t)u * a.C, pack_zero<IO, V>());
            }
        }
    }
}

// ---- single tokens ------------------------------------------------------------------------------------------------
// A lane takes the same channels of `run` rows, with the weights in registers and four rows in flight.
template <typename IO, int W>
__global__ void __launch_bounds__(kConvThreads) conv_step_kernel(const ConvArgs a, int col_blocks) {
    constexpr int V = kConvVec, U = 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = ((int)(blockIdx.x % col_blocks) * 32 + lane) * V;
    const long long first = ((long long)(blockIdx.x / col_blocks) * (kConvThreads / 32) + warp) * a.run;
    if (c >= a.C || first >= a.total_rows) return;
    const int end = (int)min((long long)a.total_rows, first + a.run);
    Quad w[W], b;
    for (int row = (int)first; row < end; row += U) {
        int slot[U];
        Pack<IO, V> p[U][W];
        step_slots(a.slots, row, end, slot);
        step_check(row, end, a.num_slots, a.status, slot);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (slot[u] < 0) continue;
            const IO *win = static_cast<const IO *>(a.init) + (size_t)slot[u] * (W - 1) * a.C + c;
#pragma unroll
            for (int j = 0; j < W - 1; ++j) p[u][j] = pack_load<IO, V>(win + (size_t)j * a.C);
            p[u][W - 1] = pack_load<IO, V>(static_cast<const IO *>(a.x) + (size_t)(row + u) * a.x_stride + c);
        }
        if (row == (int)first) conv_weights<W>(a, c, w, b);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (slot[u] < 0) continue;
            IO *win = static_cast<IO *>(a.final) + (size_t)slot[u] * (W - 1) * a.C + c;
            Quad f[W];
#pragma unroll
            for (int j = 0; j < W; ++j) f[j] = quad(p[u][j]);
            pack_store(static_cast<IO *>(a.out) + (size_t)(row + u) * a.C + c, conv_act<IO>(conv_pre<W>(f, w, b), a.silu));
#pragma unroll
            for (int j = 0; j < W - 1; ++j) pack_store(win + (size_t)j * a.C, p[u][j + 1]);
        }
    }
}

// ---- backward -----------------------------------------------------------------------------------------------------
// dpre = dout silu'(pre);  dx[t] = sum_back w[W - 1 - back] dpre[t + back] inside the row (+ dfinal where the window behind the
// row holds t);  dw[j] = sum_t dpre[t] x[t - (W - 1) + j];  dbias = sum_t dpre[t].
// The walk goes W - 1 tokens beyond its run, since dx[t] is complete with dpre[t + W - 1]; dx of the last W tokens waits in
// registers.  dw and dbias: a thread's sums over its run, a block's over its warps, then conv_reduce_kernel over the blocks,
// each in a fixed order.
__device__ __forceinline__ float2 conv_dpre(float2 pre, float2 g) {
    const float2 s = make_float2(sigmoid(pre.x), sigmoid(pre.y));
    const float2 slope = __ffma2_rn(pre, __ffma2_rn(s, both(-1.f), both(1.f)), both(1.f));  // silu' = s (1 + pre (1 - s))
    return __fmul2_rn(__fmul2_rn(g, s), slope);
}
__device__ __forceinline__ Quad conv_dpre(const Quad &pre, const Quad &g, bool silu) { return silu ? Quad{conv_dpre(pre.a, g.a), conv_dpre(pre.b, g.b)} : g; }

template <typename IO, int W>
__global__ void __launch_bounds__(kConvThreads, (sizeof(IO) == 4 ? 3 : 4)) conv_backward_kernel(const ConvArgs a, int col_blocks, long long head_blocks) {
    constexpr int V = kConvVec, U = 4, S = sizeof(IO) == 4 ? 2 : 4;
    __shared__ Pack<IO, V> ring[kConvThreads / 32][S][2][U][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = ((int)(blockIdx.x % col_blocks) * 32 + lane) * V;
    const bool live = c < a.C;
    const int cc = live ? c : 0;
    const IO *x = static_cast<const IO *>(a.x) + cc, *dout = static_cast<const IO *>(a.dout) + cc;
    const IO *init = static_cast<const IO *>(a.init), *dfinal = static_cast<const IO *>(a.dfinal);
    Quad w[W], b, p[W];
    auto window = [&](int row, int j) {  // input j of the row's window
        return init ? pack_load<IO, V>(init + ((size_t)row * (W - 1) + j) * a.C + cc) : pack_zero<IO, V>();
    };
    const long long block = blockIdx.x / col_blocks;
    if (block < head_blocks) {  // gradients of the windows
        const long long row = block * (kConvThreads / 32) + warp;
        if (row >= a.rows.n || !live) return;
        conv_weights<W>(a, cc, w, b);
        const int s = a.rows.starts[row], len = a.rows.starts[row + 1] - s;
        Quad d[W - 1];
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {
            p[i] = quad(window((int)row, i)), d[i] = quad_zero();
            if (dfinal && i >= len) d[i] = quad(pack_load<IO, V>(dfinal + ((size_t)row * (W - 1) + (i - len)) * a.C + cc));
        }
#pragma unroll
        for (int t = 0; t < W - 1; ++t) {
            if (t >= len) break;
            p[W - 1] = quad(pack_load<IO, V>(x + (size_t)(s + t) * a.x_stride));
            const Quad g = conv_dpre(conv_pre<W>(p, w, b), quad(pack_load<IO, V>(dout + (size_t)(s + t) * a.C)), a.silu);
#pragma unroll
            for (int i = t; i < W - 1; ++i) d[i] = quad_fma(w[i - t], g, d[i]);  // input i of the window is input i - t of this token's
            conv_shift(p);
        }
#pragma unroll
        for (int i = 0; i < W - 1; ++i) pack_store(static_cast<IO *>(a.dinit) + ((size_t)row * (W - 1) + i) * a.C + cc, quad_round<IO>(d[i]));
        return;
    }
    const long long group = block - head_blocks;
    const long long first = (group * (kConvThreads / 32) + warp) * a.run;
    const int t0 = (int)min(first, (long long)a.total_rows), t1 = (int)min((long long)a.total_rows, first + a.run);
    Quad dw[W + 1], pend[W];  // pend[k]: dx of token t - k so far
#pragma unroll
    for (int j = 0; j <= W; ++j) dw[j] = quad_zero();
#pragma unroll
    for (int k = 0; k < W; ++k) pend[k] = quad_zero();
    if (t0 < t1) {
        const int tokens = a.rows.n ? a.rows.starts[a.rows.n] : 0, te = min(t1 + W - 1, tokens);  // tokens whose dpre counts
        auto fetch = [&](int t, int stage) {
            if (t < te)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const long long at = min(t + u, te - 1);
                    conv_copy(&ring[warp][stage][0][u][lane], x + at * a.x_stride);
                    conv_copy(&ring[warp][stage][1][u][lane], dout + at * a.C);
                }
            cp_async_commit();
        };
#pragma unroll
        for (int s = 0; s < S - 1; ++s) fetch(t0 + s * U, s);
        conv_weights<W>(a, cc, w, b);
        int row = -1, begin = 0, end = 0;
        auto enter = [&](int t) {
            row = a.rows.of(t);
            begin = a.rows.starts[row], end = a.rows.starts[row + 1];
        };
        if (t0 < tokens) {
            enter(t0);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                const int t = t0 - (W - 1) + j;  // of the row, or of its window
                p[j] = quad(t >= begin ? pack_load<IO, V>(x + (size_t)t * a.x_stride) : window(row, W - 1 + t - begin));
            }
        }
        for (int t = t0, stage = 0; t < t1 + W - 1; t += U, stage = stage == S - 1 ? 0 : stage + 1) {
            fetch(t + (S - 1) * U, stage == 0 ? S - 1 : stage - 1);
            conv_wait<S - 1>();
            const Pack<IO, V> (*cur)[U][32] = ring[warp][stage];
            IO *to = static_cast<IO *>(a.dx) + cc + ((long long)t - (W - 1)) * a.C;
            auto shift = [&]() {
#pragma unroll
                for (int k = W - 1; k > 0; --k) pend[k] = pend[k - 1];
                pend[0] = quad_zero();
            };
            auto token = [&](int u, int reach, bool own) {  // dpre of a token, into its own and the `reach` pending dx in front
                p[W - 1] = quad(cur[0][u][lane]);
                const Quad g = conv_dpre(conv_pre<W>(p, w, b), quad(cur[1][u][lane]), a.silu);
                if (own) {
                    dw[W].a = __fadd2_rn(dw[W].a, g.a), dw[W].b = __fadd2_rn(dw[W].b, g.b);
#pragma unroll
                    for (int j = 0; j < W; ++j) dw[j] = quad_fma(g, p[j], dw[j]);
                }
#pragma unroll
                for (int k = 0; k < W; ++k)
                    if (k <= reach) pend[k] = quad_fma(w[W - 1 - k], g, pend[k]);
                conv_shift(p);
            };
            if (t - t0 >= W - 1 && t - begin >= W - 1 && t + U <= min(t1, end - (W - 1))) {  // one row, away from both ends
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    shift();
                    token(u, W - 1, true);
                    if (live) pack_store(to + (long long)u * a.C, quad_round<IO>(pend[W - 1]));
                }
                continue;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = t + u;
                if (at >= t1 + W - 1) break;
                shift();
                if (at < te) {
                    if (at >= end) {
                        enter(at);
#pragma unroll
                        for (int j = 0; j < W - 1; ++j) p[j] = quad(window(row, j));
                    }
                    if (at < t1 && dfinal && at >= end - (W - 1))
                        pend[0] = quad(pack_load<IO, V>(dfinal + ((size_t)row * (W - 1) + (at - end + W - 1)) * a.C + cc));
                    token(u, at - begin, at < t1);
                }
                if (at - (W - 1) >= t0 && live) pack_store(to + (long long)u * a.C, quad_round<IO>(pend[W - 1]));
            }
        }
    }
    // (the ring has room for the sums: every copy has arrived)
    conv_wait<0>();
    __syncthreads();
    static_assert(sizeof(ring) >= sizeof(float4) * kConvThreads * (W + 1), "the sums fit");
    auto sums = reinterpret_cast<float4 (*)[W + 1][32]>(&ring);
#pragma unroll
    for (int j = 0; j <= W; ++j) sums[warp][j][lane] = make_float4(dw[j].a.x, dw[j].a.y, dw[j].b.x, dw[j].b.y);
    __syncthreads();
    for (int i = threadIdx.x; i < (W + 1) * 32; i += kConvThreads) {
        const int j = i / 32, col = (int)(blockIdx.x % col_blocks) * 32 * V + i % 32 * V;
        if (col >= a.C) continue;
        float4 s = sums[0][j][i % 32];
#pragma unroll
        for (int k = 1; k < kConvThreads / 32; ++k) {
            const float4 f = sums[k][j][i % 32];
            s.x += f.x, s.y += f.y, s.z += f.z, s.w += f.w;
        }
        *reinterpret_cast<float4 *>(a.partial + ((size_t)group * (W + 1) + j) * a.C + col) = s;
    }
}

// dw [C, W] and dbias [C] from the blocks' partial sums.
__global__ void __launch_bounds__(256) conv_reduce_kernel(const float *partial, long long groups, int C, int W, float *dw, float *dbias) {
    const float s = column_sum(partial, groups, (W + 1) * C);
    const int i = blockIdx.x * 32 + threadIdx.x;
    if (threadIdx.x >= 32 || i >= (W + 1) * C) return;
    const int j = i / C, c = i - j * C;
    if (j < W) dw[(size_t)c * W + j] = s;
    else if (dbias) dbias[c] = s;
}

}  // namespace deltalog
