// Short causal convolution over packed sequences and for single tokens:
//     pre[t] = bias + sum_j w[j] x[t - (W - 1) + j],   out = pre or pre sigmoid(pre)
// with a row's window (its last W - 1 inputs) in front of its first token.
//
// Bound by HBM: an input is read and an output written once, a dozen operations between them.  A thread holds the weights of
// a vector of neighbouring channels (16 bytes of them) in registers and walks down a run of tokens, so that an input is
// loaded once per run and the W - 1 inputs in front of it come out of registers; the next eight tokens' loads are under way
// while eight are computed.  The first W - 1 tokens of a row, which need its window, and the window itself are left to
// blocks of their own, one warp per row and vector of channels: a window is then read and written by the same threads, in
// that order, however many blocks work on the row.
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

// Window of a row: slot or row, -1 for a row that the call skips.
__device__ __forceinline__ int conv_slot(const ConvArgs &a, int row, bool tell) {
    if (!a.slots) return row;
    const int slot = a.slots[row];
    if (slot < a.num_slots) return slot;
    if (tell && a.status) atomicOr(a.status, DELTALOG_STATUS_BAD_SLOT);
    return -1;
}

template <int W, int V>
__device__ __forceinline__ void conv_weights(const ConvArgs &a, int c, float (&w)[W][V], float (&b)[V]) {
    // [channels, W]: V * W consecutive floats
    float flat[W * V];
#pragma unroll
    for (int i = 0; i < W * V / 4; ++i) {
        const float4 f = __ldg(reinterpret_cast<const float4 *>(a.w + (size_t)c * W) + i);
        flat[4 * i] = f.x, flat[4 * i + 1] = f.y, flat[4 * i + 2] = f.z, flat[4 * i + 3] = f.w;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        b[v] = a.bias ? __ldg(a.bias + c + v) : 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) w[j][v] = flat[v * W + j];
    }
}

// pre-activations from the window `p` (p[0] the oldest input): as it is in memory, or widened
template <int W, int V>
__device__ __forceinline__ void conv_pre(const float (&p)[W][V], const float (&w)[W][V], const float (&b)[V], float (&pre)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        pre[v] = b[v];
#pragma unroll
        for (int j = 0; j < W; ++j) pre[v] = fmaf(w[j][v], p[j][v], pre[v]);
    }
}
template <typename IO, int V>
__device__ __forceinline__ void conv_floats(const Pack<IO, V> &v, float (&f)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = to_f32(v.e[i]);
}
template <typename IO, int W, int V>
__device__ __forceinline__ void conv_pre(const Pack<IO, V> (&p)[W], const float (&w)[W][V], const float (&b)[V], float (&pre)[V]) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        pre[v] = b[v];
#pragma unroll
        for (int j = 0; j < W; ++j) pre[v] = fmaf(w[j][v], to_f32(p[j].e[v]), pre[v]);
    }
}
template <typename IO, int V>
__device__ __forceinline__ Pack<IO, V> conv_act(float (&pre)[V], bool silu) {
#pragma unroll
    for (int v = 0; v < V; ++v)
        if (silu) pre[v] *= sigmoid(pre[v]);
    return pack_round<IO, V>(pre);
}

// ---- forward over packed rows ------------------------------------------------------------------------------------
// Blocks [0, head_blocks): the rows' first tokens and windows.  The others: runs of tokens.
template <typename IO, int W>
__global__ void __launch_bounds__(kConvThreads, 5) conv_forward_kernel(const ConvArgs a, int col_blocks, long long head_blocks) {
    constexpr int V = kConvVec, U = 8;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = ((int)(blockIdx.x % col_blocks) * 32 + lane) * V;
    const bool live = c < a.C;  // C is a multiple of 8
    const int cc = live ? c : 0;
    const IO *x = static_cast<const IO *>(a.x) + cc;
    IO *out = static_cast<IO *>(a.out) + cc;
    float w[W][V], b[V];
    conv_weights<W, V>(a, cc, w, b);
    Pack<IO, V> p[W];
    const long long block = blockIdx.x / col_blocks;
    if (block < head_blocks) {
        const long long row = block * (kConvThreads / 32) + warp;
        if (row >= a.rows.n) return;
        const int slot = conv_slot(a, (int)row, true);
        if (slot < 0) return;
        const int s = a.rows.starts[row], len = a.rows.starts[row + 1] - s;
        if (len == 0 && (a.slots || !a.final)) return;
        const bool old = a.init && !(a.fresh && a.fresh[row]);
        const size_t at = (size_t)slot * (W - 1) * a.C + cc;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) p[j] = old ? pack_load<IO, V>(static_cast<const IO *>(a.init) + at + (size_t)j * a.C) : pack_zero<IO, V>();
        Pack<IO, V> last[W - 1];  // of the row's tokens, in front of which come the window's
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int t = len - (W - 1) + j;
            if (t >= 0) last[j] = pack_load<IO, V>(x + (size_t)(s + t) * a.x_stride);
        }
        Pack<IO, V> keep[W - 1];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int t = len - (W - 1) + j;  // t < 0: input W - 1 + t of the window
            keep[j] = p[j];
            if (t >= 0) keep[j] = last[j];
#pragma unroll
            for (int i = 0; i < W - 1; ++i)
                if (t < 0 && W - 1 + t == i) keep[j] = p[i];
        }
#pragma unroll
        for (int t = 0; t < W - 1; ++t) {
            if (t >= len) break;
            p[W - 1] = pack_load<IO, V>(x + (size_t)(s + t) * a.x_stride);
            float pre[V];
            conv_pre<IO, W, V>(p, w, b, pre);
            const Pack<IO, V> o = conv_act<IO, V>(pre, a.silu);
            if (live) pack_store(out + (size_t)(s + t) * a.C, o);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) p[j] = p[j + 1];
        }
        if (live && a.final)
#pragma unroll
            for (int j = 0; j < W - 1; ++j) pack_store(static_cast<IO *>(a.final) + at + (size_t)j * a.C, keep[j]);
        return;
    }
    const long long first = ((block - head_blocks) * (kConvThreads / 32) + warp) * a.run;
    if (first >= a.max_tokens) return;
    const int t0 = (int)first, t1 = (int)min((long long)a.max_tokens, first + a.run);
    int row = a.rows.of(t0), end = a.max_tokens, begin = 0;
    bool mine = false;
    auto enter = [&](int r) {  // r < 0: behind the last sequence
        row = r;
        mine = r >= 0 && conv_slot(a, r, false) >= 0;
        begin = r >= 0 ? a.rows.starts[r] : 0;
        end = r >= 0 ? a.rows.starts[r + 1] : a.max_tokens;
    };
    enter(row);
    float f[W][V];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int t = t0 - (W - 1) + j;
        conv_floats(t >= 0 ? pack_load<IO, V>(x + (size_t)t * a.x_stride) : pack_zero<IO, V>(), f[j]);
    }
    Pack<IO, V> in[U];
    auto fetch = [&](int t) {
        if (t + U <= t1) {
            const IO *from = x + (size_t)t * a.x_stride;
#pragma unroll
            for (int u = 0; u < U; ++u) in[u] = pack_load<IO, V>(from + u * a.x_stride);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) in[u] = pack_load<IO, V>(x + (size_t)min(t + u, t1 - 1) * a.x_stride);
        }
    };
    fetch(t0);
    for (int t = t0; t < t1; t += U) {
        Pack<IO, V> cur[U];
#pragma unroll
        for (int u = 0; u < U; ++u) cur[u] = in[u];
        if (t + U < t1) fetch(t + U);
        IO *to = out + (size_t)t * a.C;
        auto token = [&](int u) {
            conv_floats(cur[u], f[W - 1]);
            float pre[V];
            conv_pre<W, V>(f, w, b, pre);
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) f[j][v] = f[j + 1][v];
            return conv_act<IO, V>(pre, a.silu);
        };
        if (mine && t - begin >= W - 1 && t + U <= min(t1, end)) {  // one row, none of its first tokens
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const Pack<IO, V> o = token(u);
                if (live) pack_store(to + u * a.C, o);
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
                if (live && at - begin >= W - 1) pack_store(to + u * a.C, o);
            } else if (a.clear && live) {
                pack_store(to + u * a.C, pack_zero<IO, V>());
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
    float w[W][V], b[V];
    for (int row = (int)first; row < end; row += U) {
        int slot[U];
        Pack<IO, V> p[U][W];
        step_slots(a.slots, row, end, a.num_slots, a.status, slot);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (slot[u] < 0) continue;
            const IO *win = static_cast<const IO *>(a.init) + (size_t)slot[u] * (W - 1) * a.C + c;
#pragma unroll
            for (int j = 0; j < W - 1; ++j) p[u][j] = pack_load<IO, V>(win + (size_t)j * a.C);
            p[u][W - 1] = pack_load<IO, V>(static_cast<const IO *>(a.x) + (size_t)(row + u) * a.x_stride + c);
        }
        if (row == (int)first) conv_weights<W, V>(a, c, w, b);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (slot[u] < 0) continue;
            IO *win = static_cast<IO *>(a.final) + (size_t)slot[u] * (W - 1) * a.C + c;
            float pre[V];
            conv_pre<IO, W, V>(p[u], w, b, pre);
            pack_store(static_cast<IO *>(a.out) + (size_t)(row + u) * a.C + c, conv_act<IO, V>(pre, a.silu));
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
template <int V>
__device__ __forceinline__ void conv_dpre(float (&pre)[V], const float (&g)[V], bool silu) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
        if (silu) {
            const float s = sigmoid(pre[v]);
            pre[v] = g[v] * s * (1.f + pre[v] * (1.f - s));
        } else {
            pre[v] = g[v];
        }
    }
}

template <typename IO, int W>
__global__ void __launch_bounds__(kConvThreads, 3) conv_backward_kernel(const ConvArgs a, int col_blocks, long long head_blocks) {
    constexpr int V = kConvVec, U = 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = ((int)(blockIdx.x % col_blocks) * 32 + lane) * V;
    const bool live = c < a.C;
    const int cc = live ? c : 0;
    const IO *x = static_cast<const IO *>(a.x) + cc, *dout = static_cast<const IO *>(a.dout) + cc;
    const IO *init = static_cast<const IO *>(a.init), *dfinal = static_cast<const IO *>(a.dfinal);
    float w[W][V], b[V];
    conv_weights<W, V>(a, cc, w, b);
    Pack<IO, V> p[W];
    auto window = [&](int row, int j) {  // input j of the row's window
        return init ? pack_load<IO, V>(init + ((size_t)row * (W - 1) + j) * a.C + cc) : pack_zero<IO, V>();
    };
    const long long block = blockIdx.x / col_blocks;
    if (block < head_blocks) {  // gradients of the windows
        const long long row = block * (kConvThreads / 32) + warp;
        if (row >= a.rows.n || !live) return;
        const int s = a.rows.starts[row], len = a.rows.starts[row + 1] - s;
        float d[W - 1][V];
#pragma unroll
        for (int i = 0; i < W - 1; ++i) {
            p[i] = window((int)row, i);
#pragma unroll
            for (int v = 0; v < V; ++v) d[i][v] = 0.f;
            if (dfinal && i >= len) conv_floats(pack_load<IO, V>(dfinal + ((size_t)row * (W - 1) + (i - len)) * a.C + cc), d[i]);
        }
#pragma unroll
        for (int t = 0; t < W - 1; ++t) {
            if (t >= len) break;
            p[W - 1] = pack_load<IO, V>(x + (size_t)(s + t) * a.x_stride);
            float pre[V], g[V];
            conv_pre<IO, W, V>(p, w, b, pre);
            conv_floats(pack_load<IO, V>(dout + (size_t)(s + t) * a.C), g);
            conv_dpre<V>(pre, g, a.silu);
#pragma unroll
            for (int i = t; i < W - 1; ++i)  // input i of the window is input i - t of this token's
#pragma unroll
                for (int v = 0; v < V; ++v) d[i][v] = fmaf(w[i - t][v], pre[v], d[i][v]);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) p[j] = p[j + 1];
        }
#pragma unroll
        for (int i = 0; i < W - 1; ++i) pack_store(static_cast<IO *>(a.dinit) + ((size_t)row * (W - 1) + i) * a.C + cc, pack_round<IO, V>(d[i]));
        return;
    }
    const long long group = block - head_blocks;
    const long long first = (group * (kConvThreads / 32) + warp) * a.run;
    const int t0 = (int)min(first, (long long)a.total_rows), t1 = (int)min((long long)a.total_rows, first + a.run);
    float dw[W + 1][V], pend[W][V];  // pend[k]: dx of token t - k so far
#pragma unroll
    for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) dw[j][v] = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) pend[k][v] = 0.f;
    if (t0 < t1) {
        const int tokens = a.rows.n ? a.rows.starts[a.rows.n] : 0, te = min(t1 + W - 1, tokens);  // tokens whose dpre counts
        int row = -1, begin = 0, end = 0;
        auto enter = [&](int t) {
            row = a.rows.of(t);
            begin = a.rows.starts[row], end = a.rows.starts[row + 1];
        };
        float f[W][V];
        if (t0 < tokens) {
            enter(t0);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                const int t = t0 - (W - 1) + j;  // of the row, or of its window
                conv_floats(t >= begin ? pack_load<IO, V>(x + (size_t)t * a.x_stride) : window(row, W - 1 + t - begin), f[j]);
            }
        }
        Pack<IO, V> in[U], dn[U];
        auto fetch = [&](int t) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const size_t at = max(0, min(t + u, te - 1));
                in[u] = pack_load<IO, V>(x + at * a.x_stride), dn[u] = pack_load<IO, V>(dout + at * a.C);
            }
        };
        if (t0 < te) fetch(t0);
        for (int t = t0; t < t1 + W - 1; t += U) {
            Pack<IO, V> cur[U], dcur[U];
#pragma unroll
            for (int u = 0; u < U; ++u) cur[u] = in[u], dcur[u] = dn[u];
            if (t + U < te) fetch(t + U);
            IO *to = static_cast<IO *>(a.dx) + cc + ((long long)t - (W - 1)) * a.C;
            auto shift = [&]() {
#pragma unroll
                for (int k = W - 1; k > 0; --k)
#pragma unroll
                    for (int v = 0; v < V; ++v) pend[k][v] = pend[k - 1][v];
#pragma unroll
                for (int v = 0; v < V; ++v) pend[0][v] = 0.f;
            };
            auto token = [&](int u, int reach, bool own) {  // dpre of a token, into its own and the `reach` pending dx in front
                conv_floats(cur[u], f[W - 1]);
                float pre[V], g[V];
                conv_pre<W, V>(f, w, b, pre);
                conv_floats(dcur[u], g);
                conv_dpre<V>(pre, g, a.silu);
                if (own)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        dw[W][v] += pre[v];
#pragma unroll
                        for (int j = 0; j < W; ++j) dw[j][v] = fmaf(pre[v], f[j][v], dw[j][v]);
                    }
#pragma unroll
                for (int k = 0; k < W; ++k)
                    if (k <= reach)
#pragma unroll
                        for (int v = 0; v < V; ++v) pend[k][v] = fmaf(w[W - 1 - k][v], pre[v], pend[k][v]);
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
#pragma unroll
                    for (int v = 0; v < V; ++v) f[j][v] = f[j + 1][v];
            };
            if (t - t0 >= W - 1 && t - begin >= W - 1 && t + U <= min(t1, end - (W - 1))) {  // one row, away from both ends
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    shift();
                    token(u, W - 1, true);
                    if (live) pack_store(to + u * a.C, pack_round<IO, V>(pend[W - 1]));
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
                        for (int j = 0; j < W - 1; ++j) conv_floats(window(row, j), f[j]);
                    }
                    if (at < t1 && dfinal && at >= end - (W - 1))
                        conv_floats(pack_load<IO, V>(dfinal + ((size_t)row * (W - 1) + (at - end + W - 1)) * a.C + cc), pend[0]);
                    token(u, at - begin, at < t1);
                }
                if (at - (W - 1) >= t0 && live) pack_store(to + u * a.C, pack_round<IO, V>(pend[W - 1]));
            }
        }
    }
    __shared__ float sums[kConvThreads / 32][W + 1][32 * V];
#pragma unroll
    for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int v = 0; v < V; ++v) sums[warp][j][v * 32 + lane] = dw[j][v];
    __syncthreads();
    const int c0 = (int)(blockIdx.x % col_blocks) * 32 * V;
    for (int i = threadIdx.x; i < (W + 1) * 32 * V; i += kConvThreads) {
        const int j = i / (32 * V), col = i % (32 * V), at = (col % V) * 32 + col / V;
        if (c0 + col >= a.C) continue;
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kConvThreads / 32; ++k) s += sums[k][j][at];
        a.partial[((size_t)group * (W + 1) + j) * a.C + c0 + col] = s;
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
