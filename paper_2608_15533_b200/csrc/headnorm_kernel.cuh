// Norm, rotation and scale of query and key heads, both tensors in one launch, and its gradients.
//     n = w x r,  r = 1 / sqrt(c sum x^2 + eps)  (c = 1 for unit length, 1 / d for the root of the mean square)
//     y = scale (n turned pair by pair)
// Backward, with g = scale (dy turned back):  dw = sum g x r,  dx = r (g w - c r^2 x sum(g w x)).
//
// Bound by HBM: every value is read once and written once.  L lanes hold a head, eight neighbouring values each (16 bytes of
// 16-bit values), and a warp takes one token and several of its heads, so that the token's cosines and sines are loaded once for all of
// them and four heads a lane are in flight.  The sums over a head are butterflies over its lanes; with pairs half a rotation
// apart the partner's values come from lane +- rot / 16.
#pragma once

#include "layer_common.cuh"

namespace deltalog {

struct NormArgs {
    const void *q, *k;
    long long q_stride, k_stride;
    const float *w_q, *w_k, *cos, *sin;
    const int32_t *positions;
    void *out_q, *out_k;  // backward: dq, dk
    const void *dout_q, *dout_k;
    float *partial;       // [blocks, 2, d]
    int32_t *status;
    int32_t tokens, H_q, H_k, d, norm, rot, interleaved, table_rows;
    float eps, q_scale;
};

constexpr int kNormThreads = 128;
constexpr int kNormHeads = 4, kNormHeadsBack = 2;  // heads in flight per lane

template <typename IO>
__device__ __forceinline__ void norm_load8(const IO *p, float (&x)[8]) { load8(p, x); }
__device__ __forceinline__ void norm_store8(float *p, const float (&x)[8]) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void norm_store8(__nv_bfloat16 *p, const float (&x)[8]) { pack_store<__nv_bfloat16, 8>(p, pack_round<__nv_bfloat16, 8>(x)); }

template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// A token's rotation as a lane of its heads needs it.
struct Turn {
    float c[8], s[8];  // interleaved: four of each
    int partner;       // lane of the partner's values, for pairs half a rotation apart
    bool on;           // this lane's values turn
};

// false: a token without a valid position.
__device__ __forceinline__ bool norm_turn(const NormArgs &a, int token, int l, int base, Turn &t) {
    t.on = false, t.partner = base + l;
    if (a.rot == 0) return true;
    const int p = a.positions[token], half = a.rot / 2;
    if (p < 0 || p >= a.table_rows) {
        if (p >= 0 && l == 0 && a.status) atomicOr(a.status, DELTALOG_STATUS_BAD_POSITION);
        return false;
    }
    t.on = l * 8 < a.rot;
    if (!t.on) return true;
    const float *cos = a.cos + (size_t)p * half, *sin = a.sin + (size_t)p * half;
    if (a.interleaved) {
        const float4 c = __ldg(reinterpret_cast<const float4 *>(cos + l * 4)), s = __ldg(reinterpret_cast<const float4 *>(sin + l * 4));
        t.c[0] = c.x, t.c[1] = c.y, t.c[2] = c.z, t.c[3] = c.w, t.s[0] = s.x, t.s[1] = s.y, t.s[2] = s.z, t.s[3] = s.w;
        return true;
    }
    const bool first = l * 8 < half;
    const int i = first ? l * 8 : l * 8 - half;
    load8(cos + i, t.c);
    load8(sin + i, t.s);
    t.partner = base + (first ? l + half / 8 : l - half / 8);
    if (first)  // x[i] cos - x[i + half] sin, against x[i + half] cos + x[i] sin
#pragma unroll
        for (int e = 0; e < 8; ++e) t.s[e] = -t.s[e];
    return true;
}

// x turned by the token's angles, or back by them.  All lanes of the warp call it.
template <bool BACK>
__device__ __forceinline__ void norm_rotate(const NormArgs &a, const Turn &t, float (&x)[8]) {
    if (a.rot == 0) return;
    if (a.interleaved) {
        if (!t.on) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float u = x[2 * e], v = x[2 * e + 1], s = BACK ? -t.s[e] : t.s[e];
            x[2 * e] = u * t.c[e] - v * s, x[2 * e + 1] = v * t.c[e] + u * s;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float other = __shfl_sync(0xffffffffu, x[e], t.partner);
        if (t.on) x[e] = x[e] * t.c[e] + other * (BACK ? -t.s[e] : t.s[e]);
    }
}

// Which heads of which token a warp's work item is: HEADS * 32 / L of q or of k.
struct NormItem {
    int token, head, heads;  // first head and how many heads the tensor has
    bool is_k;
};
__host__ __device__ __forceinline__ int norm_chunks(int heads, int per) { return (heads + per - 1) / per; }
template <int L, int HEADS>
__device__ __forceinline__ NormItem norm_item(const NormArgs &a, long long item) {
    constexpr int per = HEADS * 32 / L;
    const int cq = norm_chunks(a.H_q, per), all = cq + norm_chunks(a.H_k, per);
    NormItem w;
    w.token = (int)(item / all);
    const int c = (int)(item - (long long)w.token * all);
    w.is_k = c >= cq;
    w.head = (w.is_k ? c - cq : c) * per;
    w.heads = w.is_k ? a.H_k : a.H_q;
    return w;
}
template <int L, int HEADS>
__host__ __device__ __forceinline__ long long norm_items(int tokens, int H_q, int H_k) {
    constexpr int per = HEADS * 32 / L;
    return (long long)tokens * (norm_chunks(H_q, per) + norm_chunks(H_k, per));
}

template <typename IO, int L>
__global__ void __launch_bounds__(kNormThreads) head_norm_forward_kernel(const NormArgs a) {
    constexpr int G = 32 / L;
    const int lane = threadIdx.x & 31, l = lane & (L - 1), group = lane / L;
    const long long item = (long long)blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
    if (item >= norm_items<L, kNormHeads>(a.tokens, a.H_q, a.H_k)) return;
    const NormItem w = norm_item<L, kNormHeads>(a, item);
    const bool in = l * 8 < a.d;
    const IO *x = static_cast<const IO *>(w.is_k ? a.k : a.q) + (size_t)w.token * (w.is_k ? a.k_stride : a.q_stride) + l * 8;
    IO *out = static_cast<IO *>(w.is_k ? a.out_k : a.out_q) + (size_t)w.token * w.heads * a.d + l * 8;
    float v[kNormHeads][8];
#pragma unroll
    for (int i = 0; i < kNormHeads; ++i) {
        const int h = w.head + i * G + group;
        if (in && h < w.heads) {
            norm_load8(x + (size_t)h * a.d, v[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        }
    }
    Turn turn;
    const bool ok = norm_turn(a, w.token, l, group * L, turn);
    float weight[8];
    const float *wp = w.is_k ? a.w_k : a.w_q;
    if (wp && in) load8(wp + l * 8, weight);
    const float scale = w.is_k ? 1.f : a.q_scale, c = a.norm == DELTALOG_NORM_RMS ? __fdividef(1.f, (float)a.d) : 1.f;
#pragma unroll
    for (int i = 0; i < kNormHeads; ++i) {
        const int h = w.head + i * G + group;
        if (a.norm != DELTALOG_NORM_NONE) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(v[i][e], v[i][e], ss);
            const float r = rsqrtf(fmaf(c, lanes_sum<L>(ss), a.eps));
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= wp && in ? r * weight[e] : r;
        }
        norm_rotate<false>(a, turn, v[i]);
        if (in && h < w.heads) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = ok ? v[i][e] * scale : 0.f;
            norm_store8(out + (size_t)h * a.d, v[i]);
        }
    }
}

template <typename IO, int L>
__global__ void __launch_bounds__(kNormThreads, 4) head_norm_backward_kernel(const NormArgs a) {
    constexpr int G = 32 / L;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane & (L - 1), group = lane / L;
    const bool in = l * 8 < a.d, weighted = a.w_q != nullptr;
    const float c = a.norm == DELTALOG_NORM_RMS ? __fdividef(1.f, (float)a.d) : 1.f;
    const long long items = norm_items<L, kNormHeadsBack>(a.tokens, a.H_q, a.H_k);
    float dw[2][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[0][e] = dw[1][e] = 0.f;
    for (long long item = (long long)blockIdx.x * (kNormThreads / 32) + warp; item < items; item += (long long)gridDim.x * (kNormThreads / 32)) {
        const NormItem w = norm_item<L, kNormHeadsBack>(a, item);
        const IO *x = static_cast<const IO *>(w.is_k ? a.k : a.q) + (size_t)w.token * (w.is_k ? a.k_stride : a.q_stride) + l * 8;
        const size_t at = (size_t)w.token * w.heads * a.d + l * 8;
        const IO *dout = static_cast<const IO *>(w.is_k ? a.dout_k : a.dout_q) + at;
        IO *dx = static_cast<IO *>(w.is_k ? a.out_k : a.out_q) + at;
        float v[kNormHeadsBack][8], g[kNormHeadsBack][8];
#pragma unroll
        for (int i = 0; i < kNormHeadsBack; ++i) {
            const int h = w.head + i * G + group;
            if (in && h < w.heads) {
                norm_load8(dout + (size_t)h * a.d, g[i]);
                if (a.norm != DELTALOG_NORM_NONE) norm_load8(x + (size_t)h * a.d, v[i]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = g[i][e] = 0.f;
            }
        }
        Turn turn;
        const bool ok = norm_turn(a, w.token, l, group * L, turn);
        float weight[8];
        const float *wp = w.is_k ? a.w_k : a.w_q;
#pragma unroll
        for (int e = 0; e < 8; ++e) weight[e] = 1.f;
        if (wp && in) load8(wp + l * 8, weight);
        const float scale = w.is_k ? 1.f : a.q_scale;
#pragma unroll
        for (int i = 0; i < kNormHeadsBack; ++i) {
            const int h = w.head + i * G + group;
            norm_rotate<true>(a, turn, g[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) g[i][e] = ok ? g[i][e] * scale : 0.f;
            if (a.norm != DELTALOG_NORM_NONE) {
                float ss = 0.f, gx = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss = fmaf(v[i][e], v[i][e], ss), gx = fmaf(g[i][e] * weight[e], v[i][e], gx);
                const float r = rsqrtf(fmaf(c, lanes_sum<L>(ss), a.eps)), k = lanes_sum<L>(gx) * c * r * r;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (weighted && ok) {  // (a token without a position may hold anything)
                        if (w.is_k) dw[1][e] = fmaf(g[i][e], v[i][e] * r, dw[1][e]);
                        else dw[0][e] = fmaf(g[i][e], v[i][e] * r, dw[0][e]);
                    }
                    g[i][e] = ok ? r * (g[i][e] * weight[e] - k * v[i][e]) : 0.f;
                }
            }
            if (in && h < w.heads) norm_store8(dx + (size_t)h * a.d, g[i]);
        }
    }
    if (!weighted) return;
    // the block's sums: over the heads side by side in a warp, then over its warps
    __shared__ float sums[kNormThreads / 32][2][256];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float s = dw[n][e];
#pragma unroll
            for (int o = L; o < 32; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (group == 0 && in) sums[warp][n][l * 8 + e] = s;
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.d; i += kNormThreads) {
        const int n = i / a.d, e = i - n * a.d;
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kNormThreads / 32; ++k) s += sums[k][n][e];
        a.partial[(size_t)blockIdx.x * 2 * a.d + i] = s;
    }
}

__global__ void __launch_bounds__(256) head_norm_reduce_kernel(const float *partial, int blocks, int d, float *dw_q, float *dw_k) {
    const float s = column_sum(partial, blocks, 2 * d);
    const int i = blockIdx.x * 32 + threadIdx.x;
    if (threadIdx.x >= 32 || i >= 2 * d) return;
    if (i < d) dw_q[i] = s;
    else if (dw_k) dw_k[i - d] = s;
}

}  // namespace deltalog
