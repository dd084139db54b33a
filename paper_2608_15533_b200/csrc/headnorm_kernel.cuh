// Norm, rotation and scale of query and key heads, both tensors in one launch, and its gradients.
//     n = w x r,  r = 1 / sqrt(c sum x^2 + eps)  (c = 1 for unit length, 1 / d for the root of the mean square)
//     y = scale (n turned pair by pair)
// Backward, with g = scale (dy turned back):  dw = sum g x r,  dx = r (g w - c r^2 x sum(g w x)).
//
// Bound by HBM: every value is read once and written once.  L lanes hold a head, eight values each: two runs of four that are
// half a rotation apart (or neighbours, for interleaved pairs and behind the rotated part), so that a lane turns its own values.  A
// warp takes one token and several of its heads: the token's cosines and sines are loaded once for all of them, and several heads a
// lane are in flight.  The sums over a head are butterflies over its lanes.
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

// Where a lane's two runs of four values are in a head.
struct NormAt { int lo, hi; };
__device__ __forceinline__ NormAt norm_at(const NormArgs &a, int l) {
    if (!a.interleaved && l * 8 < a.rot) return {l * 4, a.rot / 2 + l * 4};
    return {l * 8, l * 8 + 4};
}
template <typename IO>
__device__ __forceinline__ void norm_load(const IO *p, NormAt at, float (&x)[8]) {
    float lo[4], hi[4];
    load_vec<IO, 4>(p + at.lo, lo);
    load_vec<IO, 4>(p + at.hi, hi);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = lo[e], x[4 + e] = hi[e];
}
template <typename IO>
__device__ __forceinline__ void norm_store(IO *p, NormAt at, const float (&x)[8]) {
    const float lo[4] = {x[0], x[1], x[2], x[3]}, hi[4] = {x[4], x[5], x[6], x[7]};
    pack_store<IO, 4>(p + at.lo, pack_round<IO, 4>(lo));
    pack_store<IO, 4>(p + at.hi, pack_round<IO, 4>(hi));
}

template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// A token's rotation as a lane of its heads needs it: the angles of its four pairs.
struct Turn {
    float c[4], s[4];
    bool on;  // this lane's values turn
};

// false: a token without a valid position.
__device__ __forceinline__ bool norm_turn(const NormArgs &a, int token, int l, Turn &t) {
    t.on = false;
    if (a.rot == 0) return true;
    const int p = a.positions[token];
    if (p < 0 || p >= a.table_rows) {
        if (p >= 0 && l == 0 && a.status) atomicOr(a.status, DELTALOG_STATUS_BAD_POSITION);
        return false;
    }
    t.on = l * 8 < a.rot;
    if (t.on) {
        load_vec<float, 4>(a.cos + (size_t)p * (a.rot / 2) + l * 4, t.c);
        load_vec<float, 4>(a.sin + (size_t)p * (a.rot / 2) + l * 4, t.s);
    }
    return true;
}

// x turned by the token's angles, or back by them.
template <bool BACK>
__device__ __forceinline__ void norm_rotate(const NormArgs &a, const Turn &t, float (&x)[8]) {
    if (!t.on) return;
    auto turn = [&](float &u, float &v, int e) {
        const float u0 = u, s = BACK ? -t.s[e] : t.s[e];
        u = u0 * t.c[e] - v * s, v = v * t.c[e] + u0 * s;
    };
    if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) turn(x[2 * e], x[2 * e + 1], e);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) turn(x[e], x[4 + e], e);
    }
}

// Work items of one tensor: HEADS * 32 / L heads of a token each.
template <int L, int HEADS>
__host__ __device__ __forceinline__ long long norm_items(int tokens, int heads) {
    constexpr int per = HEADS * 32 / L;
    return (long long)tokens * ((heads + per - 1) / per);
}

// One tensor of the two, as an item sees it.
template <typename IO>
struct NormSide {
    const IO *x, *dout;
    IO *out;
    long long stride;
    const float *w;
    float scale;
    int heads;
};
template <typename IO>
__device__ __forceinline__ NormSide<IO> norm_side(const NormArgs &a, bool is_k) {
    if (is_k) return {static_cast<const IO *>(a.k), static_cast<const IO *>(a.dout_k), static_cast<IO *>(a.out_k), a.k_stride, a.w_k, 1.f, a.H_k};
    return {static_cast<const IO *>(a.q), static_cast<const IO *>(a.dout_q), static_cast<IO *>(a.out_q), a.q_stride, a.w_q, a.q_scale, a.H_q};
}

template <typename IO, int L>
__global__ void __launch_bounds__(kNormThreads) head_norm_forward_kernel(const NormArgs a) {
    constexpr int G = 32 / L, per = kNormHeads * G;
    const int lane = threadIdx.x & 31, l = lane & (L - 1), group = lane / L;
    const long long item = (long long)blockIdx.x * (kNormThreads / 32) + (threadIdx.x >> 5);
    const int cq = (a.H_q + per - 1) / per, chunks = cq + (a.H_k + per - 1) / per;
    const int token = (int)(item / chunks), chunk = (int)(item - (long long)token * chunks);
    if (token >= a.tokens) return;
    const NormSide<IO> t = norm_side<IO>(a, chunk >= cq);
    const int head = (chunk >= cq ? chunk - cq : chunk) * per + group;
    const bool in = l * 8 < a.d;
    const NormAt at = norm_at(a, l);
    const IO *x = t.x + (size_t)token * t.stride;
    IO *out = t.out + (size_t)token * t.heads * a.d;
    float v[kNormHeads][8];
#pragma unroll
    for (int i = 0; i < kNormHeads; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        if (in && head + i * G < t.heads) norm_load(x + (head + i * G) * a.d, at, v[i]);
    }
    Turn turn;
    const bool ok = norm_turn(a, token, l, turn);
    float weight[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) weight[e] = 1.f;
    if (t.w && in) norm_load(t.w, at, weight);
    const float c = a.norm == DELTALOG_NORM_RMS ? 1.f / (float)a.d : 1.f;
#pragma unroll
    for (int i = 0; i < kNormHeads; ++i) {
        float r = t.scale;
        if (a.norm != DELTALOG_NORM_NONE) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(v[i][e], v[i][e], ss);
            r *= rsqrtf(fmaf(c, lanes_sum<L>(ss), a.eps));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] *= r * weight[e];
        norm_rotate<false>(a, turn, v[i]);
        if (in && head + i * G < t.heads) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = ok ? v[i][e] : 0.f;
            norm_store(out + (head + i * G) * a.d, at, v[i]);
        }
    }
}

// With weights the grid is fixed and every warp walks over its items of q, then over those of k, with the weights' gradient in
// registers; without, every warp has one item.
template <typename IO, int L>
__global__ void __launch_bounds__(kNormThreads) head_norm_backward_kernel(const NormArgs a) {
    constexpr int G = 32 / L, per = kNormHeadsBack * G;
    __shared__ float sums[kNormThreads / 32][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane & (L - 1), group = lane / L;
    const bool in = l * 8 < a.d, weighted = a.w_q != nullptr;
    const NormAt at = norm_at(a, l);
    const float c = a.norm == DELTALOG_NORM_RMS ? 1.f / (float)a.d : 1.f;
    const long long first = (long long)blockIdx.x * (kNormThreads / 32) + warp, step = (long long)gridDim.x * (kNormThreads / 32);
    long long skipped = 0;  // items of the tensor in front
    for (int side = 0; side < 2; ++side) {
        const NormSide<IO> t = norm_side<IO>(a, side == 1);
        const int chunks = (t.heads + per - 1) / per;
        const long long items = (long long)a.tokens * chunks;
        float weight[8], dw[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) weight[e] = 1.f, dw[e] = 0.f;
        if (t.w && in) norm_load(t.w, at, weight);
        for (long long item = first - skipped; item < items; item += step) {
            if (item < 0) continue;
            const int token = (int)(item / chunks), head = (int)(item - (long long)token * chunks) * per + group;
            const IO *x = t.x + (size_t)token * t.stride;
            const size_t to = (size_t)token * t.heads * a.d;
            float v[kNormHeadsBack][8], g[kNormHeadsBack][8];
#pragma unroll
            for (int i = 0; i < kNormHeadsBack; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = g[i][e] = 0.f;
                if (in && head + i * G < t.heads) {
                    norm_load(t.dout + to + (head + i * G) * a.d, at, g[i]);
                    if (a.norm != DELTALOG_NORM_NONE) norm_load(x + (head + i * G) * a.d, at, v[i]);
                }
            }
            Turn turn;
            const bool ok = norm_turn(a, token, l, turn);
#pragma unroll
            for (int i = 0; i < kNormHeadsBack; ++i) {
                norm_rotate<true>(a, turn, g[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) g[i][e] *= t.scale;
                if (a.norm != DELTALOG_NORM_NONE) {
                    float ss = 0.f, gx = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) ss = fmaf(v[i][e], v[i][e], ss), gx = fmaf(g[i][e] * weight[e], v[i][e], gx);
                    const float r = rsqrtf(fmaf(c, lanes_sum<L>(ss), a.eps)), k = lanes_sum<L>(gx) * c * r * r * r;
                    if (weighted && ok)  // (a token without a position may hold anything)
#pragma unroll
                        for (int e = 0; e < 8; ++e) dw[e] = fmaf(g[i][e], v[i][e] * r, dw[e]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) g[i][e] = fmaf(r * weight[e], g[i][e], -k * v[i][e]);
                }
                if (in && head + i * G < t.heads) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) g[i][e] = ok ? g[i][e] : 0.f;
                    norm_store(static_cast<IO *>(t.out) + to + (head + i * G) * a.d, at, g[i]);
                }
            }
        }
        if (!weighted) {
            skipped += items;  // the items of both tensors in one row
            continue;
        }
        // the block's sums: over the heads side by side in a warp, then over its warps
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float s = dw[e];
#pragma unroll
            for (int o = L; o < 32; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (group == 0 && in) sums[warp][(e < 4 ? at.lo : at.hi - 4) + e] = s;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < a.d; i += kNormThreads) {
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < kNormThreads / 32; ++k) s += sums[k][i];
            a.partial[((size_t)blockIdx.x * 2 + side) * a.d + i] = s;
        }
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
