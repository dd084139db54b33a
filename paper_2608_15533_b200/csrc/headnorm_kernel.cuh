// Norm, rotation and scale of query and key heads, both tensors in one launch, and its gradients.
//     n = w x r,  r = 1 / sqrt(c sum x^2 + eps)  (c = 1 for unit length, 1 / d for the root of the mean square)
//     y = scale (n turned pair by pair)
// Backward, with g = scale (dy turned back):  dw = sum g x r,  dx = r (g w - c r^2 x sum(g w x)).
//
// Bound by HBM: every value is read once and written once.  L lanes hold a head, sixteen values each: two runs of eight that are
// half a rotation apart (or neighbours, for interleaved pairs and behind the rotated part), so that a lane turns its own values and
// loads 16 bytes at a time.  A warp takes one token and several of its heads, and walks over such items with two more on their way
// in shared memory.  The sums over a head are butterflies over its lanes.
// 16k tokens x 40 heads of 128, 16-bit: 64 us (5.2 TB/s, 0.80 of a copy), gradients 117 us (4.3 TB/s; 65 % of the issue slots, 32
// instructions a value, forward 19) and 8 for the weights' sums, whose eight blocks are bound by latency.
// (Pairs exchanged between lanes: 103 and 355 us; one item a warp with its loads in registers: 80 and 149.)
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
constexpr int kNormHeads = 2, kNormHeadsBack = 1;  // heads of a lane's item
// CTAs of a wave on an SM, forward and of the gradients, by their registers, or with fp32 by the forward pass's ring (a grid for five, of
// which four fit, left a fifth for a second wave: 16k x 40 heads of 128 186 us where 168 are taken).
template <typename IO> constexpr int kNormCtas = sizeof(IO) == 4 ? 4 : 5;
template <typename IO> constexpr int kNormBackCtas = sizeof(IO) == 4 ? 3 : 4;
constexpr size_t kNormShared = 228 * 1024, kNormReserved = 1024;  // bytes of an SM, and of every CTA for the system

// Where a lane's two runs of eight values are in a head, and whether they are.
struct NormAt {
    int lo, hi;
    bool has_lo, has_hi;
};
__device__ __forceinline__ NormAt norm_at(const NormArgs &a, int l) {
    NormAt at{l * 16, l * 16 + 8, false, false};
    if (!a.interleaved && l * 16 < a.rot) at.lo = l * 8, at.hi = a.rot / 2 + l * 8;
    at.has_lo = l * 16 < a.d, at.has_hi = l * 16 + 8 < a.d;  // (the rotated part is a multiple of sixteen)
    return at;
}
template <typename IO>
__device__ __forceinline__ void norm_load(const IO *p, const NormAt &at, bool there, Pack<IO, 8> (&x)[2]) {
    x[0] = x[1] = pack_zero<IO, 8>();
    constexpr int V = 16 / sizeof(IO);
#pragma unroll
    for (int e = 0; e < 8; e += V) {
        if (there && at.has_lo) *reinterpret_cast<uint4 *>(x[0].e + e) = *reinterpret_cast<const uint4 *>(p + at.lo + e);
        if (there && at.has_hi) *reinterpret_cast<uint4 *>(x[1].e + e) = *reinterpret_cast<const uint4 *>(p + at.hi + e);
    }
}
// Values on their way: a lane copies its own sixteen into shared memory and reads nothing but its own, so that a wait for its own copies
// is all it needs.  Runs that a lane does not have are cleared once, before the first copy.
constexpr int kNormStages = 3;
template <typename IO> using NormSlot = Pack<IO, 8>[2][32];  // a head of a warp: two runs a lane
template <typename IO>
__device__ __forceinline__ void norm_copy(NormSlot<IO> &to, const IO *p, const NormAt &at, bool there, int lane) {
    constexpr int V = 16 / sizeof(IO);
#pragma unroll
    for (int e = 0; e < 8; e += V) {
        if (there && at.has_lo) cp_async16(to[0][lane].e + e, p + at.lo + e);
        if (there && at.has_hi) cp_async16(to[1][lane].e + e, p + at.hi + e);
    }
}
template <typename IO>
__device__ __forceinline__ void norm_clear(NormSlot<IO> &to, const NormAt &at, int lane) {
    if (!at.has_lo) to[0][lane] = pack_zero<IO, 8>();
    if (!at.has_hi) to[1][lane] = pack_zero<IO, 8>();
}
template <typename IO>
__device__ __forceinline__ void norm_read(const NormSlot<IO> &from, int lane, float (&f)[16]) {
    const Pack<IO, 8> v[2] = {from[0][lane], from[1][lane]};
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] = to_f32(v[e / 8].e[e % 8]);
}
template <int N>
__device__ __forceinline__ void norm_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }

template <typename IO>
__device__ __forceinline__ void norm_floats(const Pack<IO, 8> (&x)[2], float (&f)[16]) {
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] = to_f32(x[e / 8].e[e % 8]);
}
template <typename IO>
__device__ __forceinline__ void norm_store(IO *p, const NormAt &at, const float (&x)[16]) {
    constexpr int V = 16 / sizeof(IO);
    Pack<IO, 8> v[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e / 8].e[e % 8] = from_f32<IO>(x[e]);
#pragma unroll
    for (int e = 0; e < 8; e += V) {
        if (at.has_lo) *reinterpret_cast<uint4 *>(p + at.lo + e) = *reinterpret_cast<const uint4 *>(v[0].e + e);
        if (at.has_hi) *reinterpret_cast<uint4 *>(p + at.hi + e) = *reinterpret_cast<const uint4 *>(v[1].e + e);
    }
}
__device__ __forceinline__ void norm_weights(const float *w, const NormAt &at, float (&f)[16]) {
#pragma unroll
    for (int e = 0; e < 16; ++e) f[e] = 1.f;
    if (!w) return;
    Pack<float, 8> v[2];
    norm_load(w, at, true, v);
    norm_floats(v, f);
}

template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// A token's rotation as a lane of its heads needs it: the angles of its eight pairs.
struct Turn {
    float c[8], s[8];
    bool on;  // this lane's values turn
};

// false: a token without a valid position.
__device__ __forceinline__ bool norm_turn(const NormArgs &a, int p, int l, Turn &t) {
    t.on = false;
    if (a.rot == 0) return true;
    if (p < 0 || p >= a.table_rows) {
        if (p >= 0 && l == 0 && a.status) atomicOr(a.status, DELTALOG_STATUS_BAD_POSITION);
        return false;
    }
    t.on = l * 16 < a.rot;
    if (t.on) {
        load8(a.cos + (size_t)p * (a.rot / 2) + l * 8, t.c);
        load8(a.sin + (size_t)p * (a.rot / 2) + l * 8, t.s);
    }
    return true;
}

// x turned by the token's angles, or back by them.
template <bool BACK>
__device__ __forceinline__ void norm_rotate(const NormArgs &a, const Turn &t, float (&x)[16]) {
    if (!t.on) return;
    auto turn = [&](float &u, float &v, int e) {
        const float u0 = u, s = BACK ? -t.s[e] : t.s[e];
        u = u0 * t.c[e] - v * s, v = v * t.c[e] + u0 * s;
    };
    if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn(x[2 * e], x[2 * e + 1], e);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn(x[e], x[8 + e], e);
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

// A warp walks over its items, two of which are on their way while one is computed.
template <typename IO, int L>
__global__ void __launch_bounds__(kNormThreads, kNormCtas<IO>) head_norm_forward_kernel(const NormArgs a) {
    constexpr int G = 32 / L, per = kNormHeads * G, S = kNormStages;
    __shared__ NormSlot<IO> ring[kNormThreads / 32][S][kNormHeads];
    static_assert(kNormCtas<IO> * (sizeof(ring) + kNormReserved) <= kNormShared, "a wave of CTAs fits");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane & (L - 1), group = lane / L;
    const NormAt at = norm_at(a, l);
    const unsigned cq = (a.H_q + per - 1) / per, chunks = cq + (a.H_k + per - 1) / per;
    const long long items = (long long)a.tokens * chunks, step = (long long)gridDim.x * (kNormThreads / 32);  // (fewer than 2^31)
    const float c = a.norm == DELTALOG_NORM_RMS ? 1.f / (float)a.d : 1.f;
    long long item = (long long)blockIdx.x * (kNormThreads / 32) + warp;
    if (item >= items) return;
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int i = 0; i < kNormHeads; ++i) norm_clear<IO>(ring[warp][s][i], at, lane);
    int position[S];  // of the items on their way, the next first
    auto fetch = [&](long long item, int stage, int &position) {
        if (item < items) {
            const unsigned token = (unsigned)item / chunks, chunk = (unsigned)item % chunks;
            const NormSide<IO> t = norm_side<IO>(a, chunk >= cq);
            const int head = (int)(chunk >= cq ? chunk - cq : chunk) * per + group;
            const IO *x = t.x + token * t.stride;
            position = a.rot ? a.positions[token] : 0;
#pragma unroll
            for (int i = 0; i < kNormHeads; ++i) norm_copy(ring[warp][stage][i], x + (head + i * G) * a.d, at, head + i * G < t.heads, lane);
        }
        cp_async_commit();
    };
#pragma unroll
    for (int s = 0; s < S - 1; ++s) fetch(item + s * step, s, position[s]);
    for (int stage = 0; item < items; item += step, stage = stage == S - 1 ? 0 : stage + 1) {
        Turn turn;
        const bool ok = norm_turn(a, position[0], l, turn);
        fetch(item + (S - 1) * step, stage == 0 ? S - 1 : stage - 1, position[S - 1]);
#pragma unroll
        for (int s = 0; s < S - 1; ++s) position[s] = position[s + 1];
        const unsigned token = (unsigned)item / chunks, chunk = (unsigned)item % chunks;
        const NormSide<IO> t = norm_side<IO>(a, chunk >= cq);
        const int head = (int)(chunk >= cq ? chunk - cq : chunk) * per + group;
        float weight[16];
        norm_weights(t.w, at, weight);
        norm_wait<S - 1>();
        IO *out = t.out + (size_t)token * t.heads * a.d;
#pragma unroll
        for (int i = 0; i < kNormHeads; ++i) {
            float v[16], r = t.scale;
            norm_read<IO>(ring[warp][stage][i], lane, v);
            if (a.norm != DELTALOG_NORM_NONE) {
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) ss = fmaf(v[e], v[e], ss);
                r *= rsqrtf(fmaf(c, lanes_sum<L>(ss), a.eps));
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] *= r * weight[e];
            norm_rotate<false>(a, turn, v);
            if (head + i * G < t.heads) {
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = ok ? v[e] : 0.f;
                norm_store(out + (head + i * G) * a.d, at, v);
            }
        }
    }
}

// A warp walks over its items of q, then over those of k, with the weights' gradient in registers and two items on their way.
template <typename IO, int L>
__global__ void __launch_bounds__(kNormThreads, kNormBackCtas<IO>) head_norm_backward_kernel(const NormArgs a) {
    constexpr int G = 32 / L, per = G, S = kNormStages;  // one head a lane
    __shared__ NormSlot<IO> ring[kNormThreads / 32][S][2];  // gradient, value
    static_assert(kNormBackCtas<IO> * (sizeof(ring) + kNormReserved) <= kNormShared, "a wave of CTAs fits");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, l = lane & (L - 1), group = lane / L;
    const bool weighted = a.w_q != nullptr, normed = a.norm != DELTALOG_NORM_NONE;
    const NormAt at = norm_at(a, l);
    const float c = a.norm == DELTALOG_NORM_RMS ? 1.f / (float)a.d : 1.f;
    const long long first = (long long)blockIdx.x * (kNormThreads / 32) + warp, step = (long long)gridDim.x * (kNormThreads / 32);
    for (int side = 0; side < 2; ++side) {
        const NormSide<IO> t = norm_side<IO>(a, side == 1);
        const unsigned chunks = (t.heads + per - 1) / per;
        const long long items = (long long)a.tokens * chunks;  // (fewer than 2^31)
        float weight[16], dw[16];
        norm_weights(t.w, at, weight);
#pragma unroll
        for (int e = 0; e < 16; ++e) dw[e] = 0.f;
        norm_wait<0>();
        __syncthreads();  // (the ring held the other side's sums)
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                norm_clear<IO>(ring[warp][s][i], at, lane);
                if (i && !normed) ring[warp][s][i][0][lane] = ring[warp][s][i][1][lane] = pack_zero<IO, 8>();
            }
        int position[S];  // of the items on their way, the next first
        auto fetch = [&](long long item, int stage, int &position) {
            if (item < items) {
                const unsigned token = (unsigned)item / chunks;
                const int head = (int)((unsigned)item % chunks) * per + group;
                const bool there = head < t.heads;
                position = a.rot ? a.positions[token] : 0;
                norm_copy(ring[warp][stage][0], t.dout + (size_t)token * t.heads * a.d + head * a.d, at, there, lane);
                norm_copy(ring[warp][stage][1], t.x + token * t.stride + head * a.d, at, there && normed, lane);
            }
            cp_async_commit();
        };
#pragma unroll
        for (int s = 0; s < S - 1; ++s) fetch(first + s * step, s, position[s]);
        int stage = 0;
        for (long long item = first; item < items; item += step, stage = stage == S - 1 ? 0 : stage + 1) {
            Turn turn;
            const bool ok = norm_turn(a, position[0], l, turn);
            fetch(item + (S - 1) * step, stage == 0 ? S - 1 : stage - 1, position[S - 1]);
#pragma unroll
            for (int s = 0; s < S - 1; ++s) position[s] = position[s + 1];
            const unsigned token = (unsigned)item / chunks;
            const int head = (int)((unsigned)item % chunks) * per + group;
            norm_wait<S - 1>();
            float v[16], g[16];
            norm_read<IO>(ring[warp][stage][0], lane, g);
            norm_read<IO>(ring[warp][stage][1], lane, v);
            float ss = 0.f, gx = 0.f;
            if (normed) {
#pragma unroll
                for (int e = 0; e < 16; ++e) ss = fmaf(v[e], v[e], ss);
                ss = lanes_sum<L>(ss);
            }
            norm_rotate<true>(a, turn, g);
#pragma unroll
            for (int e = 0; e < 16; ++e) g[e] *= t.scale;
            if (normed) {
#pragma unroll
                for (int e = 0; e < 16; ++e) gx = fmaf(g[e] * weight[e], v[e], gx);
                const float r = rsqrtf(fmaf(c, ss, a.eps)), k = lanes_sum<L>(gx) * c * r * r * r;
                if (weighted && ok && head < t.heads)  // (a token without a position may hold anything, and so may a stage without a head)
#pragma unroll
                    for (int e = 0; e < 16; ++e) dw[e] = fmaf(g[e], v[e] * r, dw[e]);
#pragma unroll
                for (int e = 0; e < 16; ++e) g[e] = fmaf(r * weight[e], g[e], -k * v[e]);
            }
            if (head < t.heads) {
#pragma unroll
                for (int e = 0; e < 16; ++e) g[e] = ok ? g[e] : 0.f;
                norm_store(t.out + ((size_t)token * t.heads + head) * a.d, at, g);
            }
        }
        if (!weighted) continue;
        // the block's sums: over the heads side by side in a warp, then over its warps
        norm_wait<0>();
        __syncthreads();
        auto sums = reinterpret_cast<float (*)[256]>(&ring);
        static_assert(sizeof(ring) >= sizeof(float) * 256 * (kNormThreads / 32), "the sums fit");
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            float s = dw[e];
#pragma unroll
            for (int o = L; o < 32; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            if (group == 0 && (e < 8 ? at.has_lo : at.has_hi)) sums[warp][(e < 8 ? at.lo : at.hi - 8) + e] = s;
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
