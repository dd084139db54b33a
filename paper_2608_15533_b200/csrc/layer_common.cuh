// Pieces shared by the operators around the scan (causal convolution, state space scan, norm of heads): vectors of a few
// elements, the row of a packed token, elementary functions.
#pragma once

#include "common.cuh"

namespace deltalog {

// V consecutive elements kept as they are in memory.
template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T e[V]; };

template <typename T, int V>
__device__ __forceinline__ Pack<T, V> pack_load(const T *p) { return *reinterpret_cast<const Pack<T, V> *>(p); }
template <typename T, int V>
__device__ __forceinline__ void pack_store(T *p, const Pack<T, V> &v) { *reinterpret_cast<Pack<T, V> *>(p) = v; }
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> pack_zero() {
    Pack<T, V> v;
#pragma unroll
    for (int i = 0; i < V; ++i) v.e[i] = from_f32<T>(0.f);
    return v;
}
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> pack_round(const float (&x)[V]) {
    Pack<T, V> v;
#pragma unroll
    for (int i = 0; i < V; ++i) v.e[i] = from_f32<T>(x[i]);
    return v;
}

// 1 / (1 + e^-x): 0 and 1 at the infinities.
__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }

// The packed rows of a plan.
struct Rows {
    const int32_t *starts, *token_seq;
    int32_t n;
    // Row of token t, -1 behind the last sequence.  Without a token map: the last row whose first token is at most t (empty
    // rows share their offset with the row behind them, which is found).
    __device__ __forceinline__ int of(int t) const {
        if (token_seq) return token_seq[t];
        if (t >= starts[n]) return -1;
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (starts[mid] <= t) lo = mid;
            else hi = mid;
        }
        return lo;
    }
};

// Column sums of a block's 32 columns over the rows of partial [rows, cols], eight threads a column, in a fixed order; the
// sum arrives at the threads of the first warp (column blockIdx.x * 32 + lane), 0 elsewhere.  Blocks of 256 threads.
__device__ __forceinline__ float column_sum(const float *partial, long long rows, int cols) {
    __shared__ float sums[8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < cols)
#pragma unroll 8
        for (long long r = warp; r < rows; r += 8) s += partial[(size_t)r * cols + c];
    sums[warp][lane] = s;
    __syncthreads();
    if (warp) return 0.f;
#pragma unroll
    for (int i = 1; i < 8; ++i) s += sums[i][lane];
    return s;
}

}  // namespace deltalog
