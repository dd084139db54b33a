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

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 1 / (1 + e^-x): 0 and 1 at the infinities.  The exponent of two is rounded once, which costs bits far below zero, where the result is
// small: 2e-7 of it at 0 as with expf, 3.6e-7 at -5, 1e-6 at -20, 3.9e-6 at -85 (expf: 2.4e-7 throughout).  A second word of the exponent would be
// one more product for every element of kernels that are short of issue slots; a sum or a norm of results does not see it.
__device__ __forceinline__ float sigmoid(float x) { return rcp_fast(1.f + exp2_fast(-1.4426950408889634f * x)); }

// Two neighbouring elements as floats, and back.
__device__ __forceinline__ float2 load2(const float *p) { return *reinterpret_cast<const float2 *>(p); }
__device__ __forceinline__ float2 load2(const __nv_bfloat16 *p) {
    const uint32_t v = *reinterpret_cast<const uint32_t *>(p);
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ void store2(float *p, float2 v) { *reinterpret_cast<float2 *>(p) = v; }
__device__ __forceinline__ void store2(__nv_bfloat16 *p, float2 v) { *reinterpret_cast<__nv_bfloat162 *>(p) = __float22bfloat162_rn(v); }
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

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

// Slots of U rows of a single-token call as the list has them, and -1 for rows that the call skips.  The list's entries are
// loaded together: one after the other, each behind the test of the one before, they would cost a trip to memory each.
template <int U>
__device__ __forceinline__ void step_slots(const int32_t *slots, int row, int end, int (&slot)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) slot[u] = slots ? slots[min(row + u, end - 1)] : row + u;
}
template <int U>
__device__ __forceinline__ void step_check(int row, int end, int num_slots, int32_t *status, int (&slot)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (row + u >= end) slot[u] = -1;
        if (slot[u] >= num_slots) {
            if ((threadIdx.x & 31) == 0 && status) atomicOr(status, DELTALOG_STATUS_BAD_SLOT);
            slot[u] = -1;
        }
    }
}

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
