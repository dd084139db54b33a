// The plan of a serving or training step, from the lengths of its requests: token and chunk offsets, the chunk and
// token tables, and one slot list per call that a row can go through.
//
// Two exclusive scans and two expansions.  Up to kPlanShared rows every CTA scans all lengths for itself into shared
// memory and then writes its share of the tables: the scan costs a CTA a few microseconds whatever the grid, so one
// launch without any exchange between CTAs beats a scan launch in front of an expansion launch.  More rows than shared
// memory holds: one CTA scans into the plan's own offset arrays and a second launch expands from there.
#pragma once

#include "common.cuh"

namespace deltalog {

constexpr int kPlanThreads = 512;
constexpr int kPlanShared = 24576;

struct PlanArgs {
    const int32_t *lens, *slots, *log_len;
    int32_t n, H, cap, num_slots, decode_rows, max_tokens, max_chunks;
    int32_t *starts, *chunk_starts, *chunk_seq, *token_seq, *scan_slots, *append_slots, *merge_slots, *totals;
};

// Exclusive scan over the CTA's threads; `total` is the sum of all.
__device__ __forceinline__ unsigned long long plan_scan(unsigned long long x, unsigned long long *warps, unsigned long long &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    unsigned long long s = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
    }
    __syncthreads();
    if (lane == 31) warps[warp] = s;
    __syncthreads();
    unsigned long long before = 0, all = 0;
    for (int w = 0; w < nw; ++w) {
        if (w < warp) before += warps[w];
        all += warps[w];
    }
    total = all;
    return before + s - x;
}

// Offsets of all rows into `starts` and `chunk_starts` ([n + 1], shared or global).  A row whose tokens would end behind
// max_tokens is dropped (it counts as empty); all rows behind it that have tokens are dropped with it.
__device__ __forceinline__ void plan_offsets(const PlanArgs &a, int32_t *starts, int32_t *chunk_starts, bool write_totals) {
    __shared__ unsigned long long warps[32];
    const int per = (a.n + blockDim.x - 1) / blockDim.x, first = threadIdx.x * per, last = min(a.n, first + per);
    unsigned long long sum = 0, total;
    for (int i = first; i < last; ++i) sum += (unsigned long long)max(a.lens[i], 0);
    unsigned long long at = plan_scan(sum, warps, total);
    const unsigned long long most = (unsigned long long)a.max_tokens;
    unsigned long long both = 0, rows = 0;  // tokens << 32 | chunks;  scan rows << 32 | decode rows
    {
        unsigned long long s = at;
        for (int i = first; i < last; ++i) {
            int len = max(a.lens[i], 0);
            if (s + len > most) len = 0, s = most + 1;
            s += len;
            both += ((unsigned long long)len << 32) + (len + DELTALOG_SCAN_CHUNK - 1) / DELTALOG_SCAN_CHUNK;
            if (len > 0) rows += a.decode_rows && len == 1 ? 1ull : 1ull << 32;
        }
    }
    unsigned long long off = plan_scan(both, warps, total);
    for (int i = first; i < last; ++i) {
        int len = max(a.lens[i], 0);
        if (at + len > most) len = 0, at = most + 1;
        at += len;
        starts[i] = (int32_t)(off >> 32);
        chunk_starts[i] = (int32_t)(off & 0xffffffffu);
        off += ((unsigned long long)len << 32) + (len + DELTALOG_SCAN_CHUNK - 1) / DELTALOG_SCAN_CHUNK;
    }
    if (threadIdx.x == 0) {
        starts[a.n] = (int32_t)(total >> 32);
        chunk_starts[a.n] = (int32_t)(total & 0xffffffffu);
    }
    if (write_totals) {
        unsigned long long count;
        plan_scan(rows, warps, count);
        if (threadIdx.x == 0) {
            a.totals[0] = (int32_t)(total >> 32);
            a.totals[1] = (int32_t)(total & 0xffffffffu);
            a.totals[2] = (int32_t)(count >> 32);
            a.totals[3] = (int32_t)(count & 0xffffffffu);
        }
    }
    __syncthreads();
}

// The last row whose offset is at most x (empty rows share their offset with the row behind them, which is found).
__device__ __forceinline__ int plan_find(const int32_t *offsets, int n, int x) {
    int lo = 0, hi = n;  // offsets[lo] <= x < offsets[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (offsets[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void plan_tables(const PlanArgs &a, const int32_t *starts, const int32_t *chunk_starts) {
    const int stride = gridDim.x * blockDim.x, first = blockIdx.x * blockDim.x + threadIdx.x;
    for (int i = first; i < a.n; i += stride) {
        const int len = starts[i + 1] - starts[i], slot = a.slots ? a.slots[i] : i;
        const bool one = a.decode_rows && len == 1;
        bool full = false;
        if (one && a.log_len && slot >= 0 && slot < a.num_slots) full = a.log_len[(size_t)slot * a.H] >= a.cap;
        a.scan_slots[i] = len > 0 && !one ? slot : -1;
        if (a.append_slots) a.append_slots[i] = one && !full ? slot : -1;
        if (a.merge_slots) a.merge_slots[i] = one && full ? slot : -1;
    }
    const int chunks = chunk_starts[a.n];
    for (int i = first; i < a.max_chunks; i += stride) a.chunk_seq[i] = i < chunks ? plan_find(chunk_starts, a.n, i) : -1;
    if (!a.token_seq) return;
    const int tokens = starts[a.n];
    // four tokens per thread and step, neighbours side by side: one search, then along the rows
    for (long long q = first; q * 4 < a.max_tokens; q += stride) {
        const int t0 = (int)q * 4;
        int out[4], row = t0 < tokens ? plan_find(starts, a.n, t0) : 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = t0 + e;
            if (t < tokens)
                while (starts[row + 1] <= t) ++row;
            out[e] = t < tokens ? row : -1;
        }
        if (t0 + 4 <= a.max_tokens) {
            *reinterpret_cast<int4 *>(a.token_seq + t0) = make_int4(out[0], out[1], out[2], out[3]);
        } else {
            for (int e = 0; t0 + e < a.max_tokens; ++e) a.token_seq[t0 + e] = out[e];
        }
    }
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanArgs a) {
    extern __shared__ int32_t offsets[];
    int32_t *starts = offsets, *chunk_starts = offsets + a.n + 1;
    plan_offsets(a, starts, chunk_starts, blockIdx.x == 0);
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i <= a.n; i += gridDim.x * blockDim.x) {
        a.starts[i] = starts[i];
        a.chunk_starts[i] = chunk_starts[i];
    }
    plan_tables(a, starts, chunk_starts);
}

__global__ void __launch_bounds__(1024) plan_offsets_kernel(const PlanArgs a) { plan_offsets(a, a.starts, a.chunk_starts, true); }
__global__ void __launch_bounds__(kPlanThreads) plan_tables_kernel(const PlanArgs a) { plan_tables(a, a.starts, a.chunk_starts); }

}  // namespace deltalog
