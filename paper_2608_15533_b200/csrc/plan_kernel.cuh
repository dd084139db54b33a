// The plan of a serving or training step, from the lengths of its requests: token and chunk offsets, the chunk and
// token tables, and one slot list per call that a row can go through.
//
// Two exclusive scans and two expansions.  Up to kPlanShared rows every CTA scans all lengths for itself into shared
// memory and then writes its share of the tables: the scan costs a CTA a few microseconds whatever the grid, so one
// launch without any exchange between CTAs beats a scan launch in front of an expansion launch.  More rows than shared
// memory holds: one CTA scans into the plan's own offset arrays and a second launch expands from there.
// 512 requests with 50k tokens 8 us, 20k requests with 8M tokens 26 us (33 MB of tables: 1.3 TB/s, the scan in front is most of it),
// a few requests 5 us.
#pragma once

#include "common.cuh"

namespace deltalog {

constexpr int kPlanThreads = 1024;
constexpr int kPlanShared = 24576;

struct PlanArgs {
    const int32_t *lens, *slots, *log_len;
    int32_t n, H, cap, num_slots, decode_rows, max_tokens, max_chunks;
    int32_t *starts, *chunk_starts, *chunk_seq, *token_seq, *scan_slots, *append_slots, *merge_slots, *totals;
};

// Exclusive scans of two values over the CTA's threads; the totals come along.  `warps` [2][64]: one half per call in turn.
__device__ __forceinline__ void plan_scan(unsigned long long &x, unsigned long long &y, unsigned long long (*warps)[32], unsigned long long &total_x,
                                          unsigned long long &total_y) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
    auto scan = [&](unsigned long long v) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const unsigned long long u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += u;
        }
        return v;
    };
    const unsigned long long sx = scan(x), sy = scan(y);
    if (lane == 31) warps[0][warp] = sx, warps[1][warp] = sy;
    __syncthreads();
    const unsigned long long wx = scan(lane < nw ? warps[0][lane] : 0), wy = scan(lane < nw ? warps[1][lane] : 0);
    total_x = __shfl_sync(0xffffffffu, wx, 31), total_y = __shfl_sync(0xffffffffu, wy, 31);
    const unsigned long long bx = __shfl_sync(0xffffffffu, wx, max(warp - 1, 0)), by = __shfl_sync(0xffffffffu, wy, max(warp - 1, 0));
    x = sx - x + (warp ? bx : 0), y = sy - y + (warp ? by : 0);
}

__device__ __forceinline__ int plan_chunks(int len) { return (len + DELTALOG_SCAN_CHUNK - 1) / DELTALOG_SCAN_CHUNK; }

// Offsets of all rows into `starts` and `chunk_starts` ([n + 1], shared or global); `starts` holds the lengths before (the
// caller has put them there, so that a thread's run of rows costs no strided loads).  A row whose tokens would end behind
// max_tokens is dropped (it counts as empty), and so is every row behind it that has tokens.
template <bool SHARED>
__device__ __forceinline__ void plan_offsets(const PlanArgs &a, int32_t *starts, int32_t *chunk_starts, bool write_totals) {
    if (SHARED) {
        __builtin_assume(__isShared(starts));
        __builtin_assume(__isShared(chunk_starts));
    }
    __shared__ unsigned long long warps[2][2][32];
    // an odd run per thread: neighbours' accesses fall into different banks
    const int per = ((a.n + blockDim.x - 1) / blockDim.x) | 1, first = min(a.n, (int)threadIdx.x * per), last = min(a.n, first + per);
    unsigned long long tokens = 0, chunks = 0, total, total_chunks;  // chunks: of the rows as they are | scan rows << 32
    unsigned long long rows = 0, unused = 0, total_rows = 0;
    auto one = [&](int len) { return a.decode_rows && len == 1; };
    for (int i = first; i < last; ++i) {
        const int len = max(starts[i], 0);
        tokens += (unsigned long long)len;
        chunks += (unsigned long long)plan_chunks(len) + (len > 0 && !one(len) ? 1ull << 32 : 0);
        rows += len > 0;
    }
    const unsigned long long most = (unsigned long long)a.max_tokens;
    unsigned long long at = tokens, chunk_at = chunks;
    plan_scan(at, chunk_at, warps[0], total, total_chunks);
    if (total > most) {  // some rows do not fit: the same again without them
        __syncthreads();
        unsigned long long s = at;
        tokens = chunks = rows = 0;
        for (int i = first; i < last; ++i) {
            int len = max(starts[i], 0);
            if (s + len > most) len = 0, s = most + 1, starts[i] = 0;
            s += len;
            tokens += (unsigned long long)len;
            chunks += (unsigned long long)plan_chunks(len) + (len > 0 && !one(len) ? 1ull << 32 : 0);
            rows += len > 0;
        }
        at = tokens, chunk_at = chunks;
        plan_scan(at, chunk_at, warps[1], total, total_chunks);
    }
    if (write_totals) {
        __syncthreads();
        plan_scan(rows, unused, warps[0], total_rows, unused);
        if (threadIdx.x == 0) {
            const int scan_rows = (int)(total_chunks >> 32);
            *reinterpret_cast<int4 *>(a.totals) = make_int4((int)total, (int)(total_chunks & 0xffffffffu), scan_rows, (int)total_rows - scan_rows);
        }
    }
    uint32_t t = (uint32_t)at, c = (uint32_t)chunk_at;
    for (int i = first; i < last; ++i) {
        const int len = max(starts[i], 0);
        starts[i] = (int32_t)t, chunk_starts[i] = (int32_t)c;
        t += (uint32_t)len, c += (uint32_t)plan_chunks(len);
    }
    if (threadIdx.x == 0) starts[a.n] = (int32_t)total, chunk_starts[a.n] = (int32_t)(total_chunks & 0xffffffffu);
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

template <bool SHARED>
__device__ __forceinline__ void plan_tables(const PlanArgs &a, const int32_t *starts, const int32_t *chunk_starts) {
    if (SHARED) {
        __builtin_assume(__isShared(starts));
        __builtin_assume(__isShared(chunk_starts));
    }
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
    // a warp takes a run of tokens, 128 a step: the row of a step's first token is at or behind the last step's row, so the
    // search gallops from there
    const int lane = threadIdx.x & 31, warps = gridDim.x * (blockDim.x >> 5), warp = first >> 5;
    const long long steps = (a.max_tokens + 127ll) / 128, each = (steps + warps - 1) / warps;
    long long step = each * warp;
    const long long end = min(steps, step + each);
    int row = step < end && step * 128 < tokens ? plan_find(starts, a.n, (int)(step * 128)) : 0;
    for (; step < end; ++step) {
        const int base = (int)(step * 128), t0 = base + lane * 4;
        if (base + 127 < tokens && starts[row + 1] > base + 127) {  // all of one row
            *reinterpret_cast<int4 *>(a.token_seq + t0) = make_int4(row, row, row, row);
            continue;
        }
        const int before = row;
        if (t0 < tokens) {
            int ahead = 1;
            while (row + ahead <= a.n && starts[row + ahead] <= t0) ahead <<= 1;
            int hi = min(row + ahead, a.n);
            row += ahead >> 1;  // starts[row] <= t0 < starts[hi]
            while (hi - row > 1) {
                const int mid = (row + hi) >> 1;
                if (starts[mid] <= t0) row = mid;
                else hi = mid;
            }
        }
        int out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (t0 + e < tokens)
                while (starts[row + 1] <= t0 + e) ++row;
            out[e] = t0 + e < tokens ? row : -1;
        }
        if (t0 + 4 <= a.max_tokens) {
            *reinterpret_cast<int4 *>(a.token_seq + t0) = make_int4(out[0], out[1], out[2], out[3]);
        } else {
            for (int e = 0; t0 + e < a.max_tokens; ++e) a.token_seq[t0 + e] = out[e];
        }
        // the next step's tokens lie behind all of these; its first row is that of the last token here or of the next one
        row = __shfl_sync(0xffffffffu, t0 < tokens ? row : before, 31);
        if (row < a.n && base + 128 < tokens)
            while (starts[row + 1] <= base + 128) ++row;
    }
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanArgs a) {
    extern __shared__ int32_t offsets[];
    int32_t *starts = offsets, *chunk_starts = offsets + a.n + 1;
#pragma unroll 8
    for (int i = threadIdx.x; i < a.n; i += blockDim.x) starts[i] = a.lens[i];
    __syncthreads();
    plan_offsets<true>(a, starts, chunk_starts, blockIdx.x == 0);
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i <= a.n; i += gridDim.x * blockDim.x) {
        a.starts[i] = starts[i];
        a.chunk_starts[i] = chunk_starts[i];
    }
    plan_tables<true>(a, starts, chunk_starts);
}

__global__ void __launch_bounds__(1024) plan_offsets_kernel(const PlanArgs a) {
    for (int i = threadIdx.x; i < a.n; i += blockDim.x) a.starts[i] = a.lens[i];
    __syncthreads();
    plan_offsets<false>(a, a.starts, a.chunk_starts, true);
}
__global__ void __launch_bounds__(kPlanThreads) plan_tables_kernel(const PlanArgs a) { plan_tables<false>(a, a.starts, a.chunk_starts); }

}  // namespace deltalog
