// Forward pass of the selective state space scan and its single-token form.
//
// Bound by the exponentials: one per token, channel and state, 16 a clock and SM.  Everything else is arranged around that:
// step sizes and gates are worked out once per token and channel on the way into and out of shared memory, two neighbouring
// channels a thread; B and C are widened once per CTA; per pair of states a lane then does two packed products, two
// exponentials and two packed fused multiply-adds; the sums over a channel's states run over four tokens at a time, six shuffles for
// eight sums.  Two channels a lane share the loads of B and C, which at one channel cost more than the exponentials.
// 14k ragged tokens x 4096 channels x 16 states: 414 us behind a first pass of 107 (the exponentials alone: 204), special function
// units 64 % busy, issue slots 53 %: the rest is latency between the phases of a tile, three barriers apart; 16k x 2048 in one row 238 +
// 175.  Four CTAs an SM; six with fewer registers or smaller tiles took as long; four channels a lane in tiles of 16 tokens, three CTAs,
// have 420 behind 233.
#pragma once

#include "ssm_common.cuh"

namespace deltalog {

// WIDE: two channels a lane (four where a channel takes sixteen lanes); otherwise half of that, which takes a token's latency down
// where there are few CTAs.
template <typename IO, int N, bool WIDE> struct SsmForward {
    static constexpr int kPer = (N <= 32 ? 2 : 4) / (WIDE ? 1 : 2);                         // channels per lane
    static constexpr int kCols = kSsmWarps * SsmLanes<N>::kChannels * kPer, kTile = 32;    // channels of a CTA, tokens of a tile
    static constexpr int kPitch = kCols + 8;  // lanes that answer for neighbouring tokens store to different banks
    struct Raw {
        IO x[kTile * kCols], dt[kTile * kCols], z[kTile * kCols], B[kTile * N], C[kTile * N];
    };
    struct alignas(16) Shared {
        Raw raw[2];
        float2 step[kTile * kPitch];  // delta, delta x; then C . h in the first's place
        float B[kTile * N], C[kTile * N];
        int state[kTile], row[kTile];
        unsigned begins, ends, there, open;  // one bit per token of the tile; open: its row goes on behind the stretch
    };
    static constexpr int kCtas = ssm_ctas(N <= 32 ? 4 : 3, sizeof(Shared));  // on an SM
};

// LOCAL: the first pass over a part of a stretch (`span` is the part), where its last row goes on behind the stretch.
template <typename IO, int N, bool LOCAL, bool WIDE>
__global__ void __launch_bounds__(kSsmThreads, (SsmForward<IO, N, WIDE>::kCtas)) ssm_forward_kernel(const SsmArgs a) {
    using F = SsmForward<IO, N, WIDE>;
    constexpr int KC = F::kPer, CB = F::kCols, PB = F::kPitch, TT = F::kTile, LN = SsmLanes<N>::kStates, LC = SsmLanes<N>::kChannels;
    extern __shared__ __align__(16) char smem[];
    typename F::Shared &s = *reinterpret_cast<typename F::Shared *>(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per_group = a.D_ / a.G, group = blockIdx.x / a.blocks, in_group = (blockIdx.x % a.blocks) * CB;
    const int c0 = group * per_group + in_group, cols = min(CB, per_group - in_group);  // this CTA's channels
    const int span = blockIdx.y;
    const int nl = lane & (LN - 1), cl = lane / LN;
    const int first = warp * KC * LC + cl;  // this lane's channels of the block: first, first + LC ..
    auto at = [&](size_t state, int q) { return (state * a.D_ + c0 + first + q * LC) * N + nl * 4; };
    auto mine = [&](int q) { return first + q * LC < cols; };

    if (!LOCAL && span >= a.spans) {  // rows without tokens: their state is the one they came with
        ssm_empty_rows(a, span - a.spans, [&](int row) {
#pragma unroll
            for (int q = 0; q < KC; ++q)
                if (mine(q))
                    *reinterpret_cast<float4 *>(a.S_out + at(row, q)) =
                        a.S_in ? *reinterpret_cast<const float4 *>(a.S_in + at(row, q)) : make_float4(0.f, 0.f, 0.f, 0.f);
        });
        return;
    }
    const int length = LOCAL ? a.part : a.span, lo = span * length, bound = (int)min((long long)a.max_tokens, (long long)lo + length);
    const int hi = max(lo, min(bound, a.rows.starts[a.rows.n]));  // the tokens that there are
    int from = lo, only = -1;  // LOCAL: the open row alone
    if (LOCAL) {
        if (hi == lo) return;
        const SsmToken last = ssm_token(a, hi - 1, false);
        if (last.row < 0 || last.end <= (lo / a.span + 1ll) * a.span) return;
        only = last.row;
        from = max(lo, last.begin) & ~(TT - 1);
    }
    const IO *x = static_cast<const IO *>(a.x) + c0, *dt = static_cast<const IO *>(a.dt) + c0, *z = static_cast<const IO *>(a.z) + (a.z ? c0 : 0);
    const IO *Bp = static_cast<const IO *>(a.B) + group * N, *Cp = static_cast<const IO *>(a.C) + group * N;

    auto fetch = [&](int t, int stage) {
        typename F::Raw &r = s.raw[stage];
        auto parts = [&](auto all) {
            constexpr bool ALL = decltype(all)::value;
            ssm_stage<ALL, TT, CB>(r.x, x, a.x_stride, t, from, hi, cols);
            ssm_stage<ALL, TT, CB>(r.dt, dt, a.dt_stride, t, from, hi, cols);
            ssm_stage<ALL, TT, N>(r.B, Bp, a.B_stride, t, from, hi, N);
            if (!LOCAL) {
                if (a.z) ssm_stage<ALL, TT, CB>(r.z, z, a.z_stride, t, from, hi, cols);
                ssm_stage<ALL, TT, N>(r.C, Cp, a.C_stride, t, from, hi, N);
            }
        };
        if (t + TT <= hi && cols == CB) parts(std::true_type{});
        else parts(std::false_type{});
        cp_async_commit();
    };
    fetch(from, 0);

    float2 A2[KC][2], h[KC][2];  // A in powers of two
    float sum[KC];
    auto load_state = [&](const float *p, size_t state, float2 (&v)[KC][2]) {
#pragma unroll
        for (int q = 0; q < KC; ++q) {
            v[q][0] = v[q][1] = both(0.f);
            if (p && mine(q)) ssm_load(p + at(state, q), v[q]);
        }
    };
    auto store_state = [&](float *p, size_t state) {
#pragma unroll
        for (int q = 0; q < KC; ++q)
            if (mine(q)) ssm_store(p + at(state, q), h[q]);
    };
    float lift[KC];  // of the decays; at first the bias that it goes by
#pragma unroll
    for (int q = 0; q < KC; ++q) lift[q] = a.bias && mine(q) ? a.bias[c0 + first + q * LC] : 0.f;
    load_state(a.A, 0, A2);
#pragma unroll
    for (int q = 0; q < KC; ++q) {
        sum[q] = 0.f;
#pragma unroll
        for (int p = 0; p < 2; ++p) A2[q][p] = __fmul2_rn(A2[q][p], both(1.4426950408889634f)), h[q][p] = both(0.f);
    }
#pragma unroll
    for (int q = 0; q < KC; ++q) lift[q] = ssm_lift(a, A2[q], lift[q]);
    if (!LOCAL && span > 0) {
        const SsmToken head = ssm_token(a, lo, false);
        if (head.row >= 0 && head.begin < lo) load_state(a.local, lo / a.part - 1, h);  // a row from an earlier stretch
    }
    // the two channels that this thread brings in and out, and its first token of a tile
    const int col = (tid % (CB / 2)) * 2, col_token = tid / (CB / 2);
    constexpr int kTokenStep = kSsmThreads / (CB / 2);
    const float2 bias = a.bias && col < cols ? load2(a.bias + c0 + col) : both(0.f), skip = a.D && col < cols ? load2(a.D + c0 + col) : both(0.f);
    int stage = 0;
    for (int t = from; t < hi; t += TT, stage ^= 1) {
        typename F::Raw &r = s.raw[stage];
        if (warp == 0) {
            SsmToken k{-1, -1, 0, 0};
            if (lane < TT && t + lane < hi) k = ssm_token(a, t + lane, !LOCAL && blockIdx.x == 0);
            if (LOCAL && k.row != only) k.row = -1;
            if (lane < TT) s.state[lane] = k.state, s.row[lane] = k.row;
            const unsigned begins = __ballot_sync(0xffffffffu, k.row >= 0 && k.begin == t + lane);
            const unsigned ends = __ballot_sync(0xffffffffu, k.row >= 0 && k.end == t + lane + 1);
            const unsigned there = __ballot_sync(0xffffffffu, k.row >= 0), open = __ballot_sync(0xffffffffu, k.row >= 0 && k.end > hi);
            if (lane == 0) s.begins = begins, s.ends = ends, s.there = there, s.open = open;
        }
        cp_async_wait_all();
        __syncthreads();  // the tile and its tokens are there; the one before is done with
        if (t + TT < hi) fetch(t + TT, stage ^ 1);
        const unsigned there = s.there, begins = s.begins, ends = s.ends;
#pragma unroll
        for (int i = 0; i < TT / kTokenStep; ++i) {
            const int k = col_token + i * kTokenStep;
            float2 d = __fadd2_rn(load2(r.dt + k * CB + col), bias), unused;
            if (a.softplus) d = ssm_softplus(d, unused);
            const float2 u = __fmul2_rn(d, load2(r.x + k * CB + col));
            *reinterpret_cast<float4 *>(s.step + k * PB + col) = make_float4(d.x, u.x, d.y, u.y);
        }
        if (there != (unsigned)((1ull << TT) - 1)) {  // a skipped token may hold anything, and changes nothing
#pragma unroll
            for (int i = 0; i < TT / kTokenStep; ++i) {
                const int k = col_token + i * kTokenStep;
                if (!(there >> k & 1)) *reinterpret_cast<float4 *>(s.step + k * PB + col) = make_float4(0.f, 0.f, 0.f, 0.f);
            }
            for (int i = tid; i < TT * N; i += kSsmThreads)
                if (!(there >> (i / N) & 1)) r.B[i] = r.C[i] = from_f32<IO>(0.f);
            __syncthreads();
        }
#pragma unroll
        for (int i0 = 0; i0 < TT * N / 2; i0 += kSsmThreads) {
            const int i = 2 * (i0 + tid);
            if (TT * N / 2 % kSsmThreads && i >= TT * N) break;
            store2(s.B + i, load2(r.B + i));
            if (!LOCAL) store2(s.C + i, load2(r.C + i));
        }
        __syncthreads();
        // four tokens; MARKED: where rows may begin or end
        auto four = [&](int k0, auto marked) {
            constexpr bool MARKED = decltype(marked)::value;
            float y[4 * KC];
            const float2 *step = s.step + k0 * PB + first;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (MARKED && (begins >> (k0 + i) & 1)) {
                    const int k = k0 + i;
                    const bool old = a.S_in && !(a.fresh && a.fresh[s.row[k]]);
                    // another CTA may have written the pool's state of an open row already: the first pass kept it
                    if (!LOCAL && a.front && (s.open >> k & 1)) load_state(a.front, (t + k) / a.part, h);
                    else load_state(old ? a.S_in : nullptr, s.state[k], h);
                    if (LOCAL && a.front) store_state(a.front, span);
                }
                float2 b[2], c[2];
                ssm_pairs(s.B + (k0 + i) * N + nl * 4, b);
                if (!LOCAL) ssm_pairs(s.C + (k0 + i) * N + nl * 4, c);
#pragma unroll
                for (int q = 0; q < KC; ++q) {
                    const float2 d = step[i * PB + q * LC];
                    float2 out = both(0.f);
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        h[q][p] = __ffma2_rn(ssm_decay(A2[q][p], d.x, lift[q]), h[q][p], __fmul2_rn(b[p], both(d.y)));
                        if (!LOCAL) out = p ? __ffma2_rn(c[p], h[q][p], out) : __fmul2_rn(c[p], h[q][p]);
                    }
                    if (LOCAL) sum[q] += d.x;
                    else y[i * KC + q] = out.x + out.y;
                }
                if (MARKED && !LOCAL && a.S_out && (ends >> (k0 + i) & 1)) store_state(a.S_out, s.state[k0 + i]);
            }
            if (!LOCAL) {  // the warp is done with these tokens' steps
                const int v0 = lanes_reduce<4 * KC, LN>(y, lane);
#pragma unroll
                for (int j = 0; j < (4 * KC > LN ? 4 * KC / LN : 1); ++j) s.step[(k0 + (v0 + j) / KC) * PB + first + (v0 + j) % KC * LC].x = y[j];
            }
        };
        const int here = min(TT, hi - t);
        for (int k0 = 0; k0 < here; k0 += 8) {
            if (!LOCAL && a.kept) store_state(a.kept, (size_t)(t + k0) / kSsmBlock);
            if ((begins | ends) >> k0 & 255) {
                four(k0, std::true_type{});
                four(k0 + 4, std::true_type{});
            } else {  // (eight tokens without a branch: one group's sums run beside the next one's decays)
                four(k0, std::false_type{});
                four(k0 + 4, std::false_type{});
            }
        }
        __syncthreads();
        if (LOCAL) continue;
        if (a.out && col < cols) {
            const int here = min(TT, hi - t);
#pragma unroll
            for (int i = 0; i < TT / kTokenStep; ++i) {
                const int k = col_token + i * kTokenStep;
                if (k >= here) break;
                IO *out = static_cast<IO *>(a.out) + (size_t)(t + k) * a.D_ + c0 + col;
                if (!(there >> k & 1)) {
                    if (a.clear) store2(out, both(0.f));
                    continue;
                }
                const float4 y = *reinterpret_cast<const float4 *>(s.step + k * PB + col);
                float2 o = __ffma2_rn(skip, load2(r.x + k * CB + col), make_float2(y.x, y.z));
                if (a.z) {
                    const float2 g = load2(r.z + k * CB + col);
                    o = __fmul2_rn(o, make_float2(g.x * sigmoid(g.x), g.y * sigmoid(g.y)));
                }
                store2(out, o);
            }
        }
    }
    if (!LOCAL && a.out && a.clear && col < cols)  // behind the last sequence
        for (int t = hi + col_token; t < bound; t += kTokenStep) store2(static_cast<IO *>(a.out) + (size_t)t * a.D_ + c0 + col, both(0.f));
    if (LOCAL) {
        store_state(a.local, span);
        if (nl == 0)
#pragma unroll
            for (int q = 0; q < KC; ++q)
                if (mine(q)) a.sums[(size_t)span * a.D_ + c0 + first + q * LC] = sum[q];
    }
}

// One token per row.  Bound by HBM, the states' read and write.  A lane holds eight states of a channel (32 bytes, one access),
// so that step size and gate are worked out by d_state / 8 lanes, and keeps its channel's A for all of its rows, two of which are in
// flight (four, with fewer CTAs on an SM: 21 us where two take 16; with the 92 registers that a free choice takes, 20).
__device__ __forceinline__ void ssm_load8(const float *p, float2 (&v)[4]) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(v[0].x), "=f"(v[0].y), "=f"(v[1].x), "=f"(v[1].y), "=f"(v[2].x), "=f"(v[2].y), "=f"(v[3].x), "=f"(v[3].y) : "l"(p) : "memory");
}
__device__ __forceinline__ void ssm_store8(float *p, const float2 (&v)[4]) {
    asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "f"(v[0].x), "f"(v[0].y), "f"(v[1].x), "f"(v[1].y), "f"(v[2].x), "f"(v[2].y), "f"(v[3].x), "f"(v[3].y) : "memory");
}

__device__ __forceinline__ float ssm_slowest(const float2 (&A2)[4]) {
    float m = fmaxf(A2[0].x, A2[0].y);
#pragma unroll
    for (int p = 1; p < 4; ++p) m = fmaxf(m, fmaxf(A2[p].x, A2[p].y));
    return m;
}

template <typename IO, int N>
__global__ void __launch_bounds__(kSsmThreads, (sizeof(IO) == 4 ? 5 : 7)) ssm_step_kernel(const SsmArgs a, int col_blocks, int run) {
    constexpr int LN = N / 8, LC = 32 / LN, U = 2;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nl = lane & (LN - 1), cl = lane / LN;
    const int c = ((int)(blockIdx.x % col_blocks) * kSsmWarps + warp) * LC + cl;
    const bool live = c < a.D_;
    const int cc = live ? c : 0, group = cc / (a.D_ / a.G);
    const long long first = (long long)(blockIdx.x / col_blocks) * run;
    const int end = (int)min((long long)a.total_rows, first + run);
    const IO *x = static_cast<const IO *>(a.x) + cc, *dt = static_cast<const IO *>(a.dt) + cc, *z = static_cast<const IO *>(a.z) + (a.z ? cc : 0);
    const IO *B = static_cast<const IO *>(a.B) + group * N + nl * 8, *C = static_cast<const IO *>(a.C) + group * N + nl * 8;
    const size_t at = (size_t)cc * N + nl * 8, pitch = (size_t)a.D_ * N;
    struct Row {
        float2 h[4];
        Pack<IO, 8> b, c;
        IO x, d, z;
        int slot;
    };
    Row rows[U];
    if (first >= end) return;
    float2 A2[4];
    float bias = 0.f, skip = 0.f;
    for (int row = (int)first; row < end; row += U) {
        int slot[U];
        step_slots(a.slots, row, end, slot);
        step_check(row, end, a.num_slots, a.status, slot);
        // every row is loaded, a skipped one from wherever is allowed, so that no branch keeps one load behind another
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Row &r = rows[u];
            r.slot = slot[u];
            const long long t = min(row + u, end - 1);
            ssm_load8(a.S_in + max(r.slot, 0) * pitch + at, r.h);
            r.x = x[t * a.x_stride], r.d = dt[t * a.dt_stride], r.z = a.z ? z[t * a.z_stride] : r.x;
#pragma unroll
            for (int e = 0; e < 8; e += 16 / sizeof(IO)) {
                *reinterpret_cast<uint4 *>(r.b.e + e) = *reinterpret_cast<const uint4 *>(B + t * a.B_stride + e);
                *reinterpret_cast<uint4 *>(r.c.e + e) = *reinterpret_cast<const uint4 *>(C + t * a.C_stride + e);
            }
        }
        if (row == (int)first) {
            ssm_load8(a.A + at, A2);
            if (a.bias) bias = a.bias[cc];
            if (a.D) skip = a.D[cc];
#pragma unroll
            for (int p = 0; p < 4; ++p) A2[p] = __fmul2_rn(A2[p], both(1.4426950408889634f));
        }
        float out[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Row &r = rows[u];
            const float v = to_f32(r.d) + bias, xf = to_f32(r.x);
            float2 unused, y = both(0.f);
            const float delta = a.softplus ? ssm_softplus(both(v), unused).x : v, in = delta * xf;
            const float lift = ssm_lift(ssm_slowest(A2) * delta);
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                r.h[p] = __ffma2_rn(ssm_decay(A2[p], delta, lift), r.h[p], __fmul2_rn(load2(r.b.e + 2 * p), both(in)));
                y = __ffma2_rn(load2(r.c.e + 2 * p), r.h[p], y);
            }
            out[u] = y.x + y.y;
#pragma unroll
            for (int k = LN / 2; k > 0; k >>= 1) out[u] += __shfl_xor_sync(0xffffffffu, out[u], k);
            out[u] = fmaf(skip, xf, out[u]);
            if (a.z) {
                const float g = to_f32(r.z);
                out[u] *= g * sigmoid(g);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (rows[u].slot < 0 || !live) continue;
            ssm_store8(a.S_out + rows[u].slot * pitch + at, rows[u].h);
            if (nl == 0) static_cast<IO *>(a.out)[(size_t)(row + u) * a.D_ + cc] = from_f32<IO>(out[u]);
        }
    }
}

}  // namespace deltalog
