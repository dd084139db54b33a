// Forward pass of the selective state space scan and its single-token form.
//
// Bound by the exponentials: one per token, channel and state, 16 a clock and SM.  Everything else is arranged around that:
// step sizes and gates are worked out once per token and channel on the way into and out of shared memory; B and C are widened
// once per CTA; per state a lane then does two products, the exponential and two fused multiply-adds; the sums over a
// channel's states run over four tokens at a time, three shuffles for four sums.
#pragma once

#include "ssm_common.cuh"

namespace deltalog {

template <typename IO, int N> struct SsmForward {
    static constexpr int kPer = N <= 16 ? 1 : N / 16;                                       // channels per lane
    static constexpr int kCols = kSsmWarps * SsmLanes<N>::kChannels * kPer, kTile = 32;    // channels of a CTA, tokens of a tile
    struct Raw {
        IO x[kTile * kCols], dt[kTile * kCols], z[kTile * kCols], B[kTile * N], C[kTile * N];
    };
    struct alignas(16) Shared {
        Raw raw[2];
        float2 step[kTile * kCols];  // delta, delta x
        float B[kTile * N], C[kTile * N], y[kTile * kCols];
        int state[kTile], row[kTile];
        unsigned begins, ends, there, open;  // one bit per token of the tile; open: its row goes on behind the stretch
    };
};

// LOCAL: the first pass over a stretch whose last row goes on behind it.
template <typename IO, int N, bool LOCAL>
__global__ void __launch_bounds__(kSsmThreads) ssm_forward_kernel(const SsmArgs a) {
    using F = SsmForward<IO, N>;
    constexpr int KC = F::kPer, CB = F::kCols, TT = F::kTile, LN = SsmLanes<N>::kStates, LC = SsmLanes<N>::kChannels, VE = 16 / sizeof(IO);
    extern __shared__ __align__(16) char smem[];
    typename F::Shared &s = *reinterpret_cast<typename F::Shared *>(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per_group = a.D_ / a.G, group = blockIdx.x / a.blocks, in_group = (blockIdx.x % a.blocks) * CB;
    const int c0 = group * per_group + in_group, cols = min(CB, per_group - in_group);  // this CTA's channels
    const int span = blockIdx.y;
    const int nl = lane & (LN - 1), cl = lane / LN;
    int mine[KC];  // this lane's channels within the block
#pragma unroll
    for (int k = 0; k < KC; ++k) mine[k] = (warp * KC + k) * LC + cl;
    auto at = [&](size_t state, int k) { return (state * a.D_ + c0 + mine[k]) * N + nl * 4; };

    if (!LOCAL && span >= a.spans) {  // rows without tokens: their state is the one they came with
        for (int row = 0; row < a.rows.n; ++row) {
            if (a.rows.starts[row] != a.rows.starts[row + 1]) continue;
#pragma unroll
            for (int k = 0; k < KC; ++k)
                if (mine[k] < cols)
                    *reinterpret_cast<float4 *>(a.S_out + at(row, k)) =
                        a.S_in ? *reinterpret_cast<const float4 *>(a.S_in + at(row, k)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        return;
    }
    const int lo = span * a.span, hi = (int)min((long long)a.max_tokens, (long long)lo + a.span);
    int from = lo, only = -1;  // LOCAL: the open row alone
    if (LOCAL) {
        const SsmToken last = ssm_token(a, hi - 1, false);
        if (last.row < 0 || last.end <= hi) return;
        only = last.row;
        from = max(lo, last.begin) & ~(TT - 1);
    }
    const IO *x = static_cast<const IO *>(a.x) + c0, *dt = static_cast<const IO *>(a.dt) + c0, *z = static_cast<const IO *>(a.z) + (a.z ? c0 : 0);
    const IO *Bp = static_cast<const IO *>(a.B) + group * N, *Cp = static_cast<const IO *>(a.C) + group * N;

    float A2[KC][4], h[KC][4], sum[KC];
#pragma unroll
    for (int k = 0; k < KC; ++k) {
        const float4 f = mine[k] < cols ? *reinterpret_cast<const float4 *>(a.A + (size_t)(c0 + mine[k]) * N + nl * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
        A2[k][0] = f.x, A2[k][1] = f.y, A2[k][2] = f.z, A2[k][3] = f.w;
        sum[k] = 0.f;
#pragma unroll
        for (int n = 0; n < 4; ++n) A2[k][n] *= 1.4426950408889634f, h[k][n] = 0.f;
    }
    auto load_state = [&](const float *p, size_t state) {
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            const float4 f = p && mine[k] < cols ? *reinterpret_cast<const float4 *>(p + at(state, k)) : make_float4(0.f, 0.f, 0.f, 0.f);
            h[k][0] = f.x, h[k][1] = f.y, h[k][2] = f.z, h[k][3] = f.w;
        }
    };
    auto store_state = [&](float *p, size_t state) {
#pragma unroll
        for (int k = 0; k < KC; ++k)
            if (mine[k] < cols) *reinterpret_cast<float4 *>(p + at(state, k)) = make_float4(h[k][0], h[k][1], h[k][2], h[k][3]);
    };
    if (!LOCAL && span > 0) {
        const SsmToken first = ssm_token(a, lo, false);
        if (first.row >= 0 && first.begin < lo) {  // a row from an earlier stretch: its states joined
            int j = first.begin / a.span;
            load_state(a.local, j);
            for (++j; j < span; ++j) {
                float before[KC][4];
#pragma unroll
                for (int k = 0; k < KC; ++k) {
                    const float total = mine[k] < cols ? a.sums[(size_t)j * a.D_ + c0 + mine[k]] : 0.f;
#pragma unroll
                    for (int n = 0; n < 4; ++n) before[k][n] = exp2_fast(A2[k][n] * total) * h[k][n];
                }
                load_state(a.local, j);
#pragma unroll
                for (int k = 0; k < KC; ++k)
#pragma unroll
                    for (int n = 0; n < 4; ++n) h[k][n] += before[k][n];
            }
        }
    }
    // the vector of channels that this thread brings in and out, and its first token of a tile
    const int vec = (tid % (CB / VE)) * VE, vec_token = tid / (CB / VE);
    constexpr int kTokenStep = kSsmThreads / (CB / VE);
    float bias[VE], skip[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        bias[e] = a.bias && vec < cols ? a.bias[c0 + vec + e] : 0.f;
        skip[e] = a.D && vec < cols ? a.D[c0 + vec + e] : 0.f;
    }
    auto fetch = [&](int t, int stage) {
        typename F::Raw &r = s.raw[stage];
        ssm_stage(r.x, x, a.x_stride, t, TT, from, hi, CB, cols, kSsmThreads);
        ssm_stage(r.dt, dt, a.dt_stride, t, TT, from, hi, CB, cols, kSsmThreads);
        ssm_stage(r.B, Bp, a.B_stride, t, TT, from, hi, N, N, kSsmThreads);
        if (!LOCAL) {
            if (a.z) ssm_stage(r.z, z, a.z_stride, t, TT, from, hi, CB, cols, kSsmThreads);
            ssm_stage(r.C, Cp, a.C_stride, t, TT, from, hi, N, N, kSsmThreads);
        }
        cp_async_commit();
    };
    fetch(from, 0);
    int stage = 0;
    for (int t = from; t < hi; t += TT, stage ^= 1) {
        const typename F::Raw &r = s.raw[stage];
        if (warp == 0) {
            SsmToken k{-1, -1, 0, 0};
            if (t + lane < hi) k = ssm_token(a, t + lane, !LOCAL && blockIdx.x == 0);
            if (LOCAL && k.row != only) k.row = -1;
            s.state[lane] = k.state, s.row[lane] = k.row;
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
        for (int q = 0; q < TT / kTokenStep; ++q) {
            const int k = vec_token + q * kTokenStep;
            const Pack<IO, VE> xv = pack_load<IO, VE>(r.x + k * CB + vec), dv = pack_load<IO, VE>(r.dt + k * CB + vec);
            const bool ok = there >> k & 1;
#pragma unroll
            for (int e = 0; e < VE; e += 2) {
                float d[2];
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    d[f] = to_f32(dv.e[e + f]) + bias[e + f];
                    if (a.softplus) d[f] = ssm_softplus(d[f]);
                    if (!ok) d[f] = 0.f;
                }
                *reinterpret_cast<float4 *>(s.step + k * CB + vec + e) =
                    make_float4(d[0], ok ? d[0] * to_f32(xv.e[e]) : 0.f, d[1], ok ? d[1] * to_f32(xv.e[e + 1]) : 0.f);
            }
        }
        for (int i = tid; i < TT * N; i += kSsmThreads) {  // (a skipped token may hold anything)
            const bool ok = there >> (i / N) & 1;
            s.B[i] = ok ? to_f32(r.B[i]) : 0.f;
            if (!LOCAL) s.C[i] = ok ? to_f32(r.C[i]) : 0.f;
        }
        __syncthreads();
        for (int k0 = 0; k0 < min(TT, hi - t); k0 += 4) {
            if (!LOCAL && a.kept && k0 % kSsmBlock == 0) store_state(a.kept, (size_t)(t + k0) / kSsmBlock);
            float y[4 * KC];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int k = k0 + i;
                if (begins >> k & 1) {
                    const bool old = a.S_in && !(a.fresh && a.fresh[s.row[k]]);
                    // another CTA may have written the pool's state of an open row already: the first pass kept it
                    if (!LOCAL && a.front && (s.open >> k & 1)) load_state(a.front, span);
                    else load_state(old ? a.S_in : nullptr, s.state[k]);
                    if (LOCAL && a.front) store_state(a.front, span);
                }
                const float4 Bv = *reinterpret_cast<const float4 *>(s.B + k * N + nl * 4);
                const float b[4] = {Bv.x, Bv.y, Bv.z, Bv.w};
                float c[4];
                if (!LOCAL) {
                    const float4 Cv = *reinterpret_cast<const float4 *>(s.C + k * N + nl * 4);
                    c[0] = Cv.x, c[1] = Cv.y, c[2] = Cv.z, c[3] = Cv.w;
                }
#pragma unroll
                for (int q = 0; q < KC; ++q) {
                    const float2 d = s.step[k * CB + mine[q]];
                    float out = 0.f;
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        h[q][n] = fmaf(exp2_fast(d.x * A2[q][n]), h[q][n], d.y * b[n]);
                        if (!LOCAL) out = fmaf(c[n], h[q][n], out);
                    }
                    if (LOCAL) sum[q] += d.x;
                    else y[i * KC + q] = out;
                }
                if (!LOCAL && a.S_out && (ends >> k & 1)) store_state(a.S_out, s.state[k]);
            }
            if (!LOCAL) {
                const int first = lanes_reduce<4 * KC, LN>(y, lane);
#pragma unroll
                for (int j = 0; j < 4 * KC / LN; ++j) {
                    const int v = first + j, i = v / KC, q = v % KC;
                    s.y[(k0 + i) * CB + (warp * KC + q) * LC + cl] = y[j];
                }
            }
        }
        __syncthreads();
        if (LOCAL) continue;
        if (a.out && vec < cols) {
#pragma unroll
            for (int q = 0; q < TT / kTokenStep; ++q) {
                const int k = vec_token + q * kTokenStep;
                if (t + k >= hi) break;
                IO *out = static_cast<IO *>(a.out) + (size_t)(t + k) * a.D_ + c0 + vec;
                if (!(there >> k & 1)) {
                    if (a.clear) pack_store(out, pack_zero<IO, VE>());
                    continue;
                }
                const Pack<IO, VE> xv = pack_load<IO, VE>(r.x + k * CB + vec);
                Pack<IO, VE> zv, o;
                if (a.z) zv = pack_load<IO, VE>(r.z + k * CB + vec);
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    float v = fmaf(skip[e], to_f32(xv.e[e]), s.y[k * CB + vec + e]);
                    if (a.z) {
                        const float g = to_f32(zv.e[e]);
                        v *= g * sigmoid(g);
                    }
                    o.e[e] = from_f32<IO>(v);
                }
                pack_store(out, o);
            }
        }
    }
    if (LOCAL) {
        store_state(a.local, span);
        if (nl == 0)
#pragma unroll
            for (int k = 0; k < KC; ++k)
                if (mine[k] < cols) a.sums[(size_t)span * a.D_ + c0 + mine[k]] = sum[k];
    }
}

// One token per row.  Bound by HBM, the states' read and write.  A lane keeps its channel's A for all of its rows, four of
// which are in flight.
template <typename IO, int N>
__global__ void __launch_bounds__(kSsmThreads) ssm_step_kernel(const SsmArgs a, int col_blocks, int run) {
    constexpr int LN = SsmLanes<N>::kStates, LC = SsmLanes<N>::kChannels, U = 4;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nl = lane & (LN - 1), cl = lane / LN;
    const int c = ((int)(blockIdx.x % col_blocks) * kSsmWarps + warp) * LC + cl;
    const bool live = c < a.D_;
    const int cc = live ? c : 0, group = cc / (a.D_ / a.G);
    const long long first = (long long)(blockIdx.x / col_blocks) * run;
    const float4 Af = *reinterpret_cast<const float4 *>(a.A + (size_t)cc * N + nl * 4);
    const float A2[4] = {Af.x * 1.4426950408889634f, Af.y * 1.4426950408889634f, Af.z * 1.4426950408889634f, Af.w * 1.4426950408889634f};
    const float bias = a.bias ? a.bias[cc] : 0.f, skip = a.D ? a.D[cc] : 0.f;
    const int end = (int)min((long long)a.total_rows, first + run);
    for (int row = (int)first; row < end; row += U) {
        float4 h[U];
        float b[U][4], cv[U][4], x[U], d[U], z[U];
        int slot[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            slot[u] = -1;
            if (row + u < end && !resolve_slot(a.slots, row + u, a.num_slots, a.status, threadIdx.x, slot[u])) slot[u] = -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (slot[u] < 0) continue;
            const size_t t = row + u;
            h[u] = *reinterpret_cast<const float4 *>(a.S_in + ((size_t)slot[u] * a.D_ + cc) * N + nl * 4);
            load_vec<IO, 4>(static_cast<const IO *>(a.B) + t * a.B_stride + group * N + nl * 4, b[u]);
            load_vec<IO, 4>(static_cast<const IO *>(a.C) + t * a.C_stride + group * N + nl * 4, cv[u]);
            x[u] = to_f32(static_cast<const IO *>(a.x)[t * a.x_stride + cc]);
            d[u] = to_f32(static_cast<const IO *>(a.dt)[t * a.dt_stride + cc]) + bias;
            z[u] = a.z ? to_f32(static_cast<const IO *>(a.z)[t * a.z_stride + cc]) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (slot[u] < 0) continue;
            const float delta = a.softplus ? ssm_softplus(d[u]) : d[u], dx = delta * x[u];
            float4 &s = h[u];
            s.x = fmaf(exp2_fast(delta * A2[0]), s.x, dx * b[u][0]);
            s.y = fmaf(exp2_fast(delta * A2[1]), s.y, dx * b[u][1]);
            s.z = fmaf(exp2_fast(delta * A2[2]), s.z, dx * b[u][2]);
            s.w = fmaf(exp2_fast(delta * A2[3]), s.w, dx * b[u][3]);
            float y = s.x * cv[u][0] + s.y * cv[u][1] + s.z * cv[u][2] + s.w * cv[u][3];
#pragma unroll
            for (int o = LN / 2; o > 0; o >>= 1) y += __shfl_xor_sync(0xffffffffu, y, o);
            if (!live) continue;
            *reinterpret_cast<float4 *>(a.S_out + ((size_t)slot[u] * a.D_ + cc) * N + nl * 4) = s;
            if (nl == 0) {
                y = fmaf(skip, x[u], y);
                if (a.z) y *= z[u] * sigmoid(z[u]);
                static_cast<IO *>(a.out)[(size_t)(row + u) * a.D_ + cc] = from_f32<IO>(y);
            }
        }
    }
}

}  // namespace deltalog
