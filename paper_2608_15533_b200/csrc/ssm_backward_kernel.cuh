// Gradients of the selective state space scan.  With dy = dout silu(z) and dh_t the adjoint of h_t:
//     dh_t = C dy_t + a_(t+1) dh_(t+1)            dC = sum over channels dy h,   dB = sum over channels dh delta x
//     dx = delta sum dh B + D dy                  ddelta = x sum dh B + sum dh (a h_(t-1)) A,   ddt = ddelta sigmoid(dt + bias)
//     dA = sum_t dh (a h_(t-1)) delta             dz = dout (C h + D x) silu'(z),   dS_init = a_first dh_first
//
// Walks eight tokens at a time from the last to the first: the forward pass kept the state in front of every eighth token, from
// which a lane runs the eight again with a and a h_(t-1) in registers, one exponential per token, channel and state as in
// the forward pass, and then goes back over them.  (The states of every token would be 8 times the bytes; kept every 16
// tokens they would cost half the exponentials once more.)  a h_(t-1) is kept rather than h_t, from which it would come out by
// a difference that cancels where the decay is strong.
// Sums over a channel's states and over a warp's channels run over several values at once (lanes_reduce), over the warps in
// shared memory, over the CTAs in ssm_sums_kernel; each in a fixed order.
#pragma once

#include "ssm_common.cuh"

namespace deltalog {

template <typename IO, int N> struct SsmBackward {
    static constexpr int kPer = 2;
    static constexpr int kCols = kSsmWarps * SsmLanes<N>::kChannels * kPer, kTile = 16;
    struct Raw {
        IO x[kTile * kCols], dt[kTile * kCols], z[kTile * kCols], dout[kTile * kCols], B[kTile * N], C[kTile * N];
    };
    struct alignas(16) Shared {
        Raw raw[2];
        float2 step[kTile * kCols];  // delta, delta x
        float dy[kTile * kCols], B[kTile * N], C[kTile * N];
        float sums[3][kTile * kCols];  // C . h, sum dh B, sum dh a h_(t-1) A (in powers of two)
        float bc[kSsmWarps][kTile][2 * N];
        int state[kTile], row[kTile];
        unsigned begins, ends, there;
    };
};

// LOCAL: the first pass over a stretch whose first row began in front of it: the adjoint that the stretch alone hands back.
template <typename IO, int N, bool LOCAL>
__global__ void __launch_bounds__(kSsmThreads) ssm_backward_kernel(const SsmArgs a) {
    using F = SsmBackward<IO, N>;
    constexpr int KC = F::kPer, CB = F::kCols, TT = F::kTile, LN = SsmLanes<N>::kStates, LC = SsmLanes<N>::kChannels, VE = 16 / sizeof(IO), U = kSsmBlock;
    extern __shared__ __align__(16) char smem[];
    typename F::Shared &s = *reinterpret_cast<typename F::Shared *>(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per_group = a.D_ / a.G, group = blockIdx.x / a.blocks, in_group = (blockIdx.x % a.blocks) * CB;
    const int c0 = group * per_group + in_group, cols = min(CB, per_group - in_group);
    const int span = LOCAL ? blockIdx.y + 1 : blockIdx.y;
    const int nl = lane & (LN - 1), cl = lane / LN;
    int mine[KC];
#pragma unroll
    for (int k = 0; k < KC; ++k) mine[k] = (warp * KC + k) * LC + cl;
    auto at = [&](size_t state, int k) { return (state * a.D_ + c0 + mine[k]) * N + nl * 4; };
    auto load = [&](const float *p, size_t state, float (&v)[KC][4]) {
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            const float4 f = p && mine[k] < cols ? *reinterpret_cast<const float4 *>(p + at(state, k)) : make_float4(0.f, 0.f, 0.f, 0.f);
            v[k][0] = f.x, v[k][1] = f.y, v[k][2] = f.z, v[k][3] = f.w;
        }
    };
    auto store = [&](float *p, size_t state, const float (&v)[KC][4]) {
#pragma unroll
        for (int k = 0; k < KC; ++k)
            if (mine[k] < cols) *reinterpret_cast<float4 *>(p + at(state, k)) = make_float4(v[k][0], v[k][1], v[k][2], v[k][3]);
    };
    if (!LOCAL && span >= a.spans) {  // rows without tokens hand on what they get
        for (int row = 0; row < a.rows.n; ++row) {
            if (a.rows.starts[row] != a.rows.starts[row + 1]) continue;
            float v[KC][4];
            load(a.dS_final, row, v);
            store(a.dS_init, row, v);
        }
        return;
    }
    const int lo = span * a.span;
    int hi = (int)min((long long)a.total_rows, (long long)lo + a.span), only = -1;
    if (LOCAL) {
        const SsmToken first = ssm_token(a, lo, false);
        if (first.row < 0 || first.begin >= lo) return;
        only = first.row;
        hi = min(hi, first.end);
    }
    const IO *x = static_cast<const IO *>(a.x) + c0, *dt = static_cast<const IO *>(a.dt) + c0, *z = static_cast<const IO *>(a.z) + (a.z ? c0 : 0);
    const IO *dout = static_cast<const IO *>(a.dout) + c0;
    const IO *Bp = static_cast<const IO *>(a.B) + group * N, *Cp = static_cast<const IO *>(a.C) + group * N;

    float A2[KC][4], carry[KC][4], dA[KC][4], kept[KC][4], sum[KC];
    load(a.A, 0, A2);
#pragma unroll
    for (int k = 0; k < KC; ++k) {
        sum[k] = 0.f;
#pragma unroll
        for (int n = 0; n < 4; ++n) A2[k][n] *= 1.4426950408889634f, carry[k][n] = 0.f, dA[k][n] = 0.f;
    }
    if (!LOCAL && span + 1 < a.spans) {
        const SsmToken last = ssm_token(a, hi - 1, false);
        if (last.row >= 0 && last.end > hi) {  // a row that goes on: what the later stretches hand back, joined
            int j = (last.end - 1) / a.span;
            load(a.local, j, carry);
            for (--j; j > span; --j) {
                float own[KC][4];
                load(a.local, j, own);
#pragma unroll
                for (int k = 0; k < KC; ++k) {
                    const float total = mine[k] < cols ? a.sums[(size_t)j * a.D_ + c0 + mine[k]] : 0.f;
#pragma unroll
                    for (int n = 0; n < 4; ++n) carry[k][n] = fmaf(exp2_fast(A2[k][n] * total), carry[k][n], own[k][n]);
                }
            }
        }
    }
    const int vec = (tid % (CB / VE)) * VE, vec_token = tid / (CB / VE);
    constexpr int kTokenStep = kSsmThreads / (CB / VE) < TT ? kSsmThreads / (CB / VE) : TT;  // (narrow blocks leave threads without a token)
    float bias[VE], skip[VE], dD[VE], dbias[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        bias[e] = a.bias && vec < cols ? a.bias[c0 + vec + e] : 0.f;
        skip[e] = a.D && vec < cols ? a.D[c0 + vec + e] : 0.f;
        dD[e] = dbias[e] = 0.f;
    }
    auto fetch = [&](int t, int stage) {
        typename F::Raw &r = s.raw[stage];
        if (!LOCAL) ssm_stage(r.x, x, a.x_stride, t, TT, lo, hi, CB, cols, kSsmThreads);
        ssm_stage(r.dt, dt, a.dt_stride, t, TT, lo, hi, CB, cols, kSsmThreads);
        ssm_stage(r.dout, dout, a.D_, t, TT, lo, hi, CB, cols, kSsmThreads);
        if (a.z) ssm_stage(r.z, z, a.z_stride, t, TT, lo, hi, CB, cols, kSsmThreads);
        if (!LOCAL) ssm_stage(r.B, Bp, a.B_stride, t, TT, lo, hi, N, N, kSsmThreads);
        ssm_stage(r.C, Cp, a.C_stride, t, TT, lo, hi, N, N, kSsmThreads);
        cp_async_commit();
    };
    const int top = (hi - 1) & ~(TT - 1);  // lo is a multiple of the tile
    fetch(top, 0);
    // (tokens behind the plan's have no kept state)
    auto fetch_kept = [&](int t) { load(t < a.max_tokens ? a.kept : nullptr, (size_t)t / U, kept); };
    if (!LOCAL) fetch_kept((hi - 1) & ~(U - 1));
    int stage = 0;
    for (int t = top; t >= lo; t -= TT, stage ^= 1) {
        const typename F::Raw &r = s.raw[stage];
        if (warp == 0) {
            SsmToken k{-1, -1, 0, 0};
            if (lane < TT && t + lane < hi) k = ssm_token(a, t + lane, false);
            if (LOCAL && k.row != only) k.row = -1;
            if (lane < TT) s.state[lane] = k.state, s.row[lane] = k.row;
            const unsigned begins = __ballot_sync(0xffffffffu, k.row >= 0 && k.begin == t + lane);
            const unsigned ends = __ballot_sync(0xffffffffu, k.row >= 0 && k.end == t + lane + 1);
            const unsigned there = __ballot_sync(0xffffffffu, k.row >= 0);
            if (lane == 0) s.begins = begins, s.ends = ends, s.there = there;
        }
        cp_async_wait_all();
        __syncthreads();
        if (t - TT >= lo) fetch(t - TT, stage ^ 1);
        const unsigned there = s.there, begins = s.begins, ends = s.ends;
#pragma unroll
        for (int q = 0; q < TT / kTokenStep; ++q) {
            const int k = vec_token + q * kTokenStep;
            if (vec_token >= kTokenStep) break;
            const Pack<IO, VE> dv = pack_load<IO, VE>(r.dt + k * CB + vec), gv = pack_load<IO, VE>(r.dout + k * CB + vec);
            Pack<IO, VE> xv, zv;
            if (!LOCAL) xv = pack_load<IO, VE>(r.x + k * CB + vec);
            if (a.z) zv = pack_load<IO, VE>(r.z + k * CB + vec);
            const bool ok = there >> k & 1;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                float d = to_f32(dv.e[e]) + bias[e], g = to_f32(gv.e[e]);
                if (a.softplus) d = ssm_softplus(d);
                if (a.z) {
                    const float zf = to_f32(zv.e[e]);
                    g *= zf * sigmoid(zf);
                }
                s.step[k * CB + vec + e] = ok ? make_float2(d, LOCAL ? 0.f : d * to_f32(xv.e[e])) : make_float2(0.f, 0.f);
                s.dy[k * CB + vec + e] = ok ? g : 0.f;
            }
        }
        for (int i = tid; i < TT * N; i += kSsmThreads) {
            const bool ok = there >> (i / N) & 1;
            if (!LOCAL) s.B[i] = ok ? to_f32(r.B[i]) : 0.f;
            s.C[i] = ok ? to_f32(r.C[i]) : 0.f;
        }
        __syncthreads();
#pragma unroll 1
        for (int k0 = TT - U; k0 >= 0; k0 -= U) {
            if (t + k0 >= hi) continue;
            if (LOCAL) {
#pragma unroll
                for (int i = U - 1; i >= 0; --i) {
                    const int k = k0 + i;
                    if (ends >> k & 1) load(a.dS_final, s.state[k], carry);
                    const float4 Cv = *reinterpret_cast<const float4 *>(s.C + k * N + nl * 4);
                    const float c[4] = {Cv.x, Cv.y, Cv.z, Cv.w};
#pragma unroll
                    for (int q = 0; q < KC; ++q) {
                        const float d = s.step[k * CB + mine[q]].x, dy = s.dy[k * CB + mine[q]];
                        sum[q] += d;
#pragma unroll
                        for (int n = 0; n < 4; ++n) carry[q][n] = exp2_fast(d * A2[q][n]) * fmaf(c[n], dy, carry[q][n]);
                    }
                }
                continue;
            }
            float h[KC][4], decay[U][KC][4], moved[U][KC][4];
#pragma unroll
            for (int q = 0; q < KC; ++q)
#pragma unroll
                for (int n = 0; n < 4; ++n) h[q][n] = kept[q][n];
            if (t + k0 > lo) fetch_kept(t + k0 - U);
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int k = k0 + i;
                if (begins >> k & 1) load(a.S_in, s.state[k], h);
                const float4 Bv = *reinterpret_cast<const float4 *>(s.B + k * N + nl * 4);
                const float b[4] = {Bv.x, Bv.y, Bv.z, Bv.w};
#pragma unroll
                for (int q = 0; q < KC; ++q) {
                    const float2 d = s.step[k * CB + mine[q]];
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        decay[i][q][n] = exp2_fast(d.x * A2[q][n]);
                        moved[i][q][n] = decay[i][q][n] * h[q][n];
                        h[q][n] = fmaf(d.y, b[n], moved[i][q][n]);
                    }
                }
            }
            constexpr int kTogether = LN / 2;  // tokens whose sums over the states run together: three results a lane
            float out[3 * KC * kTogether];
#pragma unroll
            for (int i = U - 1; i >= 0; --i) {
                const int k = k0 + i;
                if (ends >> k & 1) load(a.dS_final, s.state[k], carry);
                const float4 Bv = *reinterpret_cast<const float4 *>(s.B + k * N + nl * 4), Cv = *reinterpret_cast<const float4 *>(s.C + k * N + nl * 4);
                const float b[4] = {Bv.x, Bv.y, Bv.z, Bv.w}, c[4] = {Cv.x, Cv.y, Cv.z, Cv.w};
                float bc[8];
#pragma unroll
                for (int q = 0; q < KC; ++q) {
                    const float2 d = s.step[k * CB + mine[q]];
                    const float dy = s.dy[k * CB + mine[q]];
                    float y = 0.f, sB = 0.f, sA = 0.f;
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const float dh = fmaf(c[n], dy, carry[q][n]), hn = fmaf(d.y, b[n], moved[i][q][n]), w = dh * moved[i][q][n];
                        y = fmaf(c[n], hn, y);
                        sB = fmaf(dh, b[n], sB);
                        sA = fmaf(w, A2[q][n], sA);
                        dA[q][n] = fmaf(w, d.x, dA[q][n]);
                        bc[n] = q ? fmaf(dh, d.y, bc[n]) : dh * d.y;
                        bc[4 + n] = q ? fmaf(dy, hn, bc[4 + n]) : dy * hn;
                        carry[q][n] = decay[i][q][n] * dh;
                    }
                    float *o = out + ((i % kTogether) * KC + q) * 3;
                    o[0] = y, o[1] = sB, o[2] = sA;
                }
                if (begins >> k & 1) {
                    if (a.dS_init) store(a.dS_init, s.state[k], carry);
#pragma unroll
                    for (int q = 0; q < KC; ++q)
#pragma unroll
                        for (int n = 0; n < 4; ++n) carry[q][n] = 0.f;
                }
                const int v0 = lanes_reduce<8, LC, LN>(bc, lane);
#pragma unroll
                for (int j = 0; j < (LC >= 8 ? 1 : 8 / LC); ++j) s.bc[warp][k][((v0 + j) / 4) * N + nl * 4 + (v0 + j) % 4] = bc[j];
                if (i % kTogether == 0) {
                    const int first = lanes_reduce<3 * KC * kTogether, LN>(out, lane) / 3, q = first % KC;
                    const int to = (k + first / KC) * CB + (warp * KC + q) * LC + cl;
                    s.sums[0][to] = out[0], s.sums[1][to] = out[1], s.sums[2][to] = out[2];
                }
            }
        }
        __syncthreads();
        if (LOCAL) continue;
        for (int i = tid; i < TT * 2 * N; i += kSsmThreads) {
            const int k = i / (2 * N), j = i - k * 2 * N;
            if (t + k >= hi) break;
            float v = s.bc[0][k][j];
#pragma unroll
            for (int w = 1; w < kSsmWarps; ++w) v += s.bc[w][k][j];
            a.part_bc[((size_t)blockIdx.x * a.total_rows + t + k) * 2 * N + j] = v;
        }
        if (vec < cols) {
#pragma unroll
            for (int q = 0; q < TT / kTokenStep; ++q) {
                const int k = vec_token + q * kTokenStep;
                if (vec_token >= kTokenStep || t + k >= hi) break;
                const size_t to = (size_t)(t + k) * a.D_ + c0 + vec;
                if (!(there >> k & 1)) {
                    pack_store(static_cast<IO *>(a.dx) + to, pack_zero<IO, VE>());
                    pack_store(static_cast<IO *>(a.ddt) + to, pack_zero<IO, VE>());
                    if (a.dz) pack_store(static_cast<IO *>(a.dz) + to, pack_zero<IO, VE>());
                    continue;
                }
                const Pack<IO, VE> xv = pack_load<IO, VE>(r.x + k * CB + vec), dv = pack_load<IO, VE>(r.dt + k * CB + vec),
                                   gv = pack_load<IO, VE>(r.dout + k * CB + vec);
                Pack<IO, VE> zv, o;
                if (a.z) zv = pack_load<IO, VE>(r.z + k * CB + vec);
                float ddt[VE], dx[VE];
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const int i = k * CB + vec + e;
                    const float xf = to_f32(xv.e[e]), dy = s.dy[i], sB = s.sums[1][i];
                    dx[e] = fmaf(s.step[i].x, sB, skip[e] * dy);
                    ddt[e] = fmaf(xf, sB, s.sums[2][i] * 0.6931471805599453f);
                    if (a.softplus) ddt[e] *= sigmoid(to_f32(dv.e[e]) + bias[e]);
                    dD[e] = fmaf(dy, xf, dD[e]);
                    dbias[e] += ddt[e];
                    if (a.z) {
                        const float zf = to_f32(zv.e[e]), g = sigmoid(zf);
                        o.e[e] = from_f32<IO>(to_f32(gv.e[e]) * fmaf(skip[e], xf, s.sums[0][i]) * g * (1.f + zf * (1.f - g)));
                    }
                }
                pack_store(static_cast<IO *>(a.dx) + to, pack_round<IO, VE>(dx));
                pack_store(static_cast<IO *>(a.ddt) + to, pack_round<IO, VE>(ddt));
                if (a.dz) pack_store(static_cast<IO *>(a.dz) + to, o);
            }
        }
    }
    if (LOCAL) {
        store(a.local, span, carry);
        if (nl == 0)
#pragma unroll
            for (int k = 0; k < KC; ++k)
                if (mine[k] < cols) a.sums[(size_t)span * a.D_ + c0 + mine[k]] = sum[k];
        return;
    }
    store(a.part_A, span, dA);
    // dD and dbias: over the threads that share a vector of channels
    __syncthreads();
    float *over = &s.sums[0][0];  // [kTokenStep][2][CB] of 3 * kTile * CB
    static_assert(kTokenStep * 2 <= 3 * TT, "the tile's sums have room for the columns' ones");
    if (vec_token < kTokenStep)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            over[(vec_token * 2) * CB + vec + e] = dD[e];
            over[(vec_token * 2 + 1) * CB + vec + e] = dbias[e];
        }
    __syncthreads();
    for (int i = tid; i < 2 * cols; i += kSsmThreads) {
        const int n = i / cols, c = i - n * cols;
        float v = 0.f;
        for (int k = 0; k < kTokenStep; ++k) v += over[(k * 2 + n) * CB + c];
        a.part_cols[((size_t)span * 2 + n) * a.D_ + c0 + c] = v;
    }
}

// dB and dC over the blocks of channels of a group (blocks [0, token_blocks)), dA, dD and dbias over the stretches (the rest).
template <typename IO, int N>
__global__ void __launch_bounds__(256) ssm_sums_kernel(const SsmArgs a, long long token_blocks) {
    if (blockIdx.x < token_blocks) {  // four values of a token and group
        constexpr int V = 2 * N / 4;
        const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
        const int v = (int)(i % V) * 4, g = (int)(i / V % a.G);
        const long long t = i / V / a.G;
        if (t >= a.total_rows) return;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (t < a.rows.starts[a.rows.n]) {
            const float *p = a.part_bc + ((size_t)g * a.blocks * a.total_rows + t) * 2 * N + v;
#pragma unroll 8
            for (int b = 0; b < a.blocks; ++b) {
                const float4 f = *reinterpret_cast<const float4 *>(p + (size_t)b * a.total_rows * 2 * N);
                s.x += f.x, s.y += f.y, s.z += f.z, s.w += f.w;
            }
        }
        const float f[4] = {s.x, s.y, s.z, s.w};
        pack_store(static_cast<IO *>(v < N ? a.dB : a.dC) + ((size_t)t * a.G + g) * N + v % N, pack_round<IO, 4>(f));
        return;
    }
    const long long i = ((long long)blockIdx.x - token_blocks) * 256 + threadIdx.x, states = (long long)a.D_ * N;
    if (i < states) {
        float s = 0.f;
#pragma unroll 8
        for (int k = 0; k < a.spans; ++k) s += a.part_A[(size_t)k * states + i];
        a.dA[i] = s;
    } else if (i < states + 2 * a.D_) {
        const long long c = i - states;
        float *to = c < a.D_ ? a.dD : a.dbias;
        if (!to) return;
        float s = 0.f;
#pragma unroll 8
        for (int k = 0; k < a.spans; ++k) s += a.part_cols[(size_t)k * 2 * a.D_ + c];
        to[c < a.D_ ? c : c - a.D_] = s;
    }
}

}  // namespace deltalog
