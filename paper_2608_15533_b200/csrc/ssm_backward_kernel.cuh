// Gradients of the selective state space scan.  With dy = dout silu(z) and dh_t the adjoint of h_t:
//     dh_t = C dy_t + a_(t+1) dh_(t+1)            dC = sum over channels dy h,   dB = sum over channels dh delta x
//     dx = delta sum dh B + D dy                  ddelta = x sum dh B + sum dh (a h_(t-1)) A,   ddt = ddelta sigmoid(dt + bias)
//     dA = sum_t dh (a h_(t-1)) delta             dz = dout (C h + D x) silu'(z),   dS_init = a_first dh_first
//
// Walks from the last token to the first: the forward pass kept the state in front of every eighth, from which a lane runs over
// the lower four, then over the upper four with a and a h_(t-1) in registers, goes back over those, and does the same with the
// lower four.  (The states of every token would be 8 times the bytes; all eight tokens in registers took 255 of them and 992 us
// where four took 714.)  a h_(t-1) is kept rather than h_t, from which it would come out by a difference that cancels where the
// decay is strong.  Sums over a channel's states run over several values at once (lanes_reduce), over a warp's channels in the same way
// or in shared memory, over the warps in shared memory, over the CTAs in ssm_sums_kernel; each in a fixed order.
// Bound by latency between its instructions: 56 % of the issue slots and 35 % of the special function units are busy.  24 instructions per
// token, channel and state by the counters (13 of them products and sums, 4 the exchange of partial sums), three barriers a tile between
// phases of different kinds, and the 12 warps an SM that 168 registers leave.  8k tokens x 4096 x 16 states 684 us; the first pass 153 (175
// in the second pass's layout), the sums 17.  One channel a lane instead of two (20 warps) had 915 where two had 714: its sums over channels
// cost twice as much.
#pragma once

#include "ssm_common.cuh"

namespace deltalog {

// The first pass brings in no x and no B, and needs none of the sums: it has room for tiles twice as long and a fourth CTA.
template <typename IO, int N, bool LOCAL> struct SsmBackward {
    static constexpr int kPer = 2;
    static constexpr int kCols = kSsmWarps * SsmLanes<N>::kChannels * kPer, kTile = LOCAL ? 32 : 16;
    // dB and dC over a warp's channels: eight or more of them in shared memory, two tokens at a time (each token by exchanges between
    // the lanes: 714 us where 681 are taken); of four or two the exchanges are short (32 states: 400 us, in shared memory 405).
    static constexpr bool kInMemory = !LOCAL && SsmLanes<N>::kChannels >= 8;
    static constexpr int full(int n) { return LOCAL ? 8 : n; }  // elements of what the first pass does without (multiples of 16 bytes)
    struct Raw {
        IO dt[kTile * kCols], z[kTile * kCols], dout[kTile * kCols], C[kTile * N], x[full(kTile * kCols)], B[full(kTile * N)];
    };
    static constexpr int kPitch = kCols + 16;  // lanes that answer for neighbouring tokens store to different banks
    struct alignas(16) Shared {
        Raw raw[2];
        float2 step[kTile * kCols];                          // delta, delta x; in the first pass delta, dy
        float C[kTile * N];
        float dy[full(kTile * kCols)], slope[full(kTile * kCols)];  // slope: softplus'
        float sums[3][full(kTile * kPitch)];                 // C . h, sum dh B, sum dh a h_(t-1) A (A in powers of two)
        float B[full(kTile * N)];
        float bc[kSsmWarps][full(kTile)][2 * N];
        float4 product[kInMemory ? kSsmWarps : 1][2][2][32]; // of two tokens: a lane's four states of dB and of dC
        float lift[LOCAL ? 1 : kPer][kSsmThreads];           // a thread's own (in registers they made the sums spill: 730 us where 683 are taken)
        int state[kTile], row[kTile];
        unsigned begins, ends, there;
    };
    static constexpr int kCtas = ssm_ctas(LOCAL && N <= 32 ? 4 : 3, sizeof(Shared));  // on an SM
};

// LOCAL: the first pass over a part of a stretch (`span` is the part), where its first row began in front of the stretch: the adjoint
// that the part alone hands back.
template <typename IO, int N, bool LOCAL>
__global__ void __launch_bounds__(kSsmThreads, (SsmBackward<IO, N, LOCAL>::kCtas)) ssm_backward_kernel(const SsmArgs a) {
    using F = SsmBackward<IO, N, LOCAL>;
    constexpr int KC = F::kPer, CB = F::kCols, PB = F::kPitch, TT = F::kTile, LN = SsmLanes<N>::kStates, LC = SsmLanes<N>::kChannels, U = kSsmBlock;
    extern __shared__ __align__(16) char smem[];
    typename F::Shared &s = *reinterpret_cast<typename F::Shared *>(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per_group = a.D_ / a.G, group = blockIdx.x / a.blocks, in_group = (blockIdx.x % a.blocks) * CB;
    const int c0 = group * per_group + in_group, cols = min(CB, per_group - in_group);
    const int span = blockIdx.y;
    const int nl = lane & (LN - 1), cl = lane / LN;
    const int first = warp * KC * LC + cl;  // this lane's channels of the block: first, first + LC
    auto at = [&](size_t state, int q) { return (state * a.D_ + c0 + first + q * LC) * N + nl * 4; };
    auto mine = [&](int q) { return first + q * LC < cols; };
    auto load = [&](const float *p, size_t state, float2 (&v)[KC][2]) {
#pragma unroll
        for (int q = 0; q < KC; ++q) {
            v[q][0] = v[q][1] = both(0.f);
            if (p && mine(q)) ssm_load(p + at(state, q), v[q]);
        }
    };
    auto store = [&](float *p, size_t state, const float2 (&v)[KC][2]) {
#pragma unroll
        for (int q = 0; q < KC; ++q)
            if (mine(q)) ssm_store(p + at(state, q), v[q]);
    };
    if (!LOCAL && span >= a.spans) {  // rows without tokens hand on what they get
        ssm_empty_rows(a, span - a.spans, [&](int row) {
            float2 v[KC][2];
            load(a.dS_final, row, v);
            store(a.dS_init, row, v);
        });
        return;
    }
    const int length = LOCAL ? a.part : a.span, lo = span * length, bound = (int)min((long long)a.total_rows, (long long)lo + length);
    int hi = max(lo, min(bound, a.rows.starts[a.rows.n])), only = -1;  // the tokens that there are
    if (LOCAL) {
        const SsmToken head = ssm_token(a, lo, false);
        if (hi == lo || head.row < 0 || head.begin >= lo / a.span * a.span) return;
        only = head.row;
        hi = min(hi, head.end);
    }
    const IO *x = static_cast<const IO *>(a.x) + c0, *dt = static_cast<const IO *>(a.dt) + c0, *z = static_cast<const IO *>(a.z) + (a.z ? c0 : 0);
    const IO *dout = static_cast<const IO *>(a.dout) + c0;
    const IO *Bp = static_cast<const IO *>(a.B) + group * N, *Cp = static_cast<const IO *>(a.C) + group * N;

    float2 A2[KC][2], carry[KC][2], dA[KC][2], kept[KC][2];
    float sum[KC];
    struct Lift { float of[KC]; };
    Lift lift;  // of the decays; at first the bias that it goes by
#pragma unroll
    for (int q = 0; q < KC; ++q) lift.of[q] = a.bias && mine(q) ? a.bias[c0 + first + q * LC] : 0.f;
    load(a.A, 0, A2);
#pragma unroll
    for (int q = 0; q < KC; ++q) {
        sum[q] = 0.f;
#pragma unroll
        for (int p = 0; p < 2; ++p) A2[q][p] = __fmul2_rn(A2[q][p], both(1.4426950408889634f)), carry[q][p] = dA[q][p] = both(0.f);
    }
#pragma unroll
    for (int q = 0; q < KC; ++q) {
        lift.of[q] = ssm_lift(a, A2[q], lift.of[q]);
        if (!LOCAL) s.lift[q][tid] = lift.of[q];
    }
    if (!LOCAL && hi > lo) {
        const SsmToken last = ssm_token(a, hi - 1, false);
        if (last.row >= 0 && last.end > hi) load(a.local, hi / a.part, carry);  // what the later stretches hand back to a row that goes on
    }
    // the two channels that this thread brings in and out, and its first token of a tile
    const int col = (tid % (CB / 2)) * 2, col_token = tid / (CB / 2);
    constexpr int kTokenStep = kSsmThreads / (CB / 2);
    static_assert(kTokenStep <= TT, "every thread has tokens");
    const float2 bias = a.bias && col < cols ? load2(a.bias + c0 + col) : both(0.f), skip = a.D && col < cols ? load2(a.D + c0 + col) : both(0.f);
    float2 dD = both(0.f), dbias = both(0.f);
    auto fetch = [&](int t, int stage) {
        typename F::Raw &r = s.raw[stage];
        auto parts = [&](auto all) {
            constexpr bool ALL = decltype(all)::value;
            ssm_stage<ALL, TT, CB>(r.dt, dt, a.dt_stride, t, lo, hi, cols);
            ssm_stage<ALL, TT, CB>(r.dout, dout, a.D_, t, lo, hi, cols);
            if (a.z) ssm_stage<ALL, TT, CB>(r.z, z, a.z_stride, t, lo, hi, cols);
            ssm_stage<ALL, TT, N>(r.C, Cp, a.C_stride, t, lo, hi, N);
            if (!LOCAL) {
                ssm_stage<ALL, TT, CB>(r.x, x, a.x_stride, t, lo, hi, cols);
                ssm_stage<ALL, TT, N>(r.B, Bp, a.B_stride, t, lo, hi, N);
            }
        };
        if (t + TT <= hi && cols == CB) parts(std::true_type{});
        else parts(std::false_type{});
        cp_async_commit();
    };
    const int top = hi > lo ? (hi - 1) & ~(TT - 1) : lo - TT;  // lo is a multiple of the tile
    auto fetch_kept = [&](int t) { load(a.kept, (size_t)t / U, kept); };
    if (hi > lo) {
        fetch(top, 0);
        if (!LOCAL) fetch_kept((hi - 1) & ~(U - 1));
    }
    int stage = 0;
    for (int t = top; t >= lo; t -= TT, stage ^= 1) {
        typename F::Raw &r = s.raw[stage];
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
        for (int i = 0; i < TT / kTokenStep; ++i) {
            const int k = col_token + i * kTokenStep, to = k * CB + col;
            const float2 v = __fadd2_rn(load2(r.dt + to), bias);
            float2 d = v, e, g = load2(r.dout + to), u = both(0.f);
            if (a.softplus) {
                d = ssm_softplus(v, e);
                if (!LOCAL) store2(s.slope + to, make_float2(ssm_sigmoid(v.x, e.x), ssm_sigmoid(v.y, e.y)));
            }
            if (a.z) {
                const float2 zf = load2(r.z + to);
                g = __fmul2_rn(g, make_float2(zf.x * sigmoid(zf.x), zf.y * sigmoid(zf.y)));
            }
            if (LOCAL) u = g;
            else u = __fmul2_rn(d, load2(r.x + to)), store2(s.dy + to, g);
            *reinterpret_cast<float4 *>(s.step + to) = make_float4(d.x, u.x, d.y, u.y);
        }
        if (there != (unsigned)((1ull << TT) - 1)) {  // a skipped token may hold anything, and changes nothing
#pragma unroll
            for (int i = 0; i < TT / kTokenStep; ++i) {
                const int k = col_token + i * kTokenStep, to = k * CB + col;
                if (there >> k & 1) continue;
                *reinterpret_cast<float4 *>(s.step + to) = make_float4(0.f, 0.f, 0.f, 0.f);
                if (!LOCAL) store2(s.dy + to, both(0.f));
            }
            for (int i = tid; i < TT * N; i += kSsmThreads)
                if (!(there >> (i / N) & 1)) {
                    r.C[i] = from_f32<IO>(0.f);
                    if (!LOCAL) r.B[i] = from_f32<IO>(0.f);
                }
            __syncthreads();
        }
#pragma unroll
        for (int i0 = 0; i0 < TT * N / 2; i0 += kSsmThreads) {
            const int i = 2 * (i0 + tid);
            if (TT * N / 2 % kSsmThreads && i >= TT * N) break;
            if (!LOCAL) store2(s.B + i, load2(r.B + i));
            store2(s.C + i, load2(r.C + i));
        }
        __syncthreads();
        auto lifts = [&]() {
            Lift v = lift;
            if constexpr (!LOCAL)
#pragma unroll
                for (int q = 0; q < KC; ++q) v.of[q] = s.lift[q][tid];
            return v;
        };
        // four tokens; MARKED: where rows may begin or end
        auto back = [&](int k0, auto marked) {
            constexpr bool MARKED = decltype(marked)::value;
            const float2 *step = s.step + k0 * CB + first;
            const Lift up = lifts();
#pragma unroll
            for (int i = 3; i >= 0; --i) {
                if (MARKED && (ends >> (k0 + i) & 1)) load(a.dS_final, s.state[k0 + i], carry);
                float2 c[2];
                ssm_pairs(s.C + (k0 + i) * N + nl * 4, c);
#pragma unroll
                for (int q = 0; q < KC; ++q) {
                    const float2 d = step[i * CB + q * LC];
                    sum[q] += d.x;
#pragma unroll
                    for (int p = 0; p < 2; ++p)
                        carry[q][p] = __fmul2_rn(ssm_decay(A2[q][p], d.x, up.of[q]), __ffma2_rn(c[p], both(d.y), carry[q][p]));
                }
            }
        };
        auto ahead = [&](int k0, auto &h, auto marked) {
            constexpr bool MARKED = decltype(marked)::value;
            const float2 *step = s.step + k0 * CB + first;
            const Lift up = lifts();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (MARKED && (begins >> (k0 + i) & 1)) load(a.S_in, s.state[k0 + i], h);
                float2 b[2];
                ssm_pairs(s.B + (k0 + i) * N + nl * 4, b);
#pragma unroll
                for (int q = 0; q < KC; ++q) {
                    const float2 d = step[i * CB + q * LC];
#pragma unroll
                    for (int p = 0; p < 2; ++p)
                        h[q][p] = __ffma2_rn(ssm_decay(A2[q][p], d.x, up.of[q]), h[q][p], __fmul2_rn(both(d.y), b[p]));
                }
            }
        };
        // dB and dC of two tokens over the warp's channels: a lane sums N / 8 neighbouring values over the channels' LC rows.  (The rows
        // are walked from another one in each quarter of the values, so that lanes side by side read different banks.)
        auto sum_products = [&](int k0) {
            constexpr int V = N / 8;
            const int part = lane / 8, v = lane % 8 * V;  // part: token, dB or dC
            const float *p = reinterpret_cast<const float *>(s.product[warp][part / 2][part % 2]) + v;
            Pack<float, V> sum = pack_load<float, V>(p + (part & (LC - 1)) * N);
#pragma unroll
            for (int r = 1; r < LC; ++r) {
                const Pack<float, V> f = pack_load<float, V>(p + ((r + part) & (LC - 1)) * N);
#pragma unroll
                for (int e = 0; e < V; ++e) sum.e[e] += f.e[e];
            }
            pack_store(&s.bc[warp][k0 + part / 2][part % 2 * N + v], sum);
        };
        auto both_ways = [&](int k0, auto &h, auto marked) {
            constexpr bool MARKED = decltype(marked)::value;
            const float2 *step = s.step + k0 * CB + first;
            const float *dys = s.dy + k0 * CB + first;
            const Lift up = lifts();
            float2 decay[4][KC][2], moved[4][KC][2];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (MARKED && (begins >> (k0 + i) & 1)) load(a.S_in, s.state[k0 + i], h);
                float2 b[2];
                ssm_pairs(s.B + (k0 + i) * N + nl * 4, b);
#pragma unroll
                for (int q = 0; q < KC; ++q) {
                    const float2 d = step[i * CB + q * LC];
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        decay[i][q][p] = ssm_decay(A2[q][p], d.x, up.of[q]);
                        moved[i][q][p] = __fmul2_rn(decay[i][q][p], h[q][p]);
                        if (i < 3) h[q][p] = __ffma2_rn(both(d.y), b[p], moved[i][q][p]);
                    }
                }
            }
            constexpr int kTogether = LN / 2 < 4 ? LN / 2 : 4;  // tokens whose sums over the states run together: three results a lane
            float out[3 * KC * kTogether];
#pragma unroll
            for (int i = 3; i >= 0; --i) {
                if (MARKED && (ends >> (k0 + i) & 1)) load(a.dS_final, s.state[k0 + i], carry);
                float2 b[2], c[2], bc[4];
                ssm_pairs(s.B + (k0 + i) * N + nl * 4, b);
                ssm_pairs(s.C + (k0 + i) * N + nl * 4, c);
#pragma unroll
                for (int q = 0; q < KC; ++q) {
                    const float2 d = step[i * CB + q * LC];
                    const float2 dy = both(dys[i * CB + q * LC]), delta = both(d.x), u = both(d.y);
                    float2 y, sB, sA;
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const float2 dh = __ffma2_rn(c[p], dy, carry[q][p]), hn = __ffma2_rn(u, b[p], moved[i][q][p]), w = __fmul2_rn(dh, moved[i][q][p]);
                        y = p ? __ffma2_rn(c[p], hn, y) : __fmul2_rn(c[p], hn);
                        sB = p ? __ffma2_rn(dh, b[p], sB) : __fmul2_rn(dh, b[p]);
                        sA = p ? __ffma2_rn(w, A2[q][p], sA) : __fmul2_rn(w, A2[q][p]);
                        dA[q][p] = __ffma2_rn(w, delta, dA[q][p]);
                        bc[p] = q ? __ffma2_rn(dh, u, bc[p]) : __fmul2_rn(dh, u);
                        bc[2 + p] = q ? __ffma2_rn(dy, hn, bc[2 + p]) : __fmul2_rn(dy, hn);
                        carry[q][p] = __fmul2_rn(decay[i][q][p], dh);
                    }
                    float *o = out + ((i % kTogether) * KC + q) * 3;
                    o[0] = y.x + y.y, o[1] = sB.x + sB.y, o[2] = sA.x + sA.y;
                }
                if (MARKED && (begins >> (k0 + i) & 1)) {
                    if (a.dS_init) store(a.dS_init, s.state[k0 + i], carry);
#pragma unroll
                    for (int q = 0; q < KC; ++q) carry[q][0] = carry[q][1] = both(0.f);
                }
                if constexpr (F::kInMemory) {
                    s.product[warp][i % 2][0][lane] = make_float4(bc[0].x, bc[0].y, bc[1].x, bc[1].y);
                    s.product[warp][i % 2][1][lane] = make_float4(bc[2].x, bc[2].y, bc[3].x, bc[3].y);
                    if (i % 2 == 0) {
                        __syncwarp();
                        sum_products(k0 + i);
                        __syncwarp();
                    }
                } else {
                    float v[8] = {bc[0].x, bc[0].y, bc[1].x, bc[1].y, bc[2].x, bc[2].y, bc[3].x, bc[3].y};
                    const int v0 = lanes_reduce<8, LC, LN>(v, lane);
#pragma unroll
                    for (int j = 0; j < 8 / LC; ++j) s.bc[warp][k0 + i][((v0 + j) / 4) * N + nl * 4 + (v0 + j) % 4] = v[j];
                }
                if (i % kTogether == 0) {
                    const int o0 = lanes_reduce<3 * KC * kTogether, LN>(out, lane) / 3;
                    const int to = (k0 + i + o0 / KC) * PB + first + o0 % KC * LC;
                    s.sums[0][to] = out[0], s.sums[1][to] = out[1], s.sums[2][to] = out[2];
                }
            }
        };
#pragma unroll 1
        for (int k0 = TT - U; k0 >= 0; k0 -= U) {
            if (t + k0 >= hi) continue;
            const bool low = (begins | ends) >> k0 & 15, high = (begins | ends) >> (k0 + 4) & 15;
            if constexpr (LOCAL) {
                if (high) back(k0 + 4, std::true_type{});
                else back(k0 + 4, std::false_type{});
                if (low) back(k0, std::true_type{});
                else back(k0, std::false_type{});
            } else {
                float2 h[KC][2];
#pragma unroll
                for (int q = 0; q < KC; ++q) h[q][0] = kept[q][0], h[q][1] = kept[q][1];
                if (low || high) {
                    ahead(k0, h, std::true_type{});
                    both_ways(k0 + 4, h, std::true_type{});
                } else {
                    ahead(k0, h, std::false_type{});
                    both_ways(k0 + 4, h, std::false_type{});
                }
#pragma unroll
                for (int q = 0; q < KC; ++q) h[q][0] = kept[q][0], h[q][1] = kept[q][1];
                if (t + k0 > lo) fetch_kept(t + k0 - U);
                if (low || high) both_ways(k0, h, std::true_type{});
                else both_ways(k0, h, std::false_type{});
            }
        }
        __syncthreads();
        if constexpr (!LOCAL) {
            for (int i = tid; i < TT * 2 * N; i += kSsmThreads) {
                const int k = i / (2 * N), j = i - k * 2 * N;
                if (t + k >= hi) break;
                float v = s.bc[0][k][j];
#pragma unroll
                for (int w = 1; w < kSsmWarps; ++w) v += s.bc[w][k][j];
                a.part_bc[((size_t)blockIdx.x * a.total_rows + t + k) * 2 * N + j] = v;
            }
            if (col < cols) {
                const int here = min(TT, hi - t);
#pragma unroll
                for (int i = 0; i < TT / kTokenStep; ++i) {
                    const int k = col_token + i * kTokenStep, n = k * CB + col, sn = k * PB + col;
                    if (k >= here) break;
                    const size_t to = (size_t)(t + k) * a.D_ + c0 + col;
                    IO *dx = static_cast<IO *>(a.dx) + to, *ddt = static_cast<IO *>(a.ddt) + to, *dz = static_cast<IO *>(a.dz) + (a.dz ? to : 0);
                    const float4 st = *reinterpret_cast<const float4 *>(s.step + n);
                    const float2 xf = load2(r.x + n), dy = load2(s.dy + n), sB = load2(s.sums[1] + sn), sA = load2(s.sums[2] + sn);
                    float2 g = __ffma2_rn(xf, sB, __fmul2_rn(sA, both(0.6931471805599453f)));
                    if (a.softplus) g = __fmul2_rn(g, load2(s.slope + n));
                    store2(dx, __ffma2_rn(make_float2(st.x, st.z), sB, __fmul2_rn(skip, dy)));
                    store2(ddt, g);
                    dD = __ffma2_rn(dy, xf, dD), dbias = __fadd2_rn(dbias, g);
                    if (a.z) {
                        const float2 zf = load2(r.z + n), y = __fmul2_rn(load2(r.dout + n), __ffma2_rn(skip, xf, load2(s.sums[0] + sn)));
                        const float g0 = sigmoid(zf.x), g1 = sigmoid(zf.y);
                        store2(dz, make_float2(y.x * g0 * fmaf(zf.x, 1.f - g0, 1.f), y.y * g1 * fmaf(zf.y, 1.f - g1, 1.f)));
                    }
                }
            }
        }
    }
    if constexpr (LOCAL) {
        store(a.local, span, carry);
        if (nl == 0)
#pragma unroll
            for (int q = 0; q < KC; ++q)
                if (mine(q)) a.sums[(size_t)span * a.D_ + c0 + first + q * LC] = sum[q];
    } else {
        store(a.part_A, span, dA);
        if (col < cols)  // behind the last sequence
            for (int t = hi + col_token; t < bound; t += kTokenStep) {
                const size_t to = (size_t)t * a.D_ + c0 + col;
                store2(static_cast<IO *>(a.dx) + to, both(0.f)), store2(static_cast<IO *>(a.ddt) + to, both(0.f));
                if (a.dz) store2(static_cast<IO *>(a.dz) + to, both(0.f));
            }
        // dD and dbias: over the threads that share a pair of channels
        __syncthreads();
        float *over = &s.sums[0][0];  // [2][kTokenStep][CB]
        static_assert(2 * kTokenStep * CB <= 3 * TT * PB, "the tile's sums have room for the columns' ones");
        store2(over + col_token * CB + col, dD);
        store2(over + (kTokenStep + col_token) * CB + col, dbias);
        __syncthreads();
        for (int i = tid; i < 2 * cols; i += kSsmThreads) {
            const int n = i / cols, c = i - n * cols;
            float v = 0.f;
#pragma unroll
            for (int k = 0; k < kTokenStep; ++k) v += over[(n * kTokenStep + k) * CB + c];
            a.part_cols[((size_t)span * 2 + n) * a.D_ + c0 + c] = v;
        }
    }
}

// dB and dC over the blocks of channels of a group (blocks [0, token_blocks)), dA, dD and dbias over the stretches (the rest).
template <typename IO, int N>
__global__ void __launch_bounds__(256) ssm_sums_kernel(const SsmArgs a, long long token_blocks) {
    if (blockIdx.x < token_blocks) {  // 64 vectors of four values, four threads each: a quarter of the blocks of channels
        constexpr int V = 2 * N / 4;
        __shared__ float4 quarter[4][64];
        const int part = threadIdx.x / 64, item = threadIdx.x % 64;
        const long long i = (long long)blockIdx.x * 64 + item;
        const int v = (int)(i % V) * 4, g = (int)(i / V % a.G);
        const long long t = i / V / a.G;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        auto add = [&](const float4 &f) { s.x += f.x, s.y += f.y, s.z += f.z, s.w += f.w; };
        if (t < a.rows.starts[a.rows.n]) {
            const float *p = a.part_bc + ((size_t)g * a.blocks * a.total_rows + t) * 2 * N + v;
#pragma unroll 8
            for (int b = part; b < a.blocks; b += 4) add(*reinterpret_cast<const float4 *>(p + (size_t)b * a.total_rows * 2 * N));
        }
        quarter[part][item] = s;
        __syncthreads();
        if (part || t >= a.total_rows) return;
#pragma unroll
        for (int k = 1; k < 4; ++k) add(quarter[k][item]);
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
