// Between the two passes of the state space scan: what every part leaves (or hands back) becomes what it leaves with
// everything in front of it, part by part,
//     h_p <- h_p + exp(A sum_p) h_(p-1)      where the row that is open at the end of part p began in front of the part,
// and from the last part to the first for the adjoints, where the row that part p begins in goes on behind it.
// (One decay a part: what the hardware's 2^x is low on average, ssm_lift, does not add up here.)
// A lane holds four states of a channel and runs over the parts, sixteen of whose values are loaded at a time: the steps between
// depend on one another, the loads do not (one at a time, in the second pass, they took 0.5 us a part).
#pragma once

#include "ssm_common.cuh"

namespace deltalog {

constexpr int kSsmJoin = 16;

template <bool BACK>
__global__ void __launch_bounds__(128) ssm_join_kernel(const SsmArgs a, int states) {
    extern __shared__ unsigned char joined[];  // [parts]
    const int tokens = BACK ? a.total_rows : a.max_tokens, there = min(tokens, a.rows.starts[a.rows.n]);
    for (int p = threadIdx.x; p < a.parts; p += blockDim.x) {
        const int lo = p * a.part, hi = (int)min((long long)there, (long long)lo + a.part);
        bool on = false;
        if (hi > lo) {
            const SsmToken k = ssm_token(a, BACK ? lo : hi - 1, false);
            on = k.row >= 0 && (BACK ? k.end > (long long)lo + a.part : k.begin < lo);
        }
        joined[p] = on;
    }
    __syncthreads();
    const long long i = ((long long)blockIdx.x * 128 + threadIdx.x) * 4;  // state
    const long long all = (long long)a.D_ * states;
    if (i >= all) return;
    const int channel = (int)(i / states);
    float2 A2[2], h[2] = {both(0.f), both(0.f)};
    ssm_load(a.A + i, A2);
    A2[0] = __fmul2_rn(A2[0], both(1.4426950408889634f)), A2[1] = __fmul2_rn(A2[1], both(1.4426950408889634f));
    for (int p0 = 0; p0 < a.parts; p0 += kSsmJoin) {
        float2 own[kSsmJoin][2];
        float sum[kSsmJoin];
        auto at = [&](int k) { return BACK ? a.parts - 1 - min(p0 + k, a.parts - 1) : min(p0 + k, a.parts - 1); };
#pragma unroll
        for (int k = 0; k < kSsmJoin; ++k) ssm_load(a.local + at(k) * all + i, own[k]), sum[k] = a.sums[(size_t)at(k) * a.D_ + channel];
#pragma unroll
        for (int k = 0; k < kSsmJoin; ++k) {
            if (p0 + k >= a.parts) break;
            const bool on = joined[at(k)];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float2 decay = exp2_fast(__fmul2_rn(A2[e], both(sum[k])));
                h[e] = on ? __ffma2_rn(decay, h[e], own[k][e]) : own[k][e];
            }
            if (on) ssm_store(a.local + at(k) * all + i, h);
        }
    }
}

}  // namespace deltalog
