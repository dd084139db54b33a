// The backward chain for d_v = 128 on the 5th-generation tensor cores: scan_forward_tc_kernel's layout, from the last chunk to
// the first.  Thread (lane v, quarter f) keeps dS[c][v] of a quarter of the channels; per chunk
//     dS planes -> tensor memory;  dU = (k e^(G_end - G)) dS + A^T dO;  dU planes;  dV = T^T dU;
//     dO and dV planes (scalar decay: times their tokens' factors);  dS <- e^(G_end) dS + dO^T (scale q e^G) - dV^T (k e^G).
// Bound as the forward chain is, and by the 64 KB of dS that every chunk leaves for its gradients.  (Taking dO's products off the
// chain's path -- its planes up front, dO^T q beside T^T dU -- changed nothing: 939 us and 939 for a step of 8k tokens.)
// GDN, bf16, 32 heads of 128: 225 us for four rows of 2048 tokens, 942 us for 36.7k tokens of 19 rows; KDA 3.9k tokens of 5 rows 141 us.
#pragma once

#include "scan_tc_common.cuh"

namespace deltalog {

template <bool VEC, int P, int DK, bool DELTA, typename IO>
struct BackwardTcSmem {
    static constexpr bool kF32 = sizeof(IO) == 4;
    static constexpr int kTile = kChunk * DK * 2, kMat = kChunk * kChunk * 2;
    static constexpr int kVecs = VEC ? kPlanes : P;
    static constexpr int kDecay = VEC ? DK * 4 : 2 * kChunk * 4;
    static constexpr int kStages = !VEC && P == 1 ? 2 : 1;
    static constexpr bool kRaw = !VEC && P == 1;  // q and k as they are, copied by all threads
    // group 0: k for dU (scalar decay: for the update as well) and the decay factors; group 1: A, T; group 2: q and, per channel,
    // k e^G.
    static constexpr int kh = 0;
    static constexpr int q = kh + kVecs * kTile;
    static constexpr int kt = q + kVecs * kTile;
    static constexpr int A = kt + (VEC && DELTA ? kVecs * kTile : 0);
    static constexpr int T = A + kPlanes * kMat;
    static constexpr int stage = T + (DELTA ? kPlanes * kMat : 0);
    static constexpr int rows = kStages * stage;                   // bf16 io: dO, and dv on its way out
    static constexpr int decay = rows + (kF32 ? 0 : 2 * kChunk * 256);
    static constexpr int control = decay + 2 * kDecay;
    static constexpr size_t total = control + kTcControlBytes;
    static constexpr size_t bytes = total > kTcMinSmem ? total : kTcMinSmem;
};

template <bool VEC, int P, int DK, bool DELTA, typename IO>
__global__ void __launch_bounds__(kTcThreads, 1) scan_backward_tc_kernel(const ScanArgs a) {
    using L = BackwardTcSmem<VEC, P, DK, DELTA, IO>;
    constexpr int DV = 128, HC = DK / 4, HT = kChunk / 4;
    constexpr int NST = L::kStages;
    constexpr bool F32IO = L::kF32;
    constexpr int OP1 = F32IO ? kPlanes : 1;  // planes of dO
    constexpr int OP2 = VEC ? OP1 : kPlanes;  // and of dO times a scalar decay
    // tensor memory: accumulators of (k dS)^T, of dO^T A, of dV^T, of the update; planes of dS, later of
    // dU and then of dV; planes of dO, as it is and for the update
    constexpr uint32_t ACC0 = 0, ACC1 = 64, ACC2 = 128, UPD = 192, PL = 320, PLO = 416;
    extern __shared__ __align__(1024) unsigned char smem_tc[];
    const uint32_t sm = smem_addr(smem_tc);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int v = 32 * (warp & 3) + lane, f = warp >> 2;
    scan_kernel_begin();
    const int seq = a.order[blockIdx.x / a.H], h = blockIdx.x % a.H, hq = h / (a.H / a.Hq);
    const int tok0 = a.starts[seq], len = a.starts[seq + 1] - tok0, nchunks = (len + kChunk - 1) / kChunk;
    const int chunk0 = a.chunk_starts[seq];
    const size_t tile = (size_t)DK * DV, s_off = ((size_t)seq * a.H + h) * tile;
    const size_t v_stride = (size_t)a.H * DV;
    const TcBlock tc = tc_setup(smem_tc + L::control, 3 * NST + 1, tid);
    const uint32_t row = tc.tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    const uint32_t mma_bar = tc.bars + 8u * (3 * NST);
    const uint32_t do_s = sm + L::rows, out_s = do_s + kChunk * 256;
    const IO *dsrc = static_cast<const IO *>(a.dout) + (size_t)tok0 * v_stride + (size_t)h * DV;
    IO *odst = static_cast<IO *>(a.dv_out) + (size_t)tok0 * v_stride + (size_t)h * DV;
    const bool loader = tid == 128, storer = lane < 4;
    bool ok = true;

    // `n` counts the chunks as they are taken; chunk c = nchunks - 1 - n
    auto full = [&](int group, int n) { return tc.bars + 8u * (3 * (n % NST) + group); };
    auto load_group = [&](int group, int n) {  // one thread
        if (n >= nchunks || *tc.abort_flag) return;
        const int c = nchunks - 1 - n;
        const size_t unit = (size_t)(chunk0 + c) * a.H + h, qunit = (size_t)(chunk0 + c) * a.Hq + hq;
        const uint32_t st = sm + (n % NST) * L::stage, bar = full(group, n);
        const size_t vec = unit * kPlanes * kChunk * DK, qvec = qunit * P * kChunk * DK, mat = unit * kPlanes * kChunk * kChunk;
        if (group == 0) {
            mbar_arrive_expect_tx(bar, (L::kRaw ? 0 : L::kVecs * L::kTile) + L::kDecay);
            if (!L::kRaw) bulk_copy_g2s(st + L::kh, VEC ? a.kh + vec : a.ki + qvec, L::kVecs * L::kTile, bar);
            bulk_copy_g2s(sm + L::decay + (n & 1) * L::kDecay, a.decay + unit * (L::kDecay / 4), L::kDecay, bar);
        } else if (group == 1) {
            mbar_arrive_expect_tx(bar, (DELTA ? 2 : 1) * kPlanes * L::kMat);
            bulk_copy_g2s(st + L::A, a.A + mat, kPlanes * L::kMat, bar);
            if (DELTA) bulk_copy_g2s(st + L::T, a.T + mat, kPlanes * L::kMat, bar);
        } else {
            mbar_arrive_expect_tx(bar, (VEC && DELTA ? 2 : 1) * L::kVecs * L::kTile);
            bulk_copy_g2s(st + L::q, VEC ? a.qt + vec : a.qi + qvec, L::kVecs * L::kTile, bar);
            if (VEC && DELTA) bulk_copy_g2s(st + L::kt, a.kt + vec, L::kVecs * L::kTile, bar);
        }
    };
    constexpr int kGroups = L::kRaw ? 2 : 3;
    if (loader)
        for (int g = 0; g < kGroups; ++g) load_group(g, 0);
    auto load_do = [&](int n) {
        if constexpr (!F32IO) {
            const int c = nchunks - 1 - n;
            if (c >= 0) tc_load_rows(do_s, dsrc + (size_t)c * kChunk * v_stride, v_stride, min(kChunk, len - c * kChunk), tid);
        }
    };
    auto load_qk = [&](int n) {
        if constexpr (L::kRaw) {
            const int c = nchunks - 1 - n;
            if (c < 0) return;
            const uint32_t st = sm + (n % NST) * L::stage;
            const size_t at = ((size_t)(tok0 + c * kChunk) * a.Hq + hq) * DK, stride = (size_t)a.Hq * DK;
            const int valid = min(kChunk, len - c * kChunk);
            tc_load_operand<DK, kChunk * 128>(st + L::kh, a.k, at, stride, valid, tid);
            tc_load_operand<DK, kChunk * 128>(st + L::q, a.q, at, stride, valid, tid);
        }
    };
    load_do(0), load_qk(0);
    cp_async_commit();

    float s[HC];
#pragma unroll
    for (int i = 0; i < HC; ++i) s[i] = a.dS_final ? a.dS_final[s_off + (size_t)(f * HC + i) * DV + v] : 0.f;
    uint32_t mma_phase = 0;
    auto products_done = [&]() {
        ok = bounded_wait(mma_bar, mma_phase, tc.abort_flag) && ok;
        mma_phase ^= 1;
        tc_fence_after();
    };
    auto handed_over = [&]() {
        tmem_wait_st();
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    };
    auto issuing = [&]() { return warp == 0 && __all_sync(0xffffffffu, ok) && elect_one(); };
    auto factors = [&](const float *src, float (&d)[HT]) {
#pragma unroll
        for (int i = 0; i < HT; i += 4) {
            const float4 x = *reinterpret_cast<const float4 *>(src + HT * f + i);
            d[i] = x.x, d[i + 1] = x.y, d[i + 2] = x.z, d[i + 3] = x.w;
        }
    };
    auto store_out = [&](int c) {
        if constexpr (!F32IO) {
            if (storer) tc_store_row(odst + (size_t)c * kChunk * v_stride, v_stride, min(kChunk, len - c * kChunk), out_s, warp * 4 + lane);
        }
    };

    for (int n = 0; n < nchunks; ++n) {
        const int c = nchunks - 1 - n;
        const size_t unit = (size_t)(chunk0 + c) * a.H + h;
        const int valid = min(kChunk, len - c * kChunk);
        const uint32_t st = sm + (n % NST) * L::stage, parity = (uint32_t)(n / NST) & 1u;
        const float *decay = reinterpret_cast<const float *>(smem_tc + L::decay + (n & 1) * L::kDecay);
        tmem_st_planes<kPlanes>(row + PL + f * HC / 2, DK / 2, s);
        if (!F32IO) cp_async_wait_all();  // this chunk's dO, q, k
        if (L::kRaw) fence_async_proxy();
        handed_over();
        // (behind a barrier of this chunk every wait of the last one is over: see scan_forward_tc_kernel)
        if (loader && NST == 2)
            for (int g = 0; g < kGroups; ++g) load_group(g, n + 1);
        if (loader && NST == 1 && n > 0)
            for (int g = VEC ? 1 : 0; g < kGroups; ++g) load_group(g, n);
        ok = bounded_wait(full(0, n), parity, tc.abort_flag) && ok;
        if (issuing()) {
            tc_product<kPlanes, 0, L::kVecs, 0, kPlanes, false, DK / 16, kChunk, DK / 2, L::kTile>(tc.tmem + ACC0, tc.tmem + PL, st + L::kh);
            tc_commit(mma_bar);
        }
        // while it runs: the gradient for the per-chunk kernel; dO of this thread's tokens
        if constexpr (F32IO) {
            float4 *dst = reinterpret_cast<float4 *>(a.dS + unit * tile + (size_t)v * DK + f * HC);
#pragma unroll
            for (int i = 0; i < HC / 4; ++i) dst[i] = make_float4(s[4 * i], s[4 * i + 1], s[4 * i + 2], s[4 * i + 3]);
        } else {
            keep_state_planes<DK>(a.dS + unit * tile, s, v, f * HC);
        }
        float x[HT];
#pragma unroll
        for (int i = 0; i < HT; ++i) {
            const int t = HT * f + i;
            if constexpr (F32IO) {
                x[i] = dsrc[(size_t)(c * kChunk + min(t, valid - 1)) * v_stride + v];
                if (t >= valid) x[i] = 0.f;
            } else {
                x[i] = __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(smem_tc + L::rows + t * 256 + v * 2));
            }
        }
        products_done();
        // dO planes for A^T dO (dS's planes are done with)
        tmem_st_planes<OP1>(row + PLO + HT / 2 * f, 32, x);
        handed_over();
        if (warp == 0) ok = bounded_wait(full(1, n), parity, tc.abort_flag) && ok;
        if (issuing()) {
            tc_product_upper<OP1, kPlanes, kPlanes, 32>(tc.tmem + ACC1, tc.tmem + PLO, st + L::A);
            tc_commit(mma_bar);
        }
        load_do(n + 1), load_qk(n + 1);
        cp_async_commit();
        if (n > 0) store_out(c + 1);
        if (loader && NST == 1 && VEC) load_group(0, n + 1);
        float u[HT], d[HT], y[HT];
        tmem_ld16(row + ACC0 + HT * f, u);
        if (!VEC) factors(decay + kChunk, d);
        products_done();
        tmem_ld16(row + ACC1 + HT * f, y);
#pragma unroll
        for (int i = 0; i < HT; ++i) u[i] = VEC ? u[i] + y[i] : fmaf(d[i], u[i], y[i]);
        if (!F32IO && storer) tc_stores_read();  // the last chunk's dv has left its tile
        if (DELTA) {
            tmem_st_planes<kPlanes>(row + PL + HT / 2 * f, 32, u);
            handed_over();
            if (issuing()) {
                tc_product_upper<kPlanes, kPlanes, kPlanes, 32>(tc.tmem + ACC2, tc.tmem + PL, st + L::T);
                tc_commit(mma_bar);
            }
            products_done();
            tmem_ld16(row + ACC2 + HT * f, u);
        }
        // planes for the update
        if (!VEC) {
            factors(decay, d);
#pragma unroll
            for (int i = 0; i < HT; ++i) x[i] *= d[i] * a.scale;
        }
        tmem_st_planes<OP2>(row + PLO + HT / 2 * f, 32, x);
        if (DELTA) {
#pragma unroll
            for (int i = 0; i < HT; ++i) x[i] = VEC ? -u[i] : -d[i] * u[i];
            tmem_st_planes<kPlanes>(row + PL + HT / 2 * f, 32, x);
        }
        handed_over();
        if (kGroups == 3 && warp == 0) ok = bounded_wait(full(2, n), parity, tc.abort_flag) && ok;
        if (issuing()) {
            tc_product<OP2, 0, L::kVecs, 0, kPlanes, true, 4, DK, 32, L::kTile>(tc.tmem + UPD, tc.tmem + PLO, st + L::q);
            if (DELTA) tc_product<kPlanes, 0, L::kVecs, 0, kPlanes, true, 4, DK, 32, L::kTile>(tc.tmem + UPD, tc.tmem + PL, st + (VEC ? L::kt : L::kh), false);
            tc_commit(mma_bar);
        }
        // while it runs: dV, for the per-chunk kernel and as the gradient of v
        if constexpr (DELTA && F32IO) {
            float *dst = a.dV + unit * kChunk * DV + (size_t)(HT * f) * DV + v;
#pragma unroll
            for (int i = 0; i < HT; ++i) dst[(size_t)i * DV] = u[i];
        } else if constexpr (DELTA) {
            keep_value_planes<false>(a.dV + unit * kChunk * DV, u, HT * f, v);
        }
#pragma unroll
        for (int i = 0; i < HT; ++i) {
            const int t = HT * f + i;
            if constexpr (F32IO) {
                if (t < valid) odst[(size_t)(c * kChunk + t) * v_stride + v] = u[i];
            } else {
                *reinterpret_cast<__nv_bfloat16 *>(smem_tc + L::rows + kChunk * 256 + t * 256 + v * 2) = __float2bfloat16_rn(u[i]);
            }
        }
        if (!F32IO) fence_async_proxy();
        products_done();
#pragma unroll
        for (int i = 0; i < HC; i += 16) {
            float z[16];
            tmem_ld16(row + UPD + f * HC + i, z);
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float4 e = VEC ? *reinterpret_cast<const float4 *>(decay + f * HC + i + j) : make_float4(decay[kChunk - 1], decay[kChunk - 1], decay[kChunk - 1], decay[kChunk - 1]);
                s[i + j] = fmaf(e.x, s[i + j], z[j]), s[i + j + 1] = fmaf(e.y, s[i + j + 1], z[j + 1]);
                s[i + j + 2] = fmaf(e.z, s[i + j + 2], z[j + 2]), s[i + j + 3] = fmaf(e.w, s[i + j + 3], z[j + 3]);
            }
        }
    }
    cp_async_wait_all();
    if (nchunks > 0) {
        __syncthreads();
        store_out(0);
    }
    if (*tc.abort_flag) {  // results are invalid; copies in flight end before the CTA's memory is given back
        if (tid == 0) {
            if (a.status) atomicOr(a.status, DELTALOG_STATUS_TIMEOUT);
            for (int i = 0; i < 3 * NST; ++i) {
                bounded_wait(tc.bars + 8u * i, 0u, tc.abort_flag + 1);
                bounded_wait(tc.bars + 8u * i, 1u, tc.abort_flag + 1);
            }
        }
    } else if (a.dS_init) {
#pragma unroll
        for (int i = 0; i < HC; ++i) a.dS_init[s_off + (size_t)(f * HC + i) * DV + v] = s[i];
    }
    if (!F32IO && storer) tc_stores_done();
    tc_teardown(tc, tid);
}

}  // namespace deltalog
