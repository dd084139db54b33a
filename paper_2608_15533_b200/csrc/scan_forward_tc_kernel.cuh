// The chain over a sequence's chunks for d_v = 128, on the 5th-generation tensor cores.  One CTA per (sequence, head).
//
// As in scan_forward_kernel everything is transposed: row v of every matrix is lane v of tensor memory, and the products'
// A operands (S^T, R^T, U^T) are written there as bf16 planes by the threads that hold the fp32 values.  Thread (lane v,
// quarter f) keeps S[c][v] for a quarter of the channels in registers for the whole sequence, and handles a quarter of the
// tokens of the [64 x 128] matrices.  Per chunk:
//     S planes -> tensor memory;  (k S)^T, (q S)^T;  R = V - ..;  R planes;  U^T = R^T T^T;  U planes;
//     A U and the state's update;  S <- e^(G_end) S + update, output.
// B operands are images that prep wrote, fetched by bulk copies a step ahead; k and q lie interleaved so that one product
// of 128 columns serves both.  The tensor cores need a quarter of mma.sync's time for the products; the rest of a chunk's
// time is the threads' plane splits in between.  Of some 8k cycles a chunk (GDN, bf16) the products take half, the splits of S, R
// and U and the update the other half, one behind the other; an SM's registers hold one such chain.
// Against the mma.sync chain, bf16, 32 heads of 128: 48 ragged prompts of 36k tokens 1328 -> 659 us, one of 16k tokens 1671 -> 1091
// us, 13k tokens of KDA 747 -> 323 us.  d_v = 64 stays there: half of an MMA's rows would be empty, though by the cycle counts
// (32 for 128 x 64 x 16 half empty, 64 on mma.sync) its products would still be faster here; no such form has been built.
// Now: 606 us of the first; the second in three segments, 349 + 17 + 352 us; 288 us of the third.  With kept states, GDN: 186 us for
// four rows of 2048 tokens, 789 us for 36.7k tokens of 19 rows (3.9 TB/s of DRAM traffic, most of it what is kept).
#pragma once

#include "scan_tc_common.cuh"

namespace deltalog {

template <bool VEC, int P, int DK, bool DELTA, typename IO>
struct ForwardTcSmem {
    static constexpr bool kF32 = sizeof(IO) == 4;
    static constexpr int kTile = kChunk * DK * 2, kMat = kChunk * kChunk * 2, kHalf = kChunk * 128;
    static constexpr int kOut = kF32 ? kPlanes : 2;
    static constexpr int kQ = VEC ? kOut : P, kK = VEC ? kPlanes : P;
    static constexpr int kDecay = VEC ? DK * 4 : 2 * kChunk * 4;
    static constexpr int kStages = !VEC && P == 1 ? 2 : 1;  // what fits
    static constexpr bool kRaw = !VEC && P == 1;            // q and k as they are, copied by all threads
    // delta rule: planes of k (per channel: k e^G) and q, 64 channels of the one and then of the other, then k's further
    // planes; otherwise q, and for scalar decay k
    static constexpr int kPair = DELTA ? 2 * kTile : kTile, kPairHalf = DELTA ? 2 * kHalf : kHalf;
    static constexpr int kq = 0;
    static constexpr int k_more = kq + kQ * kPair;
    static constexpr int kh = k_more + (DELTA ? (kK - kQ) * kTile : 0);  // k of the update, where it is not among them
    static constexpr bool kOwnKh = VEC || !DELTA;
    static constexpr int A = kh + (kOwnKh ? kK * kTile : 0);
    static constexpr int T = A + kOut * kMat;
    static constexpr int stage = T + (DELTA ? kPlanes * kMat : 0);
    static constexpr int rows = kStages * stage;                          // bf16 io: v, out
    static constexpr int decay = rows + (kF32 ? 0 : 2 * kChunk * 256);
    static constexpr int control = decay + 2 * kDecay;
    static constexpr size_t total = control + kTcControlBytes;
    static constexpr size_t bytes = total > kTcMinSmem ? total : kTcMinSmem;
};

// KEEP: what the backward pass reads is kept.  (Two kernels: serving's, without that code, is a few percent faster.)
template <bool VEC, int P, int DK, bool DELTA, typename IO, bool KEEP>
__global__ void __launch_bounds__(kTcThreads, 1) scan_forward_tc_kernel(const ScanArgs a) {
    using L = ForwardTcSmem<VEC, P, DK, DELTA, IO>;
    constexpr int DV = 128, HC = DK / 4, HT = kChunk / 4;  // channels and tokens per thread
    constexpr int NST = L::kStages;
    constexpr bool F32IO = L::kF32;
    constexpr int UP = DELTA || F32IO ? kPlanes : 1;
    constexpr int UO = UP < L::kOut ? UP : L::kOut;   // planes of U for the output
    constexpr int US = VEC ? UP : kPlanes;            // and for the state (scalar decay: times e^(G_end - G))
    // Scalar decay: nobody waits for q S before the chunk's end, so it runs behind k S while R is formed, and R's planes keep
    // out of S's (one 16k-token row 904 -> 874 us).  Per channel it is more products apart than together: 866 -> 875 us.
    // With KEEP the threads are busy storing meanwhile and nothing is gained.  The same for A U, which the state need not wait
    // for (ragged prompts 1055 -> 1026 us; GDN training 4615 -> 4670, KDA training 919 -> 916).
    constexpr bool kApart = DELTA && !VEC && !KEEP, kOutApart = VEC || !KEEP;
    // tensor memory: accumulators of (k S)^T and then U^T, of (q S)^T, of A U, of the update; planes of S, later of U for the
    // update and of U for the output; planes of R
    constexpr uint32_t ACC0 = 0, ACC1 = 64, ACC2 = 128, UPD = 192, PL = 320, PLO = 416, PR = kApart ? UPD : PL;
    extern __shared__ __align__(1024) unsigned char smem_tc[];
    const uint32_t sm = smem_addr(smem_tc);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int v = 32 * (warp & 3) + lane, f = warp >> 2;
    scan_kernel_begin(a.S_out != nullptr);
    ScanSegment seg;
    if (!scan_segment(a, blockIdx.x, seg)) return;
    const int seq = seg.seq, h = seg.h, hq = h / (a.H / a.Hq);
    int slot;
    if (!scan_slot(a, seq, tid, slot)) return;
    const int nchunks = seg.end - seg.first;
    if (nchunks == 0 && a.slots) return;
    const int tok0 = a.starts[seq] + seg.first * kChunk, len = min(a.starts[seq + 1] - tok0, nchunks * kChunk);
    const int chunk0 = a.chunk_starts[seq] + seg.first;
    // (a.keep is always set with KEEP; asked as a variable the compiler orders a chunk's stores better: 4530 us against 4615)
    const bool keep = KEEP && a.keep && seg.emit, emit = a.out && seg.emit;
    const size_t tile = (size_t)DK * DV, s_off = ((size_t)slot * a.H + h) * tile;
    const size_t pieces = ((size_t)seq * a.H + h) * scan_pieces(a.split);
    const size_t v_stride = (size_t)a.H * DV;
    const TcBlock tc = tc_setup(smem_tc + L::control, 3 * NST + 2, tid);
    const uint32_t row = tc.tmem + ((uint32_t)(32 * (warp & 3)) << 16);
    const uint32_t mma_bar = tc.bars + 8u * (3 * NST), out_bar = mma_bar + 8;
    const uint32_t v_s = sm + L::rows, out_s = v_s + kChunk * 256;
    const IO *vsrc = static_cast<const IO *>(a.v) + (size_t)tok0 * v_stride + (size_t)h * DV;
    IO *odst = static_cast<IO *>(a.out) + (size_t)tok0 * v_stride + (size_t)h * DV;
    bool ok = true;

    // operand groups: 0 = what the products with S read and the decay factors, 1 = A and T, 2 = k for the update (where it is
    // a tile of its own)
    auto full = [&](int group, int c) { return tc.bars + 8u * (3 * (c % NST) + group); };
    auto load_group = [&](int group, int c) {  // one thread
        if (c >= nchunks || *tc.abort_flag) return;
        const size_t unit = (size_t)(chunk0 + c) * a.H + h, qunit = (size_t)(chunk0 + c) * a.Hq + hq;
        const uint32_t st = sm + (c % NST) * L::stage, bar = full(group, c);
        const size_t vec = unit * kPlanes * kChunk * DK, qvec = qunit * P * kChunk * DK, mat = unit * kPlanes * kChunk * kChunk;
        const __nv_bfloat16 *q = VEC ? a.qt + vec : a.qi + qvec, *k = VEC ? a.kt + vec : a.ki + qvec, *ku = VEC ? a.kh + vec : a.ki + qvec;
        if (group == 0) {
            mbar_arrive_expect_tx(bar, (L::kRaw ? 0 : L::kh - L::kq) + L::kDecay);
            if (L::kRaw) {
            } else if (DELTA) {
                for (int i = 0; i < L::kQ * (DK / 64); ++i) {  // halves of k and q by turns
                    bulk_copy_g2s(st + L::kq + 2 * i * L::kHalf, k + (size_t)i * L::kHalf / 2, L::kHalf, bar);
                    bulk_copy_g2s(st + L::kq + (2 * i + 1) * L::kHalf, q + (size_t)i * L::kHalf / 2, L::kHalf, bar);
                }
                if (L::kK > L::kQ) bulk_copy_g2s(st + L::k_more, k + (size_t)L::kQ * L::kTile / 2, (L::kK - L::kQ) * L::kTile, bar);
            } else {
                bulk_copy_g2s(st + L::kq, q, L::kQ * L::kTile, bar);
            }
            bulk_copy_g2s(sm + L::decay + (c & 1) * L::kDecay, a.decay + unit * (L::kDecay / 4), L::kDecay, bar);
        } else if (group == 1) {
            mbar_arrive_expect_tx(bar, (L::kOut + (DELTA ? kPlanes : 0)) * L::kMat);
            bulk_copy_g2s(st + L::A, a.A + mat, L::kOut * L::kMat, bar);
            if (DELTA) bulk_copy_g2s(st + L::T, a.T + mat, kPlanes * L::kMat, bar);
        } else {
            mbar_arrive_expect_tx(bar, L::kK * L::kTile);
            bulk_copy_g2s(st + L::kh, ku, L::kK * L::kTile, bar);
        }
    };
    // who does what besides: warp 0 issues the products, one thread of warp 4 the loads, four lanes of each warp the output rows
    const bool loader = tid == 128, storer = lane < 4;
    constexpr int kGroups = L::kOwnKh && !L::kRaw ? 3 : 2;
    if (loader)
        for (int g = 0; g < kGroups; ++g) load_group(g, 0);
    auto load_v = [&](int c) {
        if constexpr (!F32IO) {
            if (c < nchunks) tc_load_rows(v_s, vsrc + (size_t)c * kChunk * v_stride, v_stride, min(kChunk, len - c * kChunk), tid);
        }
    };
    auto load_qk = [&](int c) {
        if constexpr (L::kRaw) {
            if (c >= nchunks) return;
            const uint32_t st = sm + (c % NST) * L::stage;
            const size_t at = ((size_t)(tok0 + c * kChunk) * a.Hq + hq) * DK, stride = (size_t)a.Hq * DK;
            const int valid = min(kChunk, len - c * kChunk);
            if (DELTA) {
                tc_load_operand<DK, 2 * L::kHalf>(st + L::kq, a.k, at, stride, valid, tid);
                tc_load_operand<DK, 2 * L::kHalf>(st + L::kq + L::kHalf, a.q, at, stride, valid, tid);
            } else {
                tc_load_operand<DK, L::kHalf>(st + L::kq, a.q, at, stride, valid, tid);
                tc_load_operand<DK, L::kHalf>(st + L::kh, a.k, at, stride, valid, tid);
            }
        }
    };
    load_v(0), load_qk(0);
    cp_async_commit();

    float s[HC];
    const bool zero = seg.from == -2 || (seg.from == -1 && (!a.S_in || (a.fresh && a.fresh[seq]))), as_bf16 = seg.from == -1 && a.in_bf16;
    const void *S_in = seg.from >= 0 ? a.pieces + (pieces + seg.from) * tile : a.S_in;
    const size_t in_off = seg.from >= 0 ? 0 : s_off;
#pragma unroll
    for (int i = 0; i < HC; ++i) {
        const size_t at = in_off + (size_t)(f * HC + i) * DV + v;
        s[i] = zero ? (seg.map && f * HC + i == v ? 1.f : 0.f) : as_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(S_in)[at]) : static_cast<const float *>(S_in)[at];
    }
    uint32_t mma_phase = 0;
    // the products that one thread has issued are complete
    auto products_done = [&]() {
        ok = bounded_wait(mma_bar, mma_phase, tc.abort_flag) && ok;
        mma_phase ^= 1;
        tc_fence_after();
    };
    // what the threads wrote to tensor memory is visible to the issuing thread
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

    // a chunk's output: kept in registers until the next chunk's first products run, then to its tile (fp32 io: to its place)
    // and, behind a barrier, from there
    float o[HT];
    auto write_out = [&](int c) {
        if (!emit) return;
#pragma unroll
        for (int i = 0; i < HT; ++i) {
            const int t = HT * f + i;
            if constexpr (F32IO) {
                if (c * kChunk + t < len) odst[(size_t)(c * kChunk + t) * v_stride + v] = o[i];
            } else {
                *reinterpret_cast<__nv_bfloat16 *>(smem_tc + L::rows + kChunk * 256 + t * 256 + v * 2) = __float2bfloat16_rn(o[i]);
            }
        }
        if (!F32IO) fence_async_proxy();
    };
    auto store_out = [&](int c) {
        if constexpr (!F32IO) {
            if (emit && storer) tc_store_row(odst + (size_t)c * kChunk * v_stride, v_stride, min(kChunk, len - c * kChunk), out_s, warp * 4 + lane);
        }
    };

    // behind the second barrier of chunk c: v's tile is read, the last chunk's output tile written
    auto between = [&](int c) {
        load_v(c + 1), load_qk(c + 1);
        cp_async_commit();
        if (c > 0) store_out(c - 1);
        if (NST == 1 && VEC && loader) load_group(0, c + 1);
    };

    for (int c = 0; c < nchunks; ++c) {
        const size_t unit = (size_t)(chunk0 + c) * a.H + h;
        const int valid = min(kChunk, len - c * kChunk);
        const uint32_t st = sm + (c % NST) * L::stage, parity = (uint32_t)(c / NST) & 1u;
        const float *decay = reinterpret_cast<const float *>(smem_tc + L::decay + (c & 1) * L::kDecay);
        tmem_st_planes<kPlanes>(row + PL + f * HC / 2, DK / 2, s);
        if (!F32IO) cp_async_wait_all();  // this chunk's v, q, k
        if (L::kRaw) fence_async_proxy();
        handed_over();
        // Behind a barrier of this chunk every wait of the last one is over, as is every read of its decay factors: its
        // barriers may go on to their next phase.  (A thread that comes late to a wait would else find the phase behind it gone
        // by as well and take it for the one before.)
        if (loader && NST == 2)
            for (int g = 0; g < kGroups; ++g) load_group(g, c + 1);
        if (loader && NST == 1 && c > 0)
            for (int g = VEC ? 1 : 0; g < kGroups; ++g) load_group(g, c);
        ok = bounded_wait(full(0, c), parity, tc.abort_flag) && ok;
        if (issuing()) {
            const uint32_t pl = tc.tmem + PL, b = st + L::kq;
            if (DELTA) {
                // (k S takes the same products in the same order with and without q S beside it: the same bits)
                constexpr bool kMore = L::kK > L::kQ, kAlone = kMore || L::kOut < kPlanes;
                tc_product<kPlanes, L::kQ, L::kK, 0, kPlanes, false, DK / 16, kChunk, DK / 2, L::kTile>(tc.tmem + ACC0, pl, st + L::k_more);
                tc_product<kPlanes, 0, L::kQ, L::kOut, kPlanes, false, DK / 16, kChunk, DK / 2, L::kPair, L::kPairHalf>(tc.tmem + ACC0, pl, b, !kMore);
                if (kApart || !emit)
                    tc_product<kPlanes, 0, L::kQ, 0, L::kOut, false, DK / 16, kChunk, DK / 2, L::kPair, L::kPairHalf>(tc.tmem + ACC0, pl, b, !kAlone);
                else
                    tc_product<kPlanes, 0, L::kQ, 0, L::kOut, false, DK / 16, 2 * kChunk, DK / 2, L::kPair, L::kPairHalf, kAlone>(tc.tmem + ACC0, pl, b);
            } else if (emit) {
                tc_product<kPlanes, 0, L::kQ, 0, L::kOut, false, DK / 16, kChunk, DK / 2, L::kTile>(tc.tmem + ACC1, pl, b);
            }
            tc_commit(mma_bar);
            if (kApart && emit) tc_product<kPlanes, 0, L::kQ, 0, L::kOut, false, DK / 16, kChunk, DK / 2, L::kPair, L::kPairHalf>(tc.tmem + ACC1, pl, b + L::kHalf);
        }
        // while they run: the state for the backward pass, the last chunk's output, v of this thread's tokens
        if (keep) {
            if constexpr (F32IO) {
                float4 *dst = reinterpret_cast<float4 *>(a.S + unit * tile + (size_t)v * DK + f * HC);
#pragma unroll
                for (int i = 0; i < HC / 4; ++i) dst[i] = make_float4(s[4 * i], s[4 * i + 1], s[4 * i + 2], s[4 * i + 3]);
            } else {
                keep_state_planes<DK>(a.S + unit * tile, s, v, f * HC);
            }
        }
        if (c > 0) write_out(c - 1);
        float x[HT];
#pragma unroll
        for (int i = 0; i < HT; ++i) {
            const int t = HT * f + i;
            if constexpr (F32IO) {
                x[i] = vsrc[(size_t)(c * kChunk + min(t, valid - 1)) * v_stride + v];
                if (t >= valid || seg.map) x[i] = 0.f;
            } else {
                x[i] = __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(smem_tc + L::rows + t * 256 + v * 2));
                if (seg.map) x[i] = 0.f;
            }
        }
        products_done();
        float u[HT], d[HT];
        if (DELTA) {
            // R = V - (k e^G S), then U = T R
            tmem_ld16(row + ACC0 + HT * f, u);
            if (!VEC) factors(decay, d);
#pragma unroll
            for (int i = 0; i < HT; ++i) u[i] = VEC ? x[i] - u[i] : fmaf(-d[i], u[i], x[i]);
            tmem_st_planes<kPlanes>(row + PR + HT / 2 * f, 32, u);
            handed_over();
            if (warp == 0) ok = bounded_wait(full(1, c), parity, tc.abort_flag) && ok;
            if (issuing()) {
                tc_product_lower<kPlanes, kPlanes, kPlanes, 32>(tc.tmem + ACC0, tc.tmem + PR, st + L::T);
                tc_commit(mma_bar);
            }
            between(c);
            products_done();
            tmem_ld16(row + ACC0 + HT * f, u);
            if (keep) {
                if constexpr (F32IO) {
                    float *dst = a.U + unit * kChunk * DV + (size_t)(HT * f) * DV + v;
#pragma unroll
                    for (int i = 0; i < HT; ++i) dst[(size_t)i * DV] = u[i];
                } else {
                    keep_value_planes<true>(a.U + unit * kChunk * DV, u, HT * f, v);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < HT; ++i) u[i] = x[i];
        }
        tmem_st_planes<UO>(row + PLO + HT / 2 * f, 32, u);
        if (!VEC) {
            factors(decay + kChunk, d);
#pragma unroll
            for (int i = 0; i < HT; ++i) u[i] *= d[i];
        }
        tmem_st_planes<US>(row + PL + HT / 2 * f, 32, u);
        handed_over();
        if (!DELTA && warp == 0) ok = bounded_wait(full(1, c), parity, tc.abort_flag) && ok;
        if (kGroups == 3 && warp == 0) ok = bounded_wait(full(2, c), parity, tc.abort_flag) && ok;
        if (issuing()) {
            if (L::kOwnKh) tc_product<US, 0, L::kK, 0, kPlanes, true, 4, DK, 32, L::kTile>(tc.tmem + UPD, tc.tmem + PL, st + L::kh);
            else tc_product<US, 0, L::kK, 0, kPlanes, true, 4, DK, 32, L::kPair, L::kPairHalf>(tc.tmem + UPD, tc.tmem + PL, st + L::kq);
            if (kOutApart) tc_commit(mma_bar);
            if (emit) tc_product_lower<UO, L::kOut, L::kOut, 32>(tc.tmem + ACC2, tc.tmem + PLO, st + L::A);
            if (!kOutApart) tc_commit(mma_bar);
            else if (emit) tc_commit(out_bar);
        }
        if (!DELTA) between(c);
        if (!F32IO && storer) tc_stores_read();  // the last chunk's output has left its tile
        products_done();
#pragma unroll
        for (int i = 0; i < HC; i += 16) {
            float y[16];
            tmem_ld16(row + UPD + f * HC + i, y);
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const float4 e = VEC ? *reinterpret_cast<const float4 *>(decay + f * HC + i + j) : make_float4(decay[kChunk - 1], decay[kChunk - 1], decay[kChunk - 1], decay[kChunk - 1]);
                s[i + j] = fmaf(e.x, s[i + j], y[j]), s[i + j + 1] = fmaf(e.y, s[i + j + 1], y[j + 1]);
                s[i + j + 2] = fmaf(e.z, s[i + j + 2], y[j + 2]), s[i + j + 3] = fmaf(e.w, s[i + j + 3], y[j + 3]);
            }
        }
        if (emit) {
            if (kOutApart) {
                ok = bounded_wait(out_bar, (uint32_t)c & 1u, tc.abort_flag) && ok;
                tc_fence_after();
            }
            float z[HT];
            tmem_ld16(row + ACC1 + HT * f, o);
            tmem_ld16(row + ACC2 + HT * f, z);
            if (!VEC) factors(decay, d);
#pragma unroll
            for (int i = 0; i < HT; ++i) o[i] = VEC ? o[i] + z[i] : fmaf(d[i] * a.scale, o[i], z[i]);
        }
    }
    cp_async_wait_all();
    if (nchunks > 0) {
        __syncthreads();  // (the output before has left the tile: its storers say so)
        write_out(nchunks - 1);
        __syncthreads();
        store_out(nchunks - 1);
    }
    if (*tc.abort_flag) {  // results are invalid; copies in flight end before the CTA's memory is given back
        if (tid == 0) {
            if (a.status) atomicOr(a.status, DELTALOG_STATUS_TIMEOUT);
            for (int i = 0; i < 3 * NST; ++i) {
                bounded_wait(tc.bars + 8u * i, 0u, tc.abort_flag + 1);
                bounded_wait(tc.bars + 8u * i, 1u, tc.abort_flag + 1);
            }
        }
    } else {
        if (seg.to >= 0 || (seg.to == -1 && a.S_out)) {
            float *piece = a.pieces + (pieces + max(seg.to, 0)) * tile;
#pragma unroll
            for (int i = 0; i < HC; ++i) {
                const size_t at = (size_t)(f * HC + i) * DV + v;
                if (seg.to >= 0) piece[at] = s[i];
                else if (a.out_bf16) static_cast<__nv_bfloat16 *>(a.S_out)[s_off + at] = __float2bfloat16_rn(s[i]);
                else static_cast<float *>(a.S_out)[s_off + at] = s[i];
            }
        }
        if (a.log_len && seg.to == -1 && tid == 0) a.log_len[(size_t)slot * a.H + h] = 0;
    }
    if (!F32IO && storer) tc_stores_done();
    tc_teardown(tc, tid);
}

// The states in front of a split row's segments: X_1 is the first segment's end, X_(s+1) = M_s X_s + E_s in E_s' place.
// Sixteen columns per CTA, one row of M per thread; the next M is on its way while one is multiplied.  In fp32 throughout.
// Bound by latency: a join is d_k dependent steps of loads from shared memory behind a copy of M, 5 us or so for each, one behind the
// other (16k tokens of GDN: 1 head, 30 joins 148 us of 242; 8 heads, 8 joins 43 us of 313; 32 heads, one join 16.4 us of 896, where
// 256 CTAs of 148 KB also take two waves).
constexpr int kJoinCols = 16;
template <int DK>
struct JoinSmem {
    static constexpr int stride = DK + 4;
    static constexpr size_t bytes = (size_t)(2 * DK * stride + 2 * DK * kJoinCols) * 4;
};
template <int DK>
__global__ void __launch_bounds__(DK) scan_join_kernel(const ScanArgs a) {
    constexpr int DV = 128, kStride = JoinSmem<DK>::stride;
    extern __shared__ __align__(16) unsigned char smem_join[];
    float *M = reinterpret_cast<float *>(smem_join), *X = M + 2 * DK * kStride;  // twice each
    const int tid = threadIdx.x, v0 = blockIdx.y * kJoinCols;
    scan_kernel_begin();
    const int seq = blockIdx.x / a.H;
    const int segments = scan_segments(a.chunk_starts[seq + 1] - a.chunk_starts[seq], a.split);
    if (segments < 3) return;
    if (a.slots) {
        const int slot = a.slots[seq];
        if (slot < 0 || slot >= a.num_slots) return;
    }
    float *pieces = a.pieces + (size_t)blockIdx.x * scan_pieces(a.split) * DK * DV;
    auto fetch = [&](int s) {  // M_s; its rows hold d_k of their d_v columns
        if (s <= segments - 2) {
            const float *src = pieces + (size_t)(2 * s) * DK * DV;
            const uint32_t dst = smem_addr(M + (s & 1) * DK * kStride);
            for (int i = tid; i < DK * DK / 4; i += DK) cp_async16_zfill(dst + ((i / (DK / 4)) * kStride + i % (DK / 4) * 4) * 4, src + (size_t)(i / (DK / 4)) * DV + i % (DK / 4) * 4, true);
        }
        cp_async_commit();
    };
    fetch(1);
#pragma unroll
    for (int j = 0; j < kJoinCols; j += 4)
        *reinterpret_cast<float4 *>(X + DK * kJoinCols + tid * kJoinCols + j) = *reinterpret_cast<const float4 *>(pieces + (size_t)tid * DV + v0 + j);
    for (int s = 1; s <= segments - 2; ++s) {
        float *E = pieces + (size_t)(2 * s - 1) * DK * DV + (size_t)tid * DV + v0;
        float x[kJoinCols];
#pragma unroll
        for (int j = 0; j < kJoinCols; j += 4) {
            const float4 e = *reinterpret_cast<const float4 *>(E + j);
            x[j] = e.x, x[j + 1] = e.y, x[j + 2] = e.z, x[j + 3] = e.w;
        }
        cp_async_wait_all();
        __syncthreads();  // M_s and X_s are there, the places of the ones before are free
        fetch(s + 1);
        const float *m = M + (s & 1) * DK * kStride + tid * kStride, *in = X + (s & 1) * DK * kJoinCols;
#pragma unroll 4
        for (int c = 0; c < DK; ++c) {
            const float w = m[c];
#pragma unroll
            for (int j = 0; j < kJoinCols; j += 4) {
                const float4 y = *reinterpret_cast<const float4 *>(in + c * kJoinCols + j);
                x[j] = fmaf(w, y.x, x[j]), x[j + 1] = fmaf(w, y.y, x[j + 1]);
                x[j + 2] = fmaf(w, y.z, x[j + 2]), x[j + 3] = fmaf(w, y.w, x[j + 3]);
            }
        }
        float *next = X + ((s + 1) & 1) * DK * kJoinCols + tid * kJoinCols;
#pragma unroll
        for (int j = 0; j < kJoinCols; j += 4) {
            const float4 y = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
            *reinterpret_cast<float4 *>(E + j) = y;
            *reinterpret_cast<float4 *>(next + j) = y;
        }
    }
    cp_async_wait_all();
}

}  // namespace deltalog
