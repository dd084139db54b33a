// The chain over a sequence's chunks from the last to the first: dS, and with it dU and dV.
//
//     dU = A^T dO + (k e^(G_end - G)) dS        dV = T^T dU   (or dV = dU)
//     dS <- e^(G_end) dS + (scale q e^G)^T dO - (k e^G)^T dV
//
// The layout is the forward chain's: transposed, 16 columns of d_v per warp, dS^T [16 x d_k] in its accumulators; for d_v = 64,
// bound as it is.  RWKV6, bf16, 64 heads of 64, four rows of 1024 tokens: 96 us.
#pragma once

#include "scan_common.cuh"

namespace deltalog {

template <bool VEC, int P, int DK, bool DELTA, typename IO>
struct BackwardSmem {
    static constexpr int kTile = kChunk * DK * 2;
    static constexpr int kMat = kChunk * kChunk * 2;
    static constexpr int kVecs = VEC ? kPlanes : P;  // planes of q and k
    static constexpr int kDecay = VEC ? DK * 4 : 2 * kChunk * 4;
    // Scalar decay: k (first and last product of a chunk; bf16: two places) and q.  Per channel: k e^(G_end - G), k e^G
    // (delta rule), scale q e^G.
    static constexpr bool kTwice = !VEC && P == 1;
    static constexpr int kh = 0;
    static constexpr int kt = (kTwice ? 2 : 1) * kVecs * kTile;
    static constexpr int q = kt + (VEC && DELTA ? kVecs * kTile : 0);
    static constexpr int A = q + kVecs * kTile;
    static constexpr int T = A + kPlanes * kMat;
    static constexpr int decay = T + (DELTA ? kPlanes * kMat : 0);  // twice
    static constexpr int slices = decay + 2 * kDecay;               // bf16 io, per warp: dO, staging
    static constexpr int per_warp = sizeof(IO) == 4 ? 0 : 2 * kChunk * 32;
    static constexpr size_t bytes(int warps) { return slices + (size_t)warps * per_warp; }
};

template <bool VEC, int P, int DK, bool DELTA, typename IO>
__global__ void __launch_bounds__(128, 1) scan_backward_kernel(const ScanArgs a) {
    using L = BackwardSmem<VEC, P, DK, DELTA, IO>;
    constexpr int NT = DK / 8;
    constexpr bool F32IO = sizeof(IO) == 4;
    constexpr int OP1 = F32IO ? kPlanes : 1;             // planes of dO
    constexpr int OP2 = VEC ? OP1 : kPlanes;             // and of dO times a scalar decay
    extern __shared__ __align__(128) unsigned char smem[];
    const uint32_t sm = smem_addr(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nthreads = blockDim.x;
    scan_kernel_begin();
    const int seq = a.order[blockIdx.x / a.H], h = blockIdx.x % a.H, hq = h / (a.H / a.Hq);
    const int v0 = (blockIdx.y * (nthreads >> 5) + warp) * 16;
    const int t = lane & 3;
    const int tok0 = a.starts[seq], len = a.starts[seq + 1] - tok0, nchunks = (len + kChunk - 1) / kChunk;
    const int chunk0 = a.chunk_starts[seq];
    const size_t tile = (size_t)DK * a.dv, s_off = ((size_t)seq * a.H + h) * tile;
    const size_t v_stride = (size_t)a.H * a.dv;
    const uint32_t o_s = sm + L::slices + warp * L::per_warp, stage = o_s + kChunk * 32;

    auto load_raw = [&](uint32_t dst, const void *raw, const __nv_bfloat16 *image, int c) {  // q or k of a chunk
        load_vectors_tile<P, DK>(dst, raw, image, a, tok0 + c * kChunk, chunk0 + c, hq, min(kChunk, len - c * kChunk), tid, nthreads);
    };
    auto load_decayed = [&](uint32_t dst, const __nv_bfloat16 *src, int planes, size_t unit) {
        load_image(dst, src + unit * kPlanes * kChunk * DK, planes * L::kTile, tid, nthreads);
    };
    auto load_first = [&](int c) {  // k for dU, decay factors
        const size_t unit = (size_t)(chunk0 + c) * a.H + h;
        if (VEC) load_decayed(sm + L::kh, a.kh, kPlanes, unit);
        else if (L::kTwice) load_raw(sm + L::kh + (c & 1) * L::kTile, a.k, a.ki, c);
        for (int i = tid; i < L::kDecay / 16; i += nthreads)
            cp_async16(smem + L::decay + (c & 1) * L::kDecay + i * 16, a.decay + unit * (L::kDecay / 4) + i * 4);
    };
    auto load_matrices = [&](int c) {
        const size_t at = ((size_t)(chunk0 + c) * a.H + h) * kPlanes * kChunk * kChunk;
        load_image(sm + L::A, a.A + at, kPlanes * L::kMat, tid, nthreads);
        if (DELTA) load_image(sm + L::T, a.T + at, kPlanes * L::kMat, tid, nthreads);
    };
    auto load_update = [&](int c) {  // q, k for dS, and dO
        const size_t unit = (size_t)(chunk0 + c) * a.H + h;
        if (VEC) {
            load_decayed(sm + L::q, a.qt, kPlanes, unit);
            if (DELTA) load_decayed(sm + L::kt, a.kt, kPlanes, unit);
        } else {
            load_raw(sm + L::q, a.q, a.qi, c);
            if (!L::kTwice) load_raw(sm + L::kh, a.k, a.ki, c);
        }
        if constexpr (!F32IO)
            load_slice(o_s, static_cast<const IO *>(a.dout) + (size_t)(tok0 + c * kChunk) * v_stride + (size_t)h * a.dv + v0, v_stride,
                       min(kChunk, len - c * kChunk), lane);
    };
    if (nchunks > 0) {
        load_first(nchunks - 1), cp_async_commit();
        load_matrices(nchunks - 1), cp_async_commit();
        load_update(nchunks - 1), cp_async_commit();
    }
    float s[NT][4];
    if (a.dS_final) {
        load_state<NT>(s, a.dS_final, false, s_off, a.dv, v0, lane);
    } else {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
    }

    for (int c = nchunks - 1; c >= 0; --c) {
        const size_t unit = (size_t)(chunk0 + c) * a.H + h;
        const int valid = min(kChunk, len - c * kChunk);
        const float *decay = reinterpret_cast<const float *>(smem + L::decay + (c & 1) * L::kDecay);
        const uint32_t k_s = sm + L::kh + (L::kTwice ? (c & 1) * L::kTile : 0);
        const IO *dout = static_cast<const IO *>(a.dout) + (size_t)(tok0 + c * kChunk) * v_stride + (size_t)h * a.dv + v0;
        cp_async_wait<VEC || L::kTwice ? 2 : 0>();
        __syncthreads();
        keep_state<NT>(a.dS + unit * tile, s, v0, lane);
        // dU^T = dS^T (k e^(G_end - G))^T
        float du[8][4] = {};
#pragma unroll
        for (int kk = 0; kk < DK / 16; ++kk) {
            uint32_t f[kPlanes][4];
            acc_to_a<kPlanes>(s[2 * kk], s[2 * kk + 1], f);
#pragma unroll
            for (int nn = 0; nn < 4; nn += 2) {
                // (fp32 io: a step's products apart from the sum, see mma_planes)
                float x[4][4] = {};
                float (&u0)[4] = F32IO ? x[0] : du[2 * nn], (&u1)[4] = F32IO ? x[1] : du[2 * nn + 1];
                float (&u2)[4] = F32IO ? x[2] : du[2 * nn + 2], (&u3)[4] = F32IO ? x[3] : du[2 * nn + 3];
#pragma unroll
                for (int pl = L::kVecs - 1; pl >= 0; --pl) {
                    uint32_t b[4], e[4];
                    load_b(b, k_s + pl * L::kTile, nn * 16, kk * 16, lane);
                    load_b(e, k_s + pl * L::kTile, nn * 16 + 16, kk * 16, lane);
                    mma_planes2<kPlanes, kPlanes>(u0, u1, u2, u3, f, b, e, pl);
                }
                if (F32IO) add_to(du[2 * nn], x[0]), add_to(du[2 * nn + 1], x[1]), add_to(du[2 * nn + 2], x[2]), add_to(du[2 * nn + 3], x[3]);
            }
        }
        if (!VEC) {
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                const float2 d = *reinterpret_cast<const float2 *>(decay + kChunk + n * 8 + 2 * t);
                du[n][0] *= d.x, du[n][1] *= d.y, du[n][2] *= d.x, du[n][3] *= d.y;
            }
        }
        __syncthreads();
        if (c > 0) load_first(c - 1);
        cp_async_commit();
        cp_async_wait<1>();
        __syncthreads();
        // + dO^T A: token j takes tokens i >= j
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            float x[2][4];
            read_slice(x, dout, v_stride, valid, o_s, kb, lane);
            uint32_t f[OP1][4];
            acc_to_a<OP1>(x[0], x[1], f);
#pragma unroll
            for (int nn = 0; nn <= kb; nn += 2) {  // the last block pair's second may lie above the diagonal
                float y[4][4] = {};
                float (&u0)[4] = F32IO ? y[0] : du[2 * nn], (&u1)[4] = F32IO ? y[1] : du[2 * nn + 1];
                float (&u2)[4] = F32IO ? y[2] : du[(2 * nn + 2) & 7], (&u3)[4] = F32IO ? y[3] : du[(2 * nn + 3) & 7];
#pragma unroll
                for (int pl = kPlanes - 1; pl >= 0; --pl) {
                    uint32_t b[4], e[4];
                    load_b_t(b, sm + L::A + pl * L::kMat, kb * 16, nn * 16, lane);
                    if (nn < kb) load_b_t(e, sm + L::A + pl * L::kMat, kb * 16, nn * 16 + 16, lane);
                    if (nn < kb) mma_planes2<OP1, kPlanes>(u0, u1, u2, u3, f, b, e, pl);
                    else mma_planes<OP1, kPlanes>(u0, u1, f, b, pl);
                }
                if (F32IO) add_to(du[2 * nn], y[0]), add_to(du[2 * nn + 1], y[1]);
                if (F32IO && nn < kb) add_to(du[2 * nn + 2], y[2]), add_to(du[2 * nn + 3], y[3]);
            }
        }
        // dV^T = dU^T T
        if (DELTA) {
            float w[8][4] = {};
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
                uint32_t f[kPlanes][4];
                acc_to_a<kPlanes>(du[2 * kb], du[2 * kb + 1], f);
#pragma unroll
                for (int nn = 0; nn <= kb; nn += 2) {  // the last block pair's second may lie above the diagonal
                    float y[4][4] = {};
                    float (&w0)[4] = F32IO ? y[0] : w[2 * nn], (&w1)[4] = F32IO ? y[1] : w[2 * nn + 1];
                    float (&w2)[4] = F32IO ? y[2] : w[(2 * nn + 2) & 7], (&w3)[4] = F32IO ? y[3] : w[(2 * nn + 3) & 7];
#pragma unroll
                    for (int pl = kPlanes - 1; pl >= 0; --pl) {
                        uint32_t b[4], e[4];
                        load_b_t(b, sm + L::T + pl * L::kMat, kb * 16, nn * 16, lane);
                        if (nn < kb) load_b_t(e, sm + L::T + pl * L::kMat, kb * 16, nn * 16 + 16, lane);
                        if (nn < kb) mma_planes2<kPlanes, kPlanes>(w0, w1, w2, w3, f, b, e, pl);
                        else mma_planes<kPlanes, kPlanes>(w0, w1, f, b, pl);
                    }
                    if (F32IO) add_to(w[2 * nn], y[0]), add_to(w[2 * nn + 1], y[1]);
                    if (F32IO && nn < kb) add_to(w[2 * nn + 2], y[2]), add_to(w[2 * nn + 3], y[3]);
                }
            }
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) du[n][e] = w[n][e];
            store_slice(a.dV + unit * kChunk * a.dv + v0, a.dv, kChunk, du, 0u, lane);
        }
        store_slice(static_cast<IO *>(a.dv_out) + (size_t)(tok0 + c * kChunk) * v_stride + (size_t)h * a.dv + v0, v_stride, valid, du, stage, lane);
        __syncthreads();
        if (c > 0) load_matrices(c - 1);
        cp_async_commit();
        // dS^T <- e^(G_end) dS^T + dO^T (scale q e^G) - dV^T (k e^G); scalar decay scales the tokens of dO and dV
        if (VEC) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float2 d = *reinterpret_cast<const float2 *>(decay + 8 * n + 2 * t);
                s[n][0] *= d.x, s[n][1] *= d.y, s[n][2] *= d.x, s[n][3] *= d.y;
            }
        } else {
            const float d = decay[kChunk - 1];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[n][e] *= d;
        }
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            float x[2][4];
            read_slice(x, dout, v_stride, valid, o_s, kb, lane);
            float2 d[2] = {};
            if (!VEC) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    d[n] = *reinterpret_cast<const float2 *>(decay + kb * 16 + 8 * n + 2 * t);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[n][e] *= ((e & 1) ? d[n].y : d[n].x) * a.scale;
                }
            }
            {
                uint32_t f[OP2][4];
                acc_to_a<OP2>(x[0], x[1], f);
#pragma unroll
                for (int nn = 0; nn < NT / 2; nn += 2) {
                    float y[4][4] = {};
                    float (&s0)[4] = F32IO ? y[0] : s[2 * nn], (&s1)[4] = F32IO ? y[1] : s[2 * nn + 1];
                    float (&s2)[4] = F32IO ? y[2] : s[2 * nn + 2], (&s3)[4] = F32IO ? y[3] : s[2 * nn + 3];
#pragma unroll
                    for (int pl = L::kVecs - 1; pl >= 0; --pl) {
                        uint32_t b[4], e[4];
                        load_b_t(b, sm + L::q + pl * L::kTile, kb * 16, nn * 16, lane);
                        load_b_t(e, sm + L::q + pl * L::kTile, kb * 16, nn * 16 + 16, lane);
                        mma_planes2<OP2, kPlanes>(s0, s1, s2, s3, f, b, e, pl);
                    }
                    if (F32IO) add_to(s[2 * nn], y[0]), add_to(s[2 * nn + 1], y[1]), add_to(s[2 * nn + 2], y[2]), add_to(s[2 * nn + 3], y[3]);
                }
            }
            if (DELTA) {
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[n][e] = -du[2 * kb + n][e] * (VEC ? 1.f : ((e & 1) ? d[n].y : d[n].x));
                uint32_t f[kPlanes][4];
                acc_to_a<kPlanes>(x[0], x[1], f);
                const uint32_t kt_s = VEC ? sm + L::kt : k_s;
#pragma unroll
                for (int nn = 0; nn < NT / 2; nn += 2) {
                    float y[4][4] = {};
                    float (&s0)[4] = F32IO ? y[0] : s[2 * nn], (&s1)[4] = F32IO ? y[1] : s[2 * nn + 1];
                    float (&s2)[4] = F32IO ? y[2] : s[2 * nn + 2], (&s3)[4] = F32IO ? y[3] : s[2 * nn + 3];
#pragma unroll
                    for (int pl = L::kVecs - 1; pl >= 0; --pl) {
                        uint32_t b[4], e[4];
                        load_b_t(b, kt_s + pl * L::kTile, kb * 16, nn * 16, lane);
                        load_b_t(e, kt_s + pl * L::kTile, kb * 16, nn * 16 + 16, lane);
                        mma_planes2<kPlanes, kPlanes>(s0, s1, s2, s3, f, b, e, pl);
                    }
                    if (F32IO) add_to(s[2 * nn], y[0]), add_to(s[2 * nn + 1], y[1]), add_to(s[2 * nn + 2], y[2]), add_to(s[2 * nn + 3], y[3]);
                }
            }
        }
        __syncthreads();
        if (c > 0) load_update(c - 1);
        cp_async_commit();
    }
    cp_async_wait_all();
    if (a.dS_init) store_state<NT>(s, a.dS_init, false, s_off, a.dv, v0, lane);
}

}  // namespace deltalog
