// The chain over a sequence's chunks: S, U and the outputs.
//
// Everything is computed transposed.  A warp owns 16 columns of d_v and holds S^T [16 x d_k] in its accumulators for
// the whole sequence: the accumulator layout of one product is the A operand layout of the next, so the chain
//     S^T -> (k S)^T -> R^T -> U^T = R^T T^T -> O^T, S^T
// never leaves the registers, and no two warps exchange anything.  Shared memory carries the operands common to a
// CTA's warps (q, k, A, T), which are replaced as soon as their product is done while the next product runs.
//
// For d_v = 64 (d_v = 128: scan_forward_tc_kernel).  Bound by mma.sync: a chunk's products follow
// one another, and a scheduler starts one m16n8k16 every 8 cycles, 22 from an accumulator to its next use.
// RWKV6, bf16, 64 heads of 64: 17k tokens of 33 prompts 252 us, four rows of 1024 tokens with kept states 77 us.
#pragma once

#include "scan_common.cuh"

namespace deltalog {

template <bool VEC, int P, int DK, bool DELTA, typename IO>
struct ForwardSmem {
    static constexpr int kTile = kChunk * DK * 2;       // one plane of q or k
    static constexpr int kMat = kChunk * kChunk * 2;    // one plane of A or T
    static constexpr int kOut = sizeof(IO) == 4 ? kPlanes : 2;  // planes of what only the output sees
    static constexpr int kQ = VEC ? kOut : P, kK = VEC ? kPlanes : P;
    static constexpr int kDecay = VEC ? DK * 4 : 2 * kChunk * 4;
    // Scalar decay: q and k, which the first and the last product of a chunk read; bf16 k has two places so that the next
    // chunk's can be on its way in between.  Per channel: q e^G, k e^G (delta rule) and k e^(G_end - G).
    static constexpr bool kTwice = !VEC && P == 1;
    static constexpr int q = 0;
    static constexpr int k = kQ * kTile;
    static constexpr int kh = k + (VEC && DELTA ? kK * kTile : 0);
    static constexpr int A = kh + (kTwice ? 2 : 1) * kK * kTile;
    static constexpr int T = A + kOut * kMat;
    static constexpr int decay = T + (DELTA ? kPlanes * kMat : 0);  // twice
    static constexpr int slices = decay + 2 * kDecay;               // bf16 io, per warp: v, staging
    static constexpr int per_warp = sizeof(IO) == 4 ? 0 : 2 * kChunk * 32;
    static constexpr size_t bytes(int warps) { return slices + (size_t)warps * per_warp; }
};

template <bool VEC, int P, int DK, bool DELTA, typename IO>
__global__ void __launch_bounds__(128, 1) scan_forward_kernel(const ScanArgs a) {
    using L = ForwardSmem<VEC, P, DK, DELTA, IO>;
    constexpr int NT = DK / 8;
    constexpr bool F32IO = sizeof(IO) == 4;
    constexpr int UP = DELTA || F32IO ? kPlanes : 1;  // planes of U (bf16 v is exact in one)
    constexpr int UO = UP < L::kOut ? UP : L::kOut;
    extern __shared__ __align__(128) unsigned char smem[];
    const uint32_t sm = smem_addr(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nthreads = blockDim.x;
    scan_kernel_begin(a.S_out != nullptr);
    const int seq = a.order[blockIdx.x / a.H], h = blockIdx.x % a.H, hq = h / (a.H / a.Hq);
    const int v0 = (blockIdx.y * (nthreads >> 5) + warp) * 16;
    const int t = lane & 3;
    int slot;
    if (!scan_slot(a, seq, tid, slot)) return;
    const int tok0 = a.starts[seq], len = a.starts[seq + 1] - tok0, nchunks = (len + kChunk - 1) / kChunk;
    if (nchunks == 0 && a.slots) return;
    const int chunk0 = a.chunk_starts[seq];
    const size_t tile = (size_t)DK * a.dv, s_off = ((size_t)slot * a.H + h) * tile;
    const size_t v_stride = (size_t)a.H * a.dv;
    const uint32_t v_s = sm + L::slices + warp * L::per_warp, stage = v_s + kChunk * 32;

    auto load_raw = [&](uint32_t dst, const void *raw, const __nv_bfloat16 *image, int c) {  // q or k of a chunk
        load_vectors_tile<P, DK>(dst, raw, image, a, tok0 + c * kChunk, chunk0 + c, hq, min(kChunk, len - c * kChunk), tid, nthreads);
    };
    auto load_decayed = [&](uint32_t dst, const __nv_bfloat16 *src, int planes, size_t unit) {
        load_image(dst, src + unit * kPlanes * kChunk * DK, planes * L::kTile, tid, nthreads);
    };
    auto load_vectors = [&](int c) {  // operands of the products with S, and the decay factors
        const size_t unit = (size_t)(chunk0 + c) * a.H + h;
        if (VEC) {
            load_decayed(sm + L::q, a.qt, L::kQ, unit);
            if (DELTA) load_decayed(sm + L::k, a.kt, L::kK, unit);
        } else {
            load_raw(sm + L::q, a.q, a.qi, c);
            if (L::kTwice) load_raw(sm + L::k + (c & 1) * L::kTile, a.k, a.ki, c);
        }
        for (int i = tid; i < L::kDecay / 16; i += nthreads)
            cp_async16(smem + L::decay + (c & 1) * L::kDecay + i * 16, a.decay + unit * (L::kDecay / 4) + i * 4);
    };
    auto load_matrices = [&](int c) {
        const size_t unit = (size_t)(chunk0 + c) * a.H + h, at = unit * kPlanes * kChunk * kChunk;
        load_image(sm + L::A, a.A + at, L::kOut * L::kMat, tid, nthreads);
        if (DELTA) load_image(sm + L::T, a.T + at, kPlanes * L::kMat, tid, nthreads);
        if constexpr (!F32IO)
            load_slice(v_s, static_cast<const IO *>(a.v) + (size_t)(tok0 + c * kChunk) * v_stride + (size_t)h * a.dv + v0, v_stride,
                       min(kChunk, len - c * kChunk), lane);
    };
    auto load_update = [&](int c) {
        if (VEC) load_decayed(sm + L::kh, a.kh, L::kK, (size_t)(chunk0 + c) * a.H + h);
        else if (!L::kTwice) load_raw(sm + L::k, a.k, a.ki, c);
    };
    if (nchunks > 0) {
        load_vectors(0), cp_async_commit();
        load_matrices(0), cp_async_commit();
        load_update(0), cp_async_commit();
    }
    float s[NT][4];
    if (a.S_in && !(a.fresh && a.fresh[seq])) {
        load_state<NT>(s, a.S_in, a.in_bf16, s_off, a.dv, v0, lane);
    } else {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
    }

    for (int c = 0; c < nchunks; ++c) {
        const size_t unit = (size_t)(chunk0 + c) * a.H + h;
        const int valid = min(kChunk, len - c * kChunk);
        const float *decay = reinterpret_cast<const float *>(smem + L::decay + (c & 1) * L::kDecay);
        const uint32_t k_s = sm + L::k + (L::kTwice ? (c & 1) * L::kTile : 0);
        cp_async_wait<VEC || L::kTwice ? 2 : 0>();
        __syncthreads();
        if (a.keep) keep_state<NT>(a.S + unit * tile, s, v0, lane);
        // (k S)^T and (q S)^T
        float ak[8][4] = {}, aq[8][4] = {};
#pragma unroll
        for (int kk = 0; kk < DK / 16; ++kk) {
            uint32_t f[kPlanes][4];
            acc_to_a<kPlanes>(s[2 * kk], s[2 * kk + 1], f);
#pragma unroll
            for (int nn = 0; nn < 4; nn += DELTA ? 1 : 2) {
                // delta rule: k and q in turn; otherwise two tiles of q
                // (fp32 io: a step's products apart from the sum, see mma_planes)
                float x[4][4] = {};
                float (&k0)[4] = F32IO ? x[2] : ak[2 * nn], (&k1)[4] = F32IO ? x[3] : ak[2 * nn + 1];
                float (&q0)[4] = F32IO ? x[0] : aq[2 * nn], (&q1)[4] = F32IO ? x[1] : aq[2 * nn + 1];
                float (&q2)[4] = F32IO ? x[2] : aq[(2 * nn + 2) & 7], (&q3)[4] = F32IO ? x[3] : aq[(2 * nn + 3) & 7];
#pragma unroll
                for (int pl = kPlanes - 1; pl >= 0; --pl) {
                    uint32_t b[4], e[4];
                    if (DELTA && pl < L::kK) load_b(b, k_s + pl * L::kTile, nn * 16, kk * 16, lane);
                    if (pl < L::kQ) load_b(e, sm + L::q + pl * L::kTile, nn * 16, kk * 16, lane);
                    if (!DELTA && pl < L::kQ) load_b(b, sm + L::q + pl * L::kTile, nn * 16 + 16, kk * 16, lane);
#pragma unroll
                    for (int pa = kPlanes - 1 - pl; pa >= 0; --pa) {
                        const bool q = pl < L::kQ && pa + pl < L::kOut;
                        if (DELTA && pl < L::kK) mma(k0, f[pa], b[0], b[1]), mma(k1, f[pa], b[2], b[3]);
                        if (q) mma(q0, f[pa], e[0], e[1]), mma(q1, f[pa], e[2], e[3]);
                        if (q && !DELTA) mma(q2, f[pa], b[0], b[1]), mma(q3, f[pa], b[2], b[3]);
                    }
                }
                if (F32IO) add_to(aq[2 * nn], x[0]), add_to(aq[2 * nn + 1], x[1]);
                if (F32IO && !DELTA) add_to(aq[(2 * nn + 2) & 7], x[2]), add_to(aq[(2 * nn + 3) & 7], x[3]);
                if (F32IO && DELTA) add_to(ak[2 * nn], x[2]), add_to(ak[2 * nn + 1], x[3]);
            }
        }
        __syncthreads();
        if (c + 1 < nchunks) load_vectors(c + 1);
        cp_async_commit();
        cp_async_wait<2>();
        __syncthreads();
        // R^T = V^T - (k e^G S)^T, in the registers of (k S)^T
        float u[8][4];
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            float x[2][4];
            read_slice(x, static_cast<const IO *>(a.v) + (size_t)(tok0 + c * kChunk) * v_stride + (size_t)h * a.dv + v0, v_stride, valid, v_s, kb, lane);
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int col = (2 * kb + n) * 8 + 2 * t;
                const float d0 = VEC ? 1.f : decay[col], d1 = VEC ? 1.f : decay[col + 1];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (DELTA) ak[2 * kb + n][e] = fmaf(-((e & 1) ? d1 : d0), ak[2 * kb + n][e], x[n][e]);
                    else u[2 * kb + n][e] = x[n][e];
                    if (!VEC) aq[2 * kb + n][e] *= ((e & 1) ? d1 : d0) * a.scale;
                }
            }
        }
        // U^T = R^T T^T: token i takes tokens j <= i
        if (DELTA) {
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) u[n][e] = 0.f;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb) {
                uint32_t f[kPlanes][4], b[4];
                acc_to_a<kPlanes>(ak[2 * kb], ak[2 * kb + 1], f);
#pragma unroll
                for (int nn = kb & ~1; nn < 4; nn += 2) {  // the block pairs' first may lie above the diagonal
                    float x[4][4] = {};
                    float (&u0)[4] = F32IO ? x[0] : u[2 * nn], (&u1)[4] = F32IO ? x[1] : u[2 * nn + 1];
                    float (&u2)[4] = F32IO ? x[2] : u[2 * nn + 2], (&u3)[4] = F32IO ? x[3] : u[2 * nn + 3];
#pragma unroll
                    for (int pl = kPlanes - 1; pl >= 0; --pl) {
                        uint32_t e[4];
                        if (nn >= kb) load_b(b, sm + L::T + pl * L::kMat, nn * 16, kb * 16, lane);
                        load_b(e, sm + L::T + pl * L::kMat, nn * 16 + 16, kb * 16, lane);
                        if (nn >= kb) mma_planes2<kPlanes, kPlanes>(u0, u1, u2, u3, f, b, e, pl);
                        else mma_planes<kPlanes, kPlanes>(u2, u3, f, e, pl);
                    }
                    if (F32IO && nn >= kb) add_to(u[2 * nn], x[0]), add_to(u[2 * nn + 1], x[1]);
                    if (F32IO) add_to(u[2 * nn + 2], x[2]), add_to(u[2 * nn + 3], x[3]);
                }
            }
            if (a.keep) store_slice(a.U + unit * kChunk * a.dv + v0, a.dv, kChunk, u, 0u, lane);
        }
        // O^T += U^T A^T
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            uint32_t f[UO][4], b[4];
            acc_to_a<UO>(u[2 * kb], u[2 * kb + 1], f);
#pragma unroll
            for (int nn = kb & ~1; nn < 4; nn += 2) {
                float x[4][4] = {};
                float (&o0)[4] = F32IO ? x[0] : aq[2 * nn], (&o1)[4] = F32IO ? x[1] : aq[2 * nn + 1];
                float (&o2)[4] = F32IO ? x[2] : aq[2 * nn + 2], (&o3)[4] = F32IO ? x[3] : aq[2 * nn + 3];
#pragma unroll
                for (int pl = L::kOut - 1; pl >= 0; --pl) {
                    uint32_t e[4];
                    if (nn >= kb) load_b(b, sm + L::A + pl * L::kMat, nn * 16, kb * 16, lane);
                    load_b(e, sm + L::A + pl * L::kMat, nn * 16 + 16, kb * 16, lane);
                    if (nn >= kb) mma_planes2<UO, L::kOut>(o0, o1, o2, o3, f, b, e, pl);
                    else mma_planes<UO, L::kOut>(o2, o3, f, e, pl);
                }
                if (F32IO && nn >= kb) add_to(aq[2 * nn], x[0]), add_to(aq[2 * nn + 1], x[1]);
                if (F32IO) add_to(aq[2 * nn + 2], x[2]), add_to(aq[2 * nn + 3], x[3]);
            }
        }
        if (a.out)
            store_slice(static_cast<IO *>(a.out) + (size_t)(tok0 + c * kChunk) * v_stride + (size_t)h * a.dv + v0, v_stride, valid, aq, stage, lane);
        __syncthreads();
        if (c + 1 < nchunks) load_matrices(c + 1);
        cp_async_commit();
        if (VEC) {
            cp_async_wait<2>();
            __syncthreads();
        }
        // S^T <- e^(G_end) S^T + U^T (k e^(G_end - G)); scalar decay scales U's tokens instead of k's
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
        const uint32_t ku_s = VEC ? sm + L::kh : k_s;
        constexpr int US = VEC ? UP : kPlanes;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            if (!VEC) {
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float2 d = *reinterpret_cast<const float2 *>(decay + kChunk + (2 * kb + n) * 8 + 2 * t);
                    u[2 * kb + n][0] *= d.x, u[2 * kb + n][1] *= d.y, u[2 * kb + n][2] *= d.x, u[2 * kb + n][3] *= d.y;
                }
            }
            uint32_t f[US][4];
            acc_to_a<US>(u[2 * kb], u[2 * kb + 1], f);
#pragma unroll
            for (int nn = 0; nn < NT / 2; nn += 2) {
                float x[4][4] = {};
                float (&s0)[4] = F32IO ? x[0] : s[2 * nn], (&s1)[4] = F32IO ? x[1] : s[2 * nn + 1];
                float (&s2)[4] = F32IO ? x[2] : s[2 * nn + 2], (&s3)[4] = F32IO ? x[3] : s[2 * nn + 3];
#pragma unroll
                for (int pl = L::kK - 1; pl >= 0; --pl) {
                    uint32_t b[4], e[4];
                    load_b_t(b, ku_s + pl * L::kTile, kb * 16, nn * 16, lane);
                    load_b_t(e, ku_s + pl * L::kTile, kb * 16, nn * 16 + 16, lane);
                    mma_planes2<US, kPlanes>(s0, s1, s2, s3, f, b, e, pl);
                }
                if (F32IO) add_to(s[2 * nn], x[0]), add_to(s[2 * nn + 1], x[1]), add_to(s[2 * nn + 2], x[2]), add_to(s[2 * nn + 3], x[3]);
            }
        }
        if (!L::kTwice) __syncthreads();
        if (c + 1 < nchunks) load_update(c + 1);
        cp_async_commit();
    }
    cp_async_wait_all();
    if (a.S_out) store_state<NT>(s, a.S_out, a.out_bf16, s_off, a.dv, v0, lane);
    if (a.log_len && blockIdx.y == 0 && tid == 0) a.log_len[(size_t)slot * a.H + h] = 0;
}

}  // namespace deltalog
