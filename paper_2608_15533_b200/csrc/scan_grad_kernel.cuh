// Gradients of q, k, g, beta (and the bonus) of one chunk and head, all chunks in parallel.
//
// With the state S_0 in front of the chunk, the gradient dS_1 behind it, U, dO and dV at hand:
//     dA = dO U^T   dL' = -dV U^T   (L' = L / beta)                      [64 x 64], masked
//     dq = scale e^G dO S_0^T + (dA through A)
//     dk as written = e^(G_end - G) U dS_1^T + (dA, dL' through A, L')    dk as read = -e^G dV S_0^T + (dL' through L')
//     dbeta_t = sum_v dV_t U_t / beta_t^2
// and for the log-decay, with every factor that reaches across token t's decay counted once,
//     dg_t = e^(G_end) <dS_1, S_0> + sum_(s < t) k_s (dk_s as written behind the chunk)
//          + sum_(s >= t) q_s dq_s + k_s (dk_s as read) - k_s (dk_s as written, inside the chunk).
// Only the last difference cancels, inside one chunk; the sums that span chunks come from the states themselves, so
// no error grows with the length of the sequence.  dA's diagonal, a token's readout of its own write, crosses no decay: it
// is kept out of the difference (where gates are strong it would be all that is there) and added to dq and dk afterwards;
// so is, for RWKV6, the readout of the token in front, which crosses none either.
//
// The [64 x d_k] products contract over d_v, so S_0, dS_1, dO, U and dV stream through shared memory in slices of 32
// columns of d_v, the next slice on its way while one is multiplied.  fp32 operands stay fp32 there (two bytes per element
// less than three planes, and both orientations from one tile); a warp forms its fragments' planes as it reads them.
// With bf16 io the products over d_v take fp32 operands in two planes: they end in dq, dk (bf16) and in sums that do not
// cancel.  The products inside the chunk take three: dg is the difference of their sums, and two planes left 2e-5 of it
// for per-channel gates.
// Bound by the phases of a chunk, one behind the other in the only CTA of an SM: 200 KB of operands (5k cycles, from L2), the
// products over d_v and the sums beside them (9k), the products inside the chunk (10k; per-channel gates 30k).  bf16, 32 heads of 128:
// GDN 8k tokens 427 us, 36.7k tokens 1936 us (2.8 TB/s of DRAM traffic; 2644 us before the next wave's
// operands went to L2 ahead and the in-chunk part shared its own), KDA 3.9k tokens
// 441 us; RWKV6, 64 heads of 64, 4k tokens 435 us on mma.sync.  With the products over d_v on mma.sync as well GDN took 1.5 times
// as long.
// 512 threads; warp w owns token rows 16 (w & 3) .. + 15 and the channel quarter w >> 2 of every result: the work between
// two barriers is a few hundred instructions per warp, and sixteen warps cover each other's latencies where eight did not.
#pragma once

#include "scan_common.cuh"
#include "scan_prep_kernel.cuh"
#include "scan_tc_common.cuh"

namespace deltalog {

constexpr int kGradThreads = 512;
constexpr int kSlice = 32;
constexpr int kSliceStride = kSlice + 8;

// fp32 tile of rows `stride` elements apart to padded rows of `w` floats; rows at and behind `valid` become zeros.
template <int COLS>
__device__ __forceinline__ void load_f32(float *dst, const float *src, size_t stride, int rows, int w, int valid, int tid) {
    constexpr int kUnits = COLS / 4;
    for (int i = tid; i < rows * kUnits; i += kGradThreads) {
        const int row = i / kUnits, unit = i % kUnits;
        const bool ok = row < valid;
        cp_async16_zfill(smem_addr(dst + row * w + unit * 4), src + (ok ? (size_t)row * stride + unit * 4 : 0), ok);
    }
}
// bf16 tile of 64 rows of 32 elements (64 bytes): 16-byte units permuted by the row's bits 1 and 2.
__device__ __forceinline__ uint32_t slice32_addr(uint32_t base, int row, int unit) {
    return base + (uint32_t)(row * 64 + ((unit ^ ((row >> 1) & 3)) << 4));
}
// A slice of the io tensors: bf16 as it is, fp32 padded.
__device__ __forceinline__ void load_io(unsigned char *dst, const __nv_bfloat16 *src, size_t stride, int valid, int tid) {
    if (tid < kChunk * 4) {
        const int row = tid >> 2, unit = tid & 3;
        const bool ok = row < valid;
        cp_async16_zfill(slice32_addr(smem_addr(dst), row, unit), src + (ok ? (size_t)row * stride + unit * 8 : 0), ok);
    }
}
__device__ __forceinline__ void load_io(unsigned char *dst, const float *src, size_t stride, int valid, int tid) {
    load_f32<kSlice>(reinterpret_cast<float *>(dst), src, stride, kChunk, kSliceStride, valid, tid);
}
__device__ __forceinline__ void io_frag_a(uint32_t (&f)[1][4], const unsigned char *tile, int m0, int k0, int lane) {
    const int m = lane >> 3, x = lane & 7;
    ldsm4(f[0], slice32_addr(smem_addr(tile), m0 + (m & 1) * 8 + x, (k0 >> 3) + (m >> 1)));
}
__device__ __forceinline__ void io_frag_a(uint32_t (&f)[kPlanes][4], const unsigned char *tile, int m0, int k0, int lane) {
    frag_a(f, reinterpret_cast<const float *>(tile), kSliceStride, m0, k0, lane);
}
__device__ __forceinline__ void io_frag_b(uint32_t (&f)[1][4], const unsigned char *tile, int n0, int k0, int lane) {
    const int m = lane >> 3, x = lane & 7;
    ldsm4(f[0], slice32_addr(smem_addr(tile), n0 + (m >> 1) * 8 + x, (k0 >> 3) + (m & 1)));
}
__device__ __forceinline__ void io_frag_b(uint32_t (&f)[kPlanes][4], const unsigned char *tile, int n0, int k0, int lane) {
    frag_b(f, reinterpret_cast<const float *>(tile), kSliceStride, n0, k0, lane);
}

// A strongly decaying block's own pairs, one by one: for element (i, c) the sum over j <= i of mat_ij k_jc e^(G_i - G_j) ...
// (Out of line, with pointers to the chunk's first token at channel c: rarely taken, and inlined at every element they pushed
// the kernel out of the instruction cache.)
template <typename IO, bool EXCL>
__device__ __noinline__ float pairs_front(const IO *k, int k_stride, const float *gate, int g_stride, int valid, const float *mat, int w, int i) {
    float s = 0.f, x = 0.f;
    for (int j = i; j >= (i & ~(kBlock - 1)); --j) {
        if (j < i && !(EXCL && j + 1 == i) && j + 1 < valid) x += gate[(size_t)(j + 1) * g_stride];
        s = fmaf(j < valid ? mat[i * w + j] * to_f32(k[(size_t)j * k_stride]) : 0.f, expf(x), s);
    }
    return s;
}
// ... and over i >= j of (dA_ij q_ic + dL'_ij k_ic) e^(G_i - G_j).
template <typename IO, bool EXCL, bool DELTA>
__device__ __noinline__ float pairs_back(const IO *q, const IO *k, int k_stride, const float *gate, int g_stride, int valid, const float *da, const float *dl,
                                         int w, int j) {
    float s = 0.f, x = 0.f;
    const int end = min((j & ~(kBlock - 1)) + kBlock, valid);
    for (int i = j; i < end; ++i) {
        const int m = EXCL ? i - 1 : i;  // the last gate that decays the pair
        if (m > j) x += gate[(size_t)m * g_stride];
        float y = da[i * w + j] * to_f32(q[(size_t)i * k_stride]);
        if (DELTA) y = fmaf(dl[i * w + j], to_f32(k[(size_t)i * k_stride]), y);
        s = fmaf(y, expf(x), s);
    }
    return s;
}

template <int OP, int P, int DK, typename IO, bool TC>
struct GradSmem {
    static constexpr bool VEC = OpTraits<OP>::kVecDecay, DELTA = OpTraits<OP>::kDeltaRule;
    static constexpr int kTile = kChunk * DK * 2;
    static constexpr int kSW = DK + 4;              // row of a state slice or of a decayed vector
    static constexpr int kMW = kChunk + 8;          // row of dA, dL'
    static constexpr int kMat = kChunk * kMW * 4, kMats = (DELTA ? 2 : 1) * kMat;
    static constexpr int kF32 = kChunk * kSliceStride * 4;
    static constexpr int kIO = sizeof(IO) == 4 ? kF32 : kChunk * kSlice * 2;
    static constexpr int most(int x, int y) { return x > y ? x : y; }
    // a stage: slices of S_0, dS_1, dO, U (or v), dV;  TC: S_0, dS_1, U (or v) whole, as images
    static constexpr int kState = TC ? 2 * DK * 256 : kSlice * kSW * 4;
    static constexpr int dS = kState, dO = 2 * kState, U = TC ? 2 * kState : dO + kIO;
    static constexpr int dV = U + (TC ? (DELTA ? 2 : 1) * kChunk * 256 : DELTA ? kF32 : kIO), stage = TC ? dV : dV + (DELTA ? kF32 : 0);
    static constexpr int loaded = TC ? stage : 2 * stage;
    // after them: q and k planes (bf16 io: in a place of their own, loaded meanwhile), or the three decayed vectors and the
    // decays in front of and behind a token inside its block
    static constexpr bool kOwnQK = !VEC && P == 1;
    static constexpr int qk = kOwnQK ? loaded : 0;
    static constexpr int last = VEC ? (DELTA ? 5 : 4) * kChunk * kSW * 4 : qk + 2 * P * kTile;
    // dA, dL': behind all that; where that is too much (TC, scalar decay, d_k = 128) in S_0's place, which is done with by then
    static constexpr bool kInPlace = TC && !VEC && DK == 128;
    static constexpr int mats = kInPlace ? 0 : most(loaded, last);
    static constexpr int small = kInPlace ? most(loaded, last) : mats + kMats;
    static constexpr int part = small;                  // [1024] partial sums of <dS, S>
    static constexpr int rows = part + 4096;            // [8][64] row sums of the channel quarters
    static constexpr int tables = rows + 8 * kChunk * 4; // [4][4][DK] e^(decay) of the chunk in front of / behind a block, of the block, inverse
    static constexpr int beta = tables + (VEC ? 16 * DK * 4 : 0);
    static constexpr int G = beta + 2 * kChunk * 4;     // beta, diagonal of dA;  sums of the scalar decay
    static constexpr int deep = G + kChunk * 8;
    static constexpr int control = deep + 16;
    static constexpr size_t total = control + (TC ? kTcControlBytes : 0);
    static constexpr size_t bytes = TC && total < kTcMinSmem ? kTcMinSmem : total;
};

// A pair of neighbouring channels of the io tensors' row.
template <typename IO>
__device__ __forceinline__ float2 load_pair(const void *src, size_t at) {
    float x[2];
    load_vec<IO, 2>(static_cast<const IO *>(src) + at, x);
    return make_float2(x[0], x[1]);
}

template <int OP, int P, int DK, typename IO, bool TC>
__global__ void __launch_bounds__(kGradThreads, 1) scan_grad_kernel(const ScanArgs a) {
    using L = GradSmem<OP, P, DK, IO, TC>;
    constexpr bool VEC = L::VEC, DELTA = L::DELTA, EXCL = OpTraits<OP>::kBonus;
    constexpr int NT = DK / 32, SW = L::kSW, MW = L::kMW;
    constexpr int GP = sizeof(IO) == 4 ? kPlanes : 2;  // planes of an fp32 operand
    constexpr int IP = sizeof(IO) == 4 ? GP : 1;       // and of dO and v
    constexpr bool kApart = sizeof(IO) == 4;           // a step's plane products apart from the sum (two planes leave more than the cut)
    extern __shared__ __align__(1024) unsigned char smem_grad[];
    unsigned char *smem = smem_grad;
    const uint32_t sm = smem_addr(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), chunk = blockIdx.x, h = blockIdx.y;
    const int g = lane >> 2, t = lane & 3, mt = warp & 3, cq = warp >> 2, c0 = cq * (DK / 4);
    scan_kernel_begin();
    ChunkPlace p;
    if (!chunk_place(a, chunk, p)) return;
    const int dv = a.dv, hq = h / (a.H / a.Hq);
    const size_t unit = (size_t)chunk * a.H + h, tile = (size_t)DK * dv;
    float *da_f = reinterpret_cast<float *>(smem + L::mats), *dl_f = da_f + kChunk * MW;
    float *part = reinterpret_cast<float *>(smem + L::part), *rows = reinterpret_cast<float *>(smem + L::rows);
    float *beta = reinterpret_cast<float *>(smem + L::beta), *diag = beta + kChunk;
    float *near = beta;  // RWKV6 (no beta): dA's entries next to the diagonal
    float2 *G = reinterpret_cast<float2 *>(smem + L::G);
    int *deep = reinterpret_cast<int *>(smem + L::deep);
    const size_t v_off = ((size_t)p.tok0 * a.H + h) * dv, v_stride = (size_t)a.H * dv;

    auto load_stage = [&](int s) {
        unsigned char *st = smem + (s & 1) * L::stage;
        const int v = s * kSlice;
        load_f32<DK>(reinterpret_cast<float *>(st), a.S + unit * tile + (size_t)v * DK, DK, kSlice, SW, kSlice, tid);
        load_f32<DK>(reinterpret_cast<float *>(st + L::dS), a.dS + unit * tile + (size_t)v * DK, DK, kSlice, SW, kSlice, tid);
        load_io(st + L::dO, static_cast<const IO *>(a.dout) + v_off + v, v_stride, p.valid, tid);
        if (DELTA) {
            load_f32<kSlice>(reinterpret_cast<float *>(st + L::U), a.U + unit * kChunk * dv + v, dv, kChunk, kSliceStride, kChunk, tid);
            load_f32<kSlice>(reinterpret_cast<float *>(st + L::dV), a.dV + unit * kChunk * dv + v, dv, kChunk, kSliceStride, kChunk, tid);
        } else {
            load_io(st + L::U, static_cast<const IO *>(a.v) + v_off + v, v_stride, p.valid, tid);
        }
    };
    auto load_qk = [&]() {
        load_vectors_tile<P, DK>(sm + L::qk, a.q, a.qi, a, p.tok0, chunk, hq, p.valid, tid, kGradThreads);
        load_vectors_tile<P, DK>(sm + L::qk + P * L::kTile, a.k, a.ki, a, p.tok0, chunk, hq, p.valid, tid, kGradThreads);
    };
    if (tid < 4) deep[tid] = 0;
    if (!VEC && warp == 0) chunk_decay_sums(a, p, h, G, lane);
    if (DELTA && tid >= 64 && tid < 128) beta[tid - 64] = scan_beta(tid - 64 < p.valid ? a.beta[(size_t)(p.tok0 + tid - 64) * a.H + h] : 0.f);
    // dO S_0^T, dV S_0^T, U dS_1^T [16 x DK/4] and, where the warp's 16 columns are at or below the diagonal, dO U^T, dV U^T
    float dq[NT][4] = {}, dr[NT][4] = {}, dw[NT][4] = {}, da[2][4] = {}, dl[2][4] = {};
    float dot0 = 0.f, dot1 = 0.f, db = 0.f;
    constexpr int kPairs = DK / 2, kGroups = kGradThreads / kPairs;
    // (TC: a warp reads eight v of eight channels, 128 bytes in one piece)
    const int cp = TC ? warp % (kPairs / 4) * 4 + (lane & 3) : tid % kPairs, grp = TC ? warp / (kPairs / 4) * 8 + (lane >> 2) : tid / kPairs;
    // dA and dL', masked; scalar decay multiplies e^(G_i - G_j) in here
    auto write_mats = [&]() {
        if (cq > mt) return;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int i = mt * 16 + g + 8 * half, j = cq * 16 + n * 8 + 2 * t;
                    float x[2], y[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float m = VEC ? 1.f : (j + e <= i ? decay_exp(decay_between(G[i], G[j + e])) : 0.f);
                        const float raw = da[n][2 * half + e];
                        if (i == j + e) diag[i] = raw * a.scale;
                        if (EXCL && i == j + e + 1) near[i] = raw;
                        x[e] = j + e + (EXCL ? 1 : 0) < i ? raw * m * a.scale : 0.f;
                        y[e] = j + e < i ? -dl[n][2 * half + e] * m : 0.f;
                    }
                    *reinterpret_cast<float2 *>(da_f + i * MW + j) = make_float2(x[0], x[1]);
                    if (DELTA) *reinterpret_cast<float2 *>(dl_f + i * MW + j) = make_float2(y[0], y[1]);
                }
    };
    TcBlock tc = {};
    if constexpr (TC) {
        // On the tensor cores, d_v = 128: row 32 q + r of the A operand is dO of token 16 q + r (r < 16) or dV of token 16 q + r - 16, so
        // that the warp that owns a token block reads its results from its own lanes, in mma.sync's accumulator layout.
        // Tensor memory: planes of A (of U later), [dO; dV] S_0^T, [dO; dV] U^T, U dS_1^T.
        constexpr uint32_t PA = 0, D1 = 128, D2 = 256, D3 = 320;
        constexpr int UP = DELTA ? 2 : 1;
        const int tok = mt * 16 + (lane & 15), v0 = 32 * cq;  // this thread's row of A and columns
        const bool upper = lane >= 16, inside = tok < p.valid;
        uint4 hi[4], lo[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) hi[i] = lo[i] = make_uint4(0u, 0u, 0u, 0u);
        if (!upper && inside) {
            const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.dout) + v_off + (size_t)tok * v_stride + v0);
#pragma unroll
            for (int i = 0; i < 4; ++i) hi[i] = src[i];
        }
        if (DELTA && upper) {
            const unsigned char *src = reinterpret_cast<const unsigned char *>(a.dV + unit * kChunk * 128) + kept_dv_at(tok, v0);
#pragma unroll
            for (int i = 0; i < 4; ++i) hi[i] = reinterpret_cast<const uint4 *>(src)[i], lo[i] = reinterpret_cast<const uint4 *>(src + kChunk * 256)[i];
        }
        tc = tc_setup(smem + L::control, 4, tid);
        auto bar = [&](int i) { return tc.bars + 8u * i; };  // 0: S_0, 1: U, 2: dS_1, 3: products
        if (tid == 0) {
            mbar_arrive_expect_tx(bar(0), L::kState);
            bulk_copy_g2s(sm, a.S + unit * tile, L::kState, bar(0));
            if (DELTA) {
                mbar_arrive_expect_tx(bar(1), 2 * kChunk * 256);
                bulk_copy_g2s(sm + L::U, a.U + unit * kChunk * 128, 2 * kChunk * 256, bar(1));
            }
            mbar_arrive_expect_tx(bar(2), L::kState);
            bulk_copy_g2s(sm + L::dS, a.dS + unit * tile, L::kState, bar(2));
            // One CTA fills an SM and begins by waiting for 200 KB.  What the CTA a wave further on will want goes from DRAM to
            // L2 meanwhile (a CTA's wait 12k -> 5k cycles); the wave is 148 x 192 KB, 29 MB.
            const size_t next = (size_t)h * gridDim.x + chunk + a.wave, ahead = next % gridDim.x * a.H + next / gridDim.x;
            if (next < (size_t)gridDim.x * a.H) {
                l2_prefetch(a.S + ahead * tile, L::kState), l2_prefetch(a.dS + ahead * tile, L::kState);
                if (DELTA) l2_prefetch(a.U + ahead * kChunk * 128, 2 * kChunk * 256), l2_prefetch(a.dV + ahead * kChunk * 128, 2 * kChunk * 256);
            }
        }
        if (VEC && tid >= 64 && tid < 128 && tid - 64 < p.valid) {  // read from there later on
            const size_t at = p.tok0 + tid - 64;
            l2_prefetch(a.g + (at * a.H + h) * DK, DK * 4);
            l2_prefetch(static_cast<const IO *>(a.q) + (at * a.Hq + hq) * DK, DK * 2), l2_prefetch(static_cast<const IO *>(a.k) + (at * a.Hq + hq) * DK, DK * 2);
        }
        if constexpr (!DELTA && sizeof(IO) == 2) tc_load_operand<128, kChunk * 128>(sm + L::U, a.v, v_off, v_stride, p.valid, tid);
        if (L::kOwnQK) load_qk();
        cp_async_commit();
        bool ok = true;
        uint32_t phase = 0;
        auto handed_over = [&]() {
            tmem_wait_st();
            tc_fence_before();
            __syncthreads();
            tc_fence_after();
        };
        auto products_done = [&]() {
            ok = bounded_wait(bar(3), phase, tc.abort_flag) && ok;
            phase ^= 1;
            tc_fence_after();
        };
        auto issuing = [&]() { return warp == 0 && __all_sync(0xffffffffu, ok) && elect_one(); };
        const uint32_t row = tc.tmem + ((uint32_t)(32 * mt) << 16);
        auto put_row = [&](int plane, const uint4 (&w)[4]) {
            const uint32_t x[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
            const uint32_t y[8] = {w[2].x, w[2].y, w[2].z, w[2].w, w[3].x, w[3].y, w[3].z, w[3].w};
            tmem_st8(row + PA + plane * 64 + v0 / 2, x), tmem_st8(row + PA + plane * 64 + v0 / 2 + 8, y);
        };
        put_row(0, hi);
        if (DELTA) put_row(1, lo);
        if (!DELTA) cp_async_wait_all(), fence_async_proxy();  // v
        handed_over();
        ok = bounded_wait(bar(0), 0u, tc.abort_flag) && ok;
        if (DELTA) ok = bounded_wait(bar(1), 0u, tc.abort_flag) && ok;
        if (issuing()) {
            tc_product_state<UP, DK>(tc.tmem + D1, tc.tmem + PA, sm);
            tc_product<UP, 0, UP, 0, 2, false, 8, kChunk, 64, kChunk * 256, kChunk * 128>(tc.tmem + D2, tc.tmem + PA, sm + L::U);
            tc_commit(bar(3));
        }
        // meanwhile the sums of products: dbeta (by the threads that hold dV), <dS_1, S_0> by channel
        auto both = [&](const unsigned char *at, int plane) {  // a pair of values of two planes
            const uint32_t x = *reinterpret_cast<const uint32_t *>(at), y = *reinterpret_cast<const uint32_t *>(at + plane);
            return make_float2(bf16_lo(x) + bf16_lo(y), bf16_hi(x) + bf16_hi(y));
        };
        if (DELTA && upper) {
            const float rb = 1.f / beta[tok];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned char *at = smem + L::U + kept_u_at(tok, v0 + 8 * i);
                const uint4 uh = *reinterpret_cast<const uint4 *>(at), ul = *reinterpret_cast<const uint4 *>(at + kChunk * 256);
                const uint32_t x[4] = {uh.x, uh.y, uh.z, uh.w}, y[4] = {ul.x, ul.y, ul.z, ul.w};
                const uint32_t d[4] = {hi[i].x, hi[i].y, hi[i].z, hi[i].w}, e[4] = {lo[i].x, lo[i].y, lo[i].z, lo[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    db = fmaf((bf16_lo(x[j]) + bf16_lo(y[j])) * rb, (bf16_lo(d[j]) + bf16_lo(e[j])) * rb, db);
                    db = fmaf((bf16_hi(x[j]) + bf16_hi(y[j])) * rb, (bf16_hi(d[j]) + bf16_hi(e[j])) * rb, db);
                }
            }
            rows[cq * kChunk + tok] = db;
        }
        ok = bounded_wait(bar(2), 0u, tc.abort_flag) && ok;
        for (int v = grp; v < 128; v += kGroups) {
            const int at = kept_state_at(2 * cp, v);
            const float2 x = both(smem + at, DK * 256), d = both(smem + L::dS + at, DK * 256);
            dot0 = fmaf(d.x, x.x, dot0), dot1 = fmaf(d.y, x.y, dot1);
        }
        products_done();
        tmem_ld_frag(row + D1 + c0, dq);
        if (DELTA) tmem_ld_frag(row + (16u << 16) + D1 + c0, dr);
        tmem_ld_frag(row + D2 + cq * 16, da);
        if (DELTA) tmem_ld_frag(row + (16u << 16) + D2 + cq * 16, dl);
        {
            uint4 x[4];
#pragma unroll
            for (int pl = 0; pl < UP; ++pl) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    x[i] = upper ? make_uint4(0u, 0u, 0u, 0u) : *reinterpret_cast<const uint4 *>(smem + L::U + pl * kChunk * 256 + kept_u_at(tok, v0 + 8 * i));
                put_row(pl, x);
            }
        }
        handed_over();
        if (issuing()) {
            tc_product_state<UP, DK>(tc.tmem + D3, tc.tmem + PA, sm + L::dS);
            tc_commit(bar(3));
        }
        write_mats();  // (S_0's place, if so, is free: its product and the sums are behind the barrier)
        products_done();
        tmem_ld_frag(row + D3 + c0, dw);
        tc_fence_before();
        if (__syncthreads_or(!ok)) {  // a wait gave up: nothing of this chunk is valid
            if (tid == 0) {
                if (a.status) atomicOr(a.status, DELTALOG_STATUS_TIMEOUT);
                for (int i = 0; i < 3; ++i) bounded_wait(bar(i), 0u, tc.abort_flag + 1);
            }
            cp_async_wait_all();
            tc_teardown(tc, tid);
            return;
        }
        if (tid < 32) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tc.tmem), "r"(kTmemCols));
    } else {
    const int slices = dv / kSlice;
    load_stage(0), cp_async_commit();
    if (L::kOwnQK) load_qk();
    __syncthreads();  // beta
    for (int sl = 0; sl < slices; ++sl) {
        if (sl + 1 < slices) load_stage(sl + 1);
        cp_async_commit();
        cp_async_wait<1>();
        __syncthreads();
        const unsigned char *st = smem + (sl & 1) * L::stage;
        const float *S = reinterpret_cast<const float *>(st), *dS = reinterpret_cast<const float *>(st + L::dS);
        const float *u_f = reinterpret_cast<const float *>(st + L::U), *v_f = reinterpret_cast<const float *>(st + L::dV);
#pragma unroll
        for (int k0 = 0; k0 < kSlice; k0 += 16) {
            {
                uint32_t f[IP][4], e[GP][4];
                io_frag_a(f, st + L::dO, mt * 16, k0, lane);
                if (DELTA) frag_a(e, v_f, kSliceStride, mt * 16, k0, lane);
#pragma unroll
                for (int nn = 0; nn < NT / 2; ++nn) {
                    uint32_t b[GP][4];
                    frag_b_t(b, S, SW, k0, c0 + nn * 16, lane);
                    mma_all<kApart>(dq[2 * nn], dq[2 * nn + 1], f, b);
                    if (DELTA) mma_all<kApart>(dr[2 * nn], dr[2 * nn + 1], e, b);
                }
                if (cq <= mt) {
                    if constexpr (DELTA) {
                        uint32_t b[GP][4];
                        frag_b(b, u_f, kSliceStride, cq * 16, k0, lane);
                        mma_all<kApart>(da[0], da[1], f, b);
                        mma_all<kApart>(dl[0], dl[1], e, b);
                    } else {
                        uint32_t b[IP][4];
                        io_frag_b(b, st + L::U, cq * 16, k0, lane);
                        mma_all<kApart>(da[0], da[1], f, b);
                    }
                }
            }
            constexpr int UP = DELTA ? GP : IP;
            uint32_t f[UP][4];
            if constexpr (DELTA) frag_a(f, u_f, kSliceStride, mt * 16, k0, lane);
            else io_frag_a(f, st + L::U, mt * 16, k0, lane);
#pragma unroll
            for (int nn = 0; nn < NT / 2; ++nn) {
                uint32_t b[GP][4];
                frag_b_t(b, dS, SW, k0, c0 + nn * 16, lane);
                mma_all<kApart>(dw[2 * nn], dw[2 * nn + 1], f, b);
            }
        }
        // <dS_1, S_0> by channel, and sum_v dV U by token (eight threads each)
#pragma unroll
        for (int v = grp; v < kSlice; v += kGroups) {
            const float2 x = *reinterpret_cast<const float2 *>(S + v * SW + cp * 2), d = *reinterpret_cast<const float2 *>(dS + v * SW + cp * 2);
            dot0 = fmaf(d.x, x.x, dot0), dot1 = fmaf(d.y, x.y, dot1);
        }
        if (DELTA) {
            const int i = tid >> 3, v = (tid & 7) * 4;
            const float rb = 1.f / beta[i];
            const float4 u = *reinterpret_cast<const float4 *>(u_f + i * kSliceStride + v), d = *reinterpret_cast<const float4 *>(v_f + i * kSliceStride + v);
            db = fmaf(u.x * rb, d.x * rb, db), db = fmaf(u.y * rb, d.y * rb, db), db = fmaf(u.z * rb, d.z * rb, db), db = fmaf(u.w * rb, d.w * rb, db);
        }
        __syncthreads();
    }
    }
    part[grp * DK + cp * 2] = dot0, part[grp * DK + cp * 2 + 1] = dot1;
    if (DELTA && !TC) {
        db += __shfl_xor_sync(0xffffffffu, db, 1);
        db += __shfl_xor_sync(0xffffffffu, db, 2);
        db += __shfl_xor_sync(0xffffffffu, db, 4);
        if ((tid & 7) == 0 && (tid >> 3) < p.valid) a.dbeta[(size_t)(p.tok0 + (tid >> 3)) * a.H + h] = db;
    }
    if (DELTA && TC && tid < p.valid)  // (the quarters' sums met at a barrier)
        a.dbeta[(size_t)(p.tok0 + tid) * a.H + h] = (rows[tid] + rows[kChunk + tid]) + (rows[2 * kChunk + tid] + rows[3 * kChunk + tid]);
    if (!VEC && !L::kOwnQK) load_qk(), cp_async_commit();
    if (!TC) write_mats();
    const bool whole = a.H == a.Hq;
    // results of element pair (row i, channels c, c + 1)
    auto put = [&](void *io_dst, float *part_dst, int i, int c, float x, float y) {
        if (i >= p.valid) return;
        if (whole) {
            IO *d = static_cast<IO *>(io_dst) + ((size_t)(p.tok0 + i) * a.Hq + hq) * DK + c;
            if constexpr (sizeof(IO) == 2) *reinterpret_cast<uint32_t *>(d) = pack_bf16(x, y);
            else *reinterpret_cast<float2 *>(d) = make_float2(x, y);
        } else {
            *reinterpret_cast<float2 *>(part_dst + ((size_t)(p.tok0 + i) * a.H + h) * DK + c) = make_float2(x, y);
        }
    };

    if constexpr (!VEC) {
        const uint32_t q_s = sm + L::qk, k_s = q_s + P * L::kTile;
        cp_async_wait_all();
        __syncthreads();
        float y[2] = {0.f, 0.f}, b2[2] = {0.f, 0.f};
        auto value = [&](uint32_t base, int i, int c) {
            const unsigned char *at = smem + (base - sm) + image_at(i, c) * 2;
            const uint32_t w = *reinterpret_cast<const uint32_t *>(at);
            float2 v = make_float2(bf16_lo(w), bf16_hi(w));
#pragma unroll
            for (int pl = 1; pl < P; ++pl) {
                const uint32_t more = *reinterpret_cast<const uint32_t *>(at + pl * L::kTile);
                v.x += bf16_lo(more), v.y += bf16_hi(more);
            }
            return v;
        };
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int i = mt * 16 + g + 8 * r;
            const float front = expf(G[i].x + G[i].y), back = expf(decay_between(G[kChunk - 1], G[i]));
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float2 kv = value(k_s, i, c0 + n * 8 + 2 * t);
#pragma unroll
                for (int e = 2 * r; e < 2 * r + 2; ++e) {
                    dq[n][e] *= a.scale * front;
                    dr[n][e] *= -front;
                    dw[n][e] *= back;
                    b2[r] = fmaf((e & 1) ? kv.y : kv.x, dw[n][e], b2[r]);
                }
            }
        }
        // inside the chunk: dq += dA K, dk as written += dA^T Q + dL'^T K, dk as read += dL' K
        float di[NT][4] = {};
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            uint32_t m[kPlanes][4];
            // a product of one matrix (or its transpose) with the 16 tokens of block kb of q or k
            auto product = [&](float (&x)[NT][4], const float *mat, bool transposed, uint32_t vec) {
                if (transposed) frag_a_t(m, mat, MW, kb * 16, mt * 16, lane);
                else frag_a(m, mat, MW, mt * 16, kb * 16, lane);
#pragma unroll
                for (int nn = 0; nn < NT / 2; ++nn) {
                    uint32_t b[P][4];
#pragma unroll
                    for (int pl = 0; pl < P; ++pl) load_b_t(b[pl], vec + pl * L::kTile, kb * 16, c0 + nn * 16, lane);
                    mma_all<kApart>(x[2 * nn], x[2 * nn + 1], m, b);
                }
            };
            if (kb <= mt) {
                product(dq, da_f, false, k_s);
                if (DELTA) product(dr, dl_f, false, k_s);
            }
            if (kb >= mt) {
                product(di, da_f, true, q_s);
                if (DELTA) product(di, dl_f, true, k_s);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int i = mt * 16 + g + 8 * r, c = c0 + n * 8 + 2 * t;
                const float2 qv = value(q_s, i, c), kv = value(k_s, i, c);
                y[r] = fmaf(qv.x, dq[n][2 * r], fmaf(qv.y, dq[n][2 * r + 1], y[r]));
                y[r] = fmaf(kv.x, dr[n][2 * r] - di[n][2 * r], fmaf(kv.y, dr[n][2 * r + 1] - di[n][2 * r + 1], y[r]));
                const float own = diag[i];
                put(a.dq, a.dq_part, i, c, fmaf(own, kv.x, dq[n][2 * r]), fmaf(own, kv.y, dq[n][2 * r + 1]));
                put(a.dk, a.dk_part, i, c, fmaf(own, qv.x, dw[n][2 * r] + di[n][2 * r] + dr[n][2 * r]),
                    fmaf(own, qv.y, dw[n][2 * r + 1] + di[n][2 * r + 1] + dr[n][2 * r + 1]));
            }
        if (!a.dg) return;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            y[r] += __shfl_xor_sync(0xffffffffu, y[r], 1), b2[r] += __shfl_xor_sync(0xffffffffu, b2[r], 1);
            y[r] += __shfl_xor_sync(0xffffffffu, y[r], 2), b2[r] += __shfl_xor_sync(0xffffffffu, b2[r], 2);
            if (t == 0) {
                const int i = mt * 16 + g + 8 * r;
                rows[cq * kChunk + i] = y[r];
                rows[(4 + cq) * kChunk + i] = b2[r];
            }
        }
        __syncthreads();
        if (warp == 0) {
            float s = 0.f;
            for (int i = lane; i < 1024; i += 32) s += part[i];
            const float across = warp_sum(s) * expf(G[kChunk - 1].x + G[kChunk - 1].y);
            float yy[2] = {0.f, 0.f}, ww[2] = {0.f, 0.f};  // lane holds tokens 2 lane, 2 lane + 1
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int e = 0; e < 2; ++e) yy[e] += rows[x * kChunk + 2 * lane + e], ww[e] += rows[(4 + x) * kChunk + 2 * lane + e];
            float suf = yy[0] + yy[1], pre = ww[0] + ww[1];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const float u = __shfl_down_sync(0xffffffffu, suf, o), v = __shfl_up_sync(0xffffffffu, pre, o);
                if (lane + o < 32) suf += u;
                if (lane >= o) pre += v;
            }
            float after = __shfl_down_sync(0xffffffffu, suf, 1), before = __shfl_up_sync(0xffffffffu, pre, 1);
            if (lane == 31) after = 0.f;
            if (lane == 0) before = 0.f;
            const int i = 2 * lane;
            if (i < p.valid) a.dg[(size_t)(p.tok0 + i) * a.H + h] = across + before + (after + yy[1] + yy[0]);
            if (i + 1 < p.valid) a.dg[(size_t)(p.tok0 + i + 1) * a.H + h] = across + (before + ww[0]) + (after + yy[1]);
        }
    } else {
        // decayed vectors, and the decay factors in front of / behind a token inside its block; one (block, channel) per thread
        constexpr int kV = kChunk * SW;
        float *qs = reinterpret_cast<float *>(smem), *kc = qs + kV, *ps = kc + kV, *ss = ps + kV, *ks = ss + kV;
        float *front = reinterpret_cast<float *>(smem + L::tables), *back = front + 4 * DK, *eB = back + 4 * DK, *eI = eB + 4 * DK;
        const int blk = tid / DK, c = tid % DK;
        const bool mine = tid < 4 * DK;
        auto raw = [&](const void *src, int i, int ch) { return i < p.valid ? to_f32(static_cast<const IO *>(src)[((size_t)(p.tok0 + i) * a.Hq + hq) * DK + ch]) : 0.f; };
        auto gate_at = [&](int i, int ch) { return i < p.valid ? a.g[((size_t)(p.tok0 + i) * a.H + h) * DK + ch] : 0.f; };
        float Bc = 0.f, Ec = 1.f;  // sum of the gates, product of their exponentials (see block_vectors)
        if (mine) {
            float gate[kBlock], kk[kBlock], qq[kBlock];
#pragma unroll
            for (int r = 0; r < kBlock; ++r) gate[r] = gate_at(blk * kBlock + r, c), kk[r] = raw(a.k, blk * kBlock + r, c), qq[r] = raw(a.q, blk * kBlock + r, c);
#pragma unroll
            for (int r = 0; r < kBlock; ++r) {
                const int at = (blk * kBlock + r) * SW + c;
                if (EXCL) qs[at] = qq[r] * Ec, ps[at] = Ec;
                Bc += gate[r];
                gate[r] = expf(gate[r]);
                Ec *= gate[r];
                if (!EXCL) qs[at] = qq[r] * Ec, ps[at] = Ec;
                if (DELTA) ks[at] = kk[r] * Ec;
            }
            float e = 1.f;
#pragma unroll
            for (int r = kBlock - 1; r >= 0; --r) {
                const int at = (blk * kBlock + r) * SW + c;
                kc[at] = kk[r] * e, ss[at] = e;
                e *= gate[r];
            }
            if (!(Bc > -kBlockDecay)) deep[blk] = 1;
            eB[blk * DK + c] = Bc;
        }
        __syncthreads();
        if (mine) {
            float f = 0.f, b = 0.f;
            for (int m = 0; m < 4; ++m) {
                const float x = eB[m * DK + c];
                if (m < blk) f += x;
                if (m > blk) b += x;
            }
            front[blk * DK + c] = decay_exp(f), back[blk * DK + c] = decay_exp(b), eI[blk * DK + c] = 1.f / Ec;
        }
        __syncthreads();
        if (mine) eB[blk * DK + c] = decay_exp(Bc);
        __syncthreads();
        // sum over blocks J < mt (towards the front) or I > mt (towards the back) of a row block's pairs, the decay of the
        // blocks in between multiplied in by Horner's rule, then the block's own pairs
        float acc[NT][4] = {}, acc_l[NT][4] = {};
        auto times_block = [&](float (&x)[NT][4], int b) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float2 d = *reinterpret_cast<const float2 *>(eB + b * DK + c0 + n * 8 + 2 * t);
                x[n][0] *= d.x, x[n][1] *= d.y, x[n][2] *= d.x, x[n][3] *= d.y;
            }
        };
        // the 16 tokens of block b_ of a decayed vector as operand B; of the warp's own block times e^(-B)
        auto vector_frag = [&](uint32_t (&b)[kPlanes][4], const float *vec, int b_, int nn) {
            const int c = c0 + nn * 16 + g;
            const float f0 = b_ == mt ? eI[mt * DK + c] : 1.f, f1 = b_ == mt ? eI[mt * DK + c + 8] : 1.f;
            const float *at = vec + (b_ * 16 + 2 * t) * SW + c;
            frag_pair(b, 0, at[0] * f0, at[SW] * f0), frag_pair(b, 1, at[8 * SW] * f0, at[9 * SW] * f0);
            frag_pair(b, 2, at[8] * f1, at[SW + 8] * f1), frag_pair(b, 3, at[8 * SW + 8] * f1, at[9 * SW + 8] * f1);
        };
        const bool own_deep = deep[mt] != 0;
        const IO *q0 = static_cast<const IO *>(a.q) + ((size_t)p.tok0 * a.Hq + hq) * DK, *k0 = static_cast<const IO *>(a.k) + ((size_t)p.tok0 * a.Hq + hq) * DK;
        const float *g0 = a.g + ((size_t)p.tok0 * a.H + h) * DK;
        // dq, and dk as read: x <- sign e^G x + e^p (pairs inside the chunk), both over the same k
        for (int J = 0; J <= mt; ++J) {
            if (J == mt && own_deep) break;
            if (J && J < mt) {
                times_block(acc, J);
                if (DELTA) times_block(acc_l, J);
            }
            uint32_t m[kPlanes][4], l[kPlanes][4];
            frag_a(m, da_f, MW, mt * 16, J * 16, lane);
            if (DELTA) frag_a(l, dl_f, MW, mt * 16, J * 16, lane);
#pragma unroll
            for (int nn = 0; nn < NT / 2; ++nn) {
                uint32_t b[kPlanes][4];
                vector_frag(b, kc, J, nn);
                mma_all<kApart>(acc[2 * nn], acc[2 * nn + 1], m, b);
                if (DELTA) mma_all<kApart>(acc_l[2 * nn], acc_l[2 * nn + 1], l, b);
            }
        }
        auto finish_front = [&](float (&x)[NT][4], float (&in)[NT][4], const float *mat, float sign) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = mt * 16 + g + 8 * (e >> 1), ch = c0 + n * 8 + 2 * t + (e & 1);
                    x[n][e] = ps[i * SW + ch] * fmaf(sign * front[mt * DK + ch], x[n][e], in[n][e]);
                    if (own_deep) x[n][e] += pairs_front<IO, EXCL>(k0 + ch, a.Hq * DK, g0 + ch, a.H * DK, p.valid, mat, MW, i);
                    in[n][e] = 0.f;
                }
        };
        finish_front(dq, acc, da_f, a.scale);
        if (DELTA) finish_front(dr, acc_l, dl_f, -1.f);
        // dk as written: behind the chunk (dw), inside it (acc)
        for (int I = 3; I >= mt; --I) {
            if (I == mt && own_deep) break;
            if (I < 3 && I > mt) times_block(acc, I);
            uint32_t m[kPlanes][4], b[kPlanes][4];
            frag_a_t(m, da_f, MW, I * 16, mt * 16, lane);
#pragma unroll
            for (int nn = 0; nn < NT / 2; ++nn) {
                vector_frag(b, qs, I, nn);
                mma_all<kApart>(acc[2 * nn], acc[2 * nn + 1], m, b);
            }
            if (DELTA) {
                frag_a_t(m, dl_f, MW, I * 16, mt * 16, lane);
#pragma unroll
                for (int nn = 0; nn < NT / 2; ++nn) {
                    vector_frag(b, ks, I, nn);
                    mma_all<kApart>(acc[2 * nn], acc[2 * nn + 1], m, b);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int i = mt * 16 + g + 8 * r, ch = c0 + n * 8 + 2 * t;
                float2 qv = make_float2(0.f, 0.f), kv = qv, q_next = qv, k_prev = qv;
                if (i < p.valid) {
                    const size_t at = ((size_t)(p.tok0 + i) * a.Hq + hq) * DK + ch, row = (size_t)a.Hq * DK;
                    qv = load_pair<IO>(a.q, at), kv = load_pair<IO>(a.k, at);
                    if (EXCL && i > 0) k_prev = load_pair<IO>(a.k, at - row);
                    if (EXCL && i + 1 < p.valid) q_next = load_pair<IO>(a.q, at + row);
                }
                const float to_prev = EXCL && i > 0 ? near[i] : 0.f, from_next = EXCL && i + 1 < p.valid ? near[i + 1] : 0.f;
                float oq[2], ok[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int el = 2 * r + e;
                    const float es = ss[i * SW + ch + e];
                    float in = es * acc[n][el];
                    if (own_deep) in += pairs_back<IO, EXCL, DELTA>(q0 + ch + e, k0 + ch + e, a.Hq * DK, g0 + ch + e, a.H * DK, p.valid, da_f, dl_f, MW, i);
                    const float out = back[mt * DK + ch + e] * es * dw[n][el];
                    const float qe = e ? qv.y : qv.x, ke = e ? kv.y : kv.x;
                    // the readout of RWKV6 sees the decays in front of its token only: its term belongs to the token before
                    float y = ke * ((DELTA ? dr[n][el] : 0.f) - in);
                    if (!EXCL) y = fmaf(qe, dq[n][el], y);
                    ps[i * SW + ch + e] = y;
                    ss[i * SW + ch + e] = ke * out;
                    oq[e] = dq[n][el], ok[e] = out + in + (DELTA ? dr[n][el] : 0.f);
                    if (EXCL) dq[n][el] *= qe;
                    const float own = EXCL ? diag[i] * a.bonus[h * DK + ch + e] : diag[i];
                    oq[e] = fmaf(own, ke, oq[e]), ok[e] = fmaf(own, qe, ok[e]);
                    if (EXCL) oq[e] = fmaf(to_prev, e ? k_prev.y : k_prev.x, oq[e]), ok[e] = fmaf(from_next, e ? q_next.y : q_next.x, ok[e]);
                }
                put(a.dq, a.dq_part, i, ch, oq[0], oq[1]);
                put(a.dk, a.dk_part, i, ch, ok[0], ok[1]);
            }
        if (EXCL) {  // q dq goes one token up, now that every y stands
            __syncthreads();
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = mt * 16 + g + 8 * (e >> 1), ch = c0 + n * 8 + 2 * t + (e & 1);
                    if (i > 0) ps[(i - 1) * SW + ch] += dq[n][e];
                }
        }
        __syncthreads();
        // sums over the tokens of a block, then over the blocks (the tables' places are free, but for the chunk's decay)
        float *ysum = eI, *bsum = kc, *bonus_sum = kc + 4 * DK;
        if (mine) {
            float y = 0.f, b = 0.f, w = 0.f;
#pragma unroll
            for (int r = 0; r < kBlock; ++r) {
                const int i = blk * kBlock + r;
                y += ps[i * SW + c], b += ss[i * SW + c];
                if (EXCL) w = fmaf(diag[i], raw(a.q, i, c) * raw(a.k, i, c), w);
            }
            ysum[blk * DK + c] = y, bsum[blk * DK + c] = b;
            if (EXCL) bonus_sum[blk * DK + c] = w;
        }
        __syncthreads();
        if (mine) {
            float x = 0.f, y = 0.f;
            for (int i = 0; i < kGroups; ++i) x += part[i * DK + c];
            x *= front[3 * DK + c] * eB[3 * DK + c];  // e^(G_end)
            for (int m = 0; m < 4; ++m) {
                if (m < blk) x += bsum[m * DK + c];
                if (m > blk) y += ysum[m * DK + c];
            }
            float before[kBlock];  // <dS, S> and what comes from the tokens in front
#pragma unroll
            for (int r = 0; r < kBlock; ++r) before[r] = x, x += ss[(blk * kBlock + r) * SW + c];
#pragma unroll
            for (int r = kBlock - 1; r >= 0; --r) {
                const int i = blk * kBlock + r;
                y += ps[i * SW + c];
                if (i < p.valid) a.dg[((size_t)(p.tok0 + i) * a.H + h) * DK + c] = before[r] + y;
            }
            if (EXCL && blk == 0)
                a.dbonus_part[unit * DK + c] = (bonus_sum[c] + bonus_sum[DK + c]) + (bonus_sum[2 * DK + c] + bonus_sum[3 * DK + c]);
        }
    }
}

// dq, dk of heads that several value heads share: the sum over them, in order.
template <typename IO>
__global__ void __launch_bounds__(256) scan_group_sum_kernel(const ScanArgs a, int dk) {
    scan_kernel_begin();
    const int tokens = a.starts[a.n], rep = a.H / a.Hq, upr = dk / 4;
    const size_t total = (size_t)tokens * a.Hq * upr;
    for (size_t i = blockIdx.x * 256ull + threadIdx.x; i < total; i += gridDim.x * 256ull) {
        const size_t row = i / upr;
        const int c = (int)(i % upr) * 4;
        const size_t src = row * rep * dk + c;  // heads of a group are neighbours
        float4 sq = make_float4(0.f, 0.f, 0.f, 0.f), sk = sq;
        for (int r = 0; r < rep; ++r) {
            const float4 x = *reinterpret_cast<const float4 *>(a.dq_part + src + (size_t)r * dk);
            const float4 y = *reinterpret_cast<const float4 *>(a.dk_part + src + (size_t)r * dk);
            sq.x += x.x, sq.y += x.y, sq.z += x.z, sq.w += x.w;
            sk.x += y.x, sk.y += y.y, sk.z += y.z, sk.w += y.w;
        }
        base_store4<IO>(static_cast<IO *>(a.dq) + row * dk + c, sq);
        base_store4<IO>(static_cast<IO *>(a.dk) + row * dk + c, sk);
    }
}

// Bonus gradient: the chunks' parts summed in order, one CTA per head.
__global__ void __launch_bounds__(256) scan_bonus_sum_kernel(const ScanArgs a, int dk, float *dbonus) {
    scan_kernel_begin();
    __shared__ float s[256];
    const int h = blockIdx.x, c = threadIdx.x % dk, lane = threadIdx.x / dk, lanes = 256 / dk;
    const int chunks = a.chunk_starts[a.n];
    float x = 0.f;
    for (int i = lane; i < chunks; i += lanes) x += a.dbonus_part[((size_t)i * a.H + h) * dk + c];
    s[threadIdx.x] = x;
    __syncthreads();
    if (lane == 0) {
        for (int l = 1; l < lanes; ++l) x += s[l * dk + c];
        dbonus[(size_t)h * dk + c] = x;
    }
}

// Gradient rows behind the last sequence are zero.
__global__ void __launch_bounds__(256) scan_tail_kernel(const ScanArgs a, int rows, int qk_bytes, int v_bytes, int g_bytes, int beta_bytes) {
    scan_kernel_begin();
    const int first = a.starts[a.n];
    auto clear = [&](void *p, int row_bytes) {
        if (!p || !row_bytes) return;
        uint32_t *d = reinterpret_cast<uint32_t *>(static_cast<char *>(p) + (size_t)first * row_bytes);
        const size_t words = (size_t)(rows - first) * row_bytes / 4;
        for (size_t i = blockIdx.x * 256ull + threadIdx.x; i < words; i += gridDim.x * 256ull) d[i] = 0;
    };
    if (first >= rows) return;
    clear(a.dq, qk_bytes), clear(a.dk, qk_bytes), clear(a.dv_out, v_bytes), clear(a.dg, g_bytes), clear(a.dbeta, beta_bytes);
}

}  // namespace deltalog
