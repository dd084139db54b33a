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
// 256 threads; warp w owns token rows 16 (w & 3) .. + 15 and the channel half w >> 2 of every [64 x d_k] result.  fp32
// operands stay fp32 in shared memory (two bytes per element less than three planes, and both orientations from one
// tile); a warp forms its fragments' planes as it reads them.
#pragma once

#include "scan_common.cuh"
#include "scan_prep_kernel.cuh"

namespace deltalog {

// ---- fragments of fp32 tiles in shared memory ---------------------------------------------------------------
// A pair of values into place r of N planes.
template <int N>
__device__ __forceinline__ void frag_pair(uint32_t (&f)[N][4], int r, float x, float y) {
    uint32_t w[N];
    split_pair<N>(x, y, w);
#pragma unroll
    for (int p = 0; p < N; ++p) f[p][r] = w[p];
}
// Operand A (m16 x k16) of a tile [m][k] of rows of `w` floats (w = 8 mod 32: no bank conflicts) ...
__device__ __forceinline__ void frag_a(uint32_t (&f)[kPlanes][4], const float *tile, int w, int m0, int k0, int lane) {
    const float *p = tile + (m0 + (lane >> 2)) * w + k0 + 2 * (lane & 3);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float2 x = *reinterpret_cast<const float2 *>(p + (r & 1) * 8 * w + (r >> 1) * 8);
        frag_pair(f, r, x.x, x.y);
    }
}
// ... and of a tile [k][m].
__device__ __forceinline__ void frag_a_t(uint32_t (&f)[kPlanes][4], const float *tile, int w, int k0, int m0, int lane) {
    const float *p = tile + (k0 + 2 * (lane & 3)) * w + m0 + (lane >> 2);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float *q = p + (r >> 1) * 8 * w + (r & 1) * 8;
        frag_pair(f, r, q[0], q[w]);
    }
}
// Operand B (k16 x n16) of a tile [n][k] ...
__device__ __forceinline__ void frag_b(uint32_t (&f)[kPlanes][4], const float *tile, int w, int n0, int k0, int lane) {
    const float *p = tile + (n0 + (lane >> 2)) * w + k0 + 2 * (lane & 3);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float2 x = *reinterpret_cast<const float2 *>(p + (r >> 1) * 8 * w + (r & 1) * 8);
        frag_pair(f, r, x.x, x.y);
    }
}
// ... and of a tile [k][n] (w = 4 mod 16: no bank conflicts).
__device__ __forceinline__ void frag_b_t(uint32_t (&f)[kPlanes][4], const float *tile, int w, int k0, int n0, int lane) {
    const float *p = tile + (k0 + 2 * (lane & 3)) * w + n0 + (lane >> 2);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float *q = p + (r & 1) * 8 * w + (r >> 1) * 8;
        frag_pair(f, r, q[0], q[w]);
    }
}
// fp32 tile of rows `stride` elements apart to padded rows of `w` floats; rows at and behind `valid` become zeros.
__device__ __forceinline__ void load_f32(float *dst, const float *src, size_t stride, int rows, int cols, int w, int valid, int tid) {
    const int upr = cols >> 2, sh = cols == 128 ? 5 : 4;
    for (int i = tid; i < rows * upr; i += 256) {
        const int row = i >> sh, unit = i & (upr - 1);
        const bool ok = row < valid;
        cp_async16_zfill(smem_addr(dst + row * w + unit * 4), src + (ok ? (size_t)row * stride + unit * 4 : 0), ok);
    }
}
// The token rows of an io tensor that is an operand of this kernel: bf16 as it is (swizzled), fp32 padded.
__device__ __forceinline__ void load_io(unsigned char *dst, const __nv_bfloat16 *src, size_t stride, int dv, int valid, int tid) {
    load_tile(smem_addr(dst), src, stride, kChunk, dv, valid, tid, 256);
}
__device__ __forceinline__ void load_io(unsigned char *dst, const float *src, size_t stride, int dv, int valid, int tid) {
    load_f32(reinterpret_cast<float *>(dst), src, stride, kChunk, dv, dv + 8, valid, tid);
}
__device__ __forceinline__ void io_frag_a(uint32_t (&f)[1][4], const unsigned char *tile, int dv, int m0, int k0, int lane) {
    load_a(f[0], smem_addr(tile), dv, m0, k0, lane);
}
__device__ __forceinline__ void io_frag_a(uint32_t (&f)[kPlanes][4], const unsigned char *tile, int dv, int m0, int k0, int lane) {
    frag_a(f, reinterpret_cast<const float *>(tile), dv + 8, m0, k0, lane);
}
__device__ __forceinline__ void io_frag_b(uint32_t (&f)[1][4], const unsigned char *tile, int dv, int n0, int k0, int lane) {
    load_b(f[0], smem_addr(tile), dv, n0, k0, lane);
}
__device__ __forceinline__ void io_frag_b(uint32_t (&f)[kPlanes][4], const unsigned char *tile, int dv, int n0, int k0, int lane) {
    frag_b(f, reinterpret_cast<const float *>(tile), dv + 8, n0, k0, lane);
}
// c0, c1 += a b over all plane products that count.
template <int PA, int PB>
__device__ __forceinline__ void mma_all(float (&c0)[4], float (&c1)[4], const uint32_t (&a)[PA][4], const uint32_t (&b)[PB][4]) {
#pragma unroll
    for (int pb = 0; pb < PB; ++pb) mma_planes<PA, kPlanes>(c0, c1, a, b[pb], pb);
}

template <int OP, int P, int DK, typename IO>
struct GradSmem {
    static constexpr bool VEC = OpTraits<OP>::kVecDecay, DELTA = OpTraits<OP>::kDeltaRule;
    static constexpr int kTile = kChunk * DK * 2;
    static constexpr int kSW = DK + 4;              // row of a state tile or of a decayed vector
    static constexpr int kMW = kChunk + 8;          // row of dA, dL'
    static constexpr int kMat = kChunk * kMW * 4;
    // last phase: q and k planes, or the three decayed vectors and two more fp32 tiles
    static constexpr int last = VEC ? (DELTA ? 5 : 4) * kChunk * kSW * 4 : 2 * P * kTile;
    __host__ __device__ static constexpr int f32_tile(int dv) { return kChunk * (dv + 8) * 4; }
    __host__ __device__ static constexpr int io_tile(int dv) { return sizeof(IO) == 4 ? f32_tile(dv) : kChunk * dv * 2; }
    __host__ __device__ static constexpr int u_tile(int dv) { return DELTA ? f32_tile(dv) : io_tile(dv); }
    __host__ __device__ static constexpr int dout(int dv) { return dv * kSW * 4; }   // behind the state tile
    __host__ __device__ static constexpr int mats(int dv) {
        const int first = dout(dv) + io_tile(dv) + u_tile(dv) + (DELTA ? f32_tile(dv) : 0);
        return first > last ? first : last;
    }
    __host__ __device__ static constexpr int small(int dv) { return mats(dv) + (DELTA ? 2 : 1) * kMat; }
    static constexpr int kSmall = 8 * DK * 4       // partial sums of <dS, S>
                                  + 4 * kChunk * 4 // row sums
                                  + 4 * DK * 4     // block decays
                                  + 2 * kChunk * 4 // beta, diagonal of dA
                                  + kChunk * 8     // G
                                  + 16;
    static constexpr size_t bytes(int dv) { return small(dv) + kSmall; }
};

// A pair of neighbouring channels of the io tensors' row.
template <typename IO>
__device__ __forceinline__ float2 load_pair(const void *src, size_t at) {
    float x[2];
    load_vec<IO, 2>(static_cast<const IO *>(src) + at, x);
    return make_float2(x[0], x[1]);
}

template <int OP, int P, int DK, typename IO>
__global__ void __launch_bounds__(256, 1) scan_grad_kernel(const ScanArgs a) {
    using L = GradSmem<OP, P, DK, IO>;
    constexpr bool VEC = L::VEC, DELTA = L::DELTA, EXCL = OpTraits<OP>::kBonus;
    constexpr int NT = DK / 16, SW = L::kSW, MW = L::kMW;
    constexpr int IP = sizeof(IO) == 4 ? kPlanes : 1;  // planes of dO and of v
    extern __shared__ __align__(128) unsigned char smem[];
    const uint32_t sm = smem_addr(smem);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, chunk = blockIdx.x, h = blockIdx.y;
    const int g = lane >> 2, t = lane & 3, mt = warp & 3, c0 = (warp >> 2) * (DK / 2);
    ChunkPlace p;
    if (!chunk_place(a, chunk, p)) return;
    const int dv = a.dv, hq = h / (a.H / a.Hq);
    const size_t unit = (size_t)chunk * a.H + h, tile = (size_t)DK * dv;
    float *st = reinterpret_cast<float *>(smem);
    unsigned char *do_t = smem + L::dout(dv), *u_t = do_t + L::io_tile(dv);
    const float *u_f = reinterpret_cast<const float *>(u_t);            // delta rule: U and dV, fp32
    float *dv_f = reinterpret_cast<float *>(u_t + L::u_tile(dv));
    float *da_f = reinterpret_cast<float *>(smem + L::mats(dv)), *dl_f = da_f + kChunk * MW;
    float *part = reinterpret_cast<float *>(smem + L::small(dv));  // [8][DK]
    float *rows = part + 8 * DK;                                  // [4][64]: y and b of the two channel halves
    float *B = rows + 4 * kChunk;                                 // [4][DK]
    float *beta = B + 4 * DK, *diag = beta + kChunk;
    float *near = beta;  // RWKV6 (no beta): dA's entries next to the diagonal
    double *G = reinterpret_cast<double *>(diag + kChunk);
    int *deep = reinterpret_cast<int *>(G + kChunk);

    // S_0, dO, U, dV
    load_f32(st, a.S + unit * tile, DK, dv, DK, SW, dv, tid);
    const size_t v_off = ((size_t)p.tok0 * a.H + h) * dv;
    load_io(do_t, static_cast<const IO *>(a.dout) + v_off, (size_t)a.H * dv, dv, p.valid, tid);
    if (DELTA) {
        load_f32(reinterpret_cast<float *>(u_t), a.U + unit * kChunk * dv, dv, kChunk, dv, dv + 8, kChunk, tid);
        load_f32(dv_f, a.dV + unit * kChunk * dv, dv, kChunk, dv, dv + 8, kChunk, tid);
    } else {
        load_io(u_t, static_cast<const IO *>(a.v) + v_off, (size_t)a.H * dv, dv, p.valid, tid);
    }
    cp_async_commit();
    if (tid < 4) deep[tid] = 0;
    if (!VEC && warp == 0) chunk_decay_sums(a, p, h, G, lane);
    if (DELTA && tid >= 64 && tid < 128) beta[tid - 64] = scan_beta(tid - 64 < p.valid ? a.beta[(size_t)(p.tok0 + tid - 64) * a.H + h] : 0.f);
    cp_async_wait_all();
    __syncthreads();

    // dO S_0^T and dV S_0^T
    float dq[NT][4] = {}, dr[NT][4] = {}, dw[NT][4] = {};
    for (int k0 = 0; k0 < dv; k0 += 16) {
        uint32_t f[IP][4], e[kPlanes][4];
        io_frag_a(f, do_t, dv, mt * 16, k0, lane);
        if (DELTA) frag_a(e, dv_f, dv + 8, mt * 16, k0, lane);
#pragma unroll
        for (int nn = 0; nn < NT / 2; ++nn) {
            uint32_t b[kPlanes][4];
            frag_b_t(b, st, SW, k0, c0 + nn * 16, lane);
            mma_all(dq[2 * nn], dq[2 * nn + 1], f, b);
            if (DELTA) mma_all(dr[2 * nn], dr[2 * nn + 1], e, b);
        }
    }
    // <dS_1, S_0> by channel
    {
        constexpr int kPairs = DK / 2, kGroups = 256 / kPairs;
        const int cp = tid % kPairs, grp = tid / kPairs;
        float s0 = 0.f, s1 = 0.f;
        const float *src = a.dS + unit * tile + cp * 2;
        for (int v = grp; v < dv; v += kGroups) {
            const float2 d = *reinterpret_cast<const float2 *>(src + (size_t)v * DK), x = *reinterpret_cast<const float2 *>(st + v * SW + cp * 2);
            s0 = fmaf(d.x, x.x, s0), s1 = fmaf(d.y, x.y, s1);
        }
        part[grp * DK + cp * 2] = s0, part[grp * DK + cp * 2 + 1] = s1;
    }
    __syncthreads();
    load_f32(st, a.dS + unit * tile, DK, dv, DK, SW, dv, tid);
    cp_async_commit();
    // dbeta: four threads per token
    if (DELTA) {
        const int i = tid >> 2, qd = tid & 3;
        const float rb = 1.f / beta[i];
        float s = 0.f;
        for (int v = qd * 2; v < dv; v += 8) {
            const float2 u = *reinterpret_cast<const float2 *>(u_f + i * (dv + 8) + v), d = *reinterpret_cast<const float2 *>(dv_f + i * (dv + 8) + v);
            s = fmaf(u.x * rb, d.x * rb, s), s = fmaf(u.y * rb, d.y * rb, s);
        }
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        s += __shfl_xor_sync(0xffffffffu, s, 2);
        if (qd == 0 && i < p.valid) a.dbeta[(size_t)(p.tok0 + i) * a.H + h] = s;
    }
    // dA and dL', masked; scalar decay multiplies e^(G_i - G_j) in here
    {
        const int j0 = (warp >> 2) * 32;
        float da[4][4] = {}, dl[4][4] = {};
        if (j0 <= mt * 16 + 15) {
            for (int k0 = 0; k0 < dv; k0 += 16) {
                uint32_t f[IP][4], e[kPlanes][4];
                io_frag_a(f, do_t, dv, mt * 16, k0, lane);
                if (DELTA) frag_a(e, dv_f, dv + 8, mt * 16, k0, lane);
#pragma unroll
                for (int nn = 0; nn < 2; ++nn) {
                    if constexpr (DELTA) {
                        uint32_t b[kPlanes][4];
                        frag_b(b, u_f, dv + 8, j0 + nn * 16, k0, lane);
                        mma_all(da[2 * nn], da[2 * nn + 1], f, b);
                        mma_all(dl[2 * nn], dl[2 * nn + 1], e, b);
                    } else {
                        uint32_t b[IP][4];
                        io_frag_b(b, u_t, dv, j0 + nn * 16, k0, lane);
                        mma_all(da[2 * nn], da[2 * nn + 1], f, b);
                    }
                }
            }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int i = mt * 16 + g + 8 * half, j = j0 + n * 8 + 2 * t;
                float x[2], y[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float m = VEC ? 1.f : (j + e <= i ? expf((float)(G[i] - G[j + e])) : 0.f);
                    const float raw = da[n][2 * half + e];
                    if (i == j + e) diag[i] = raw * a.scale;
                    if (EXCL && i == j + e + 1) near[i] = raw;
                    x[e] = j + e + (EXCL ? 1 : 0) < i ? raw * m * a.scale : 0.f;
                    y[e] = j + e < i ? -dl[n][2 * half + e] * m : 0.f;
                }
                *reinterpret_cast<float2 *>(da_f + i * MW + j) = make_float2(x[0], x[1]);
                if (DELTA) *reinterpret_cast<float2 *>(dl_f + i * MW + j) = make_float2(y[0], y[1]);
            }
    }
    cp_async_wait_all();
    __syncthreads();
    // U dS_1^T
    for (int k0 = 0; k0 < dv; k0 += 16) {
        constexpr int UP = DELTA ? kPlanes : IP;
        uint32_t f[UP][4];
        if constexpr (DELTA) frag_a(f, u_f, dv + 8, mt * 16, k0, lane);
        else io_frag_a(f, u_t, dv, mt * 16, k0, lane);
#pragma unroll
        for (int nn = 0; nn < NT / 2; ++nn) {
            uint32_t b[kPlanes][4];
            frag_b_t(b, st, SW, k0, c0 + nn * 16, lane);
            mma_all(dw[2 * nn], dw[2 * nn + 1], f, b);
        }
    }
    __syncthreads();  // state tile, dO, U, dV are done with

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
        const uint32_t q_s = sm, k_s = sm + P * L::kTile;
        const size_t off = ((size_t)p.tok0 * a.Hq + hq) * DK;
#pragma unroll
        for (int pl = 0; pl < P; ++pl) {
            load_tile(q_s + pl * L::kTile, a.qp + pl * a.q_plane + off, (size_t)a.Hq * DK, kChunk, DK, p.valid, tid, 256);
            load_tile(k_s + pl * L::kTile, a.kp + pl * a.q_plane + off, (size_t)a.Hq * DK, kChunk, DK, p.valid, tid, 256);
        }
        cp_async_commit();
        float front[2], back[2];  // e^G and e^(G_end - G) of rows g, g + 8
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int i = mt * 16 + g + 8 * r;
            front[r] = expf((float)G[i]), back[r] = expf((float)(G[kChunk - 1] - G[i]));
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                dq[n][e] *= a.scale * front[e >> 1];
                dr[n][e] *= -front[e >> 1];
                dw[n][e] *= back[e >> 1];
            }
        cp_async_wait_all();
        __syncthreads();
        float y[2] = {0.f, 0.f}, b2[2] = {0.f, 0.f};
        auto value = [&](uint32_t base, int i, int c) {
            const unsigned char *at = smem + (base - sm) + i * DK * 2 + (((c >> 3) ^ (i & 7)) << 4) + (c & 7) * 2;
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
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float2 kv = value(k_s, mt * 16 + g + 8 * r, c0 + n * 8 + 2 * t);
                b2[r] = fmaf(kv.x, dw[n][2 * r], fmaf(kv.y, dw[n][2 * r + 1], b2[r]));
            }
        // inside the chunk: dq += dA K, dk as written += dA^T Q + dL'^T K, dk as read += dL' K
        float di[NT][4] = {};
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            uint32_t am[kPlanes][4], lm[kPlanes][4];
            if (kb <= mt) {
                frag_a(am, da_f, MW, mt * 16, kb * 16, lane);
                if (DELTA) frag_a(lm, dl_f, MW, mt * 16, kb * 16, lane);
#pragma unroll
                for (int nn = 0; nn < NT / 2; ++nn)
#pragma unroll
                    for (int pl = 0; pl < P; ++pl) {
                        uint32_t b[4];
                        load_b_t(b, k_s + pl * L::kTile, DK, kb * 16, c0 + nn * 16, lane);
                        mma_planes<kPlanes, kPlanes>(dq[2 * nn], dq[2 * nn + 1], am, b, pl);
                        if (DELTA) mma_planes<kPlanes, kPlanes>(dr[2 * nn], dr[2 * nn + 1], lm, b, pl);
                    }
            }
            if (kb >= mt) {
                frag_a_t(am, da_f, MW, kb * 16, mt * 16, lane);
                if (DELTA) frag_a_t(lm, dl_f, MW, kb * 16, mt * 16, lane);
#pragma unroll
                for (int nn = 0; nn < NT / 2; ++nn)
#pragma unroll
                    for (int pl = 0; pl < P; ++pl) {
                        uint32_t b[4];
                        load_b_t(b, q_s + pl * L::kTile, DK, kb * 16, c0 + nn * 16, lane);
                        mma_planes<kPlanes, kPlanes>(di[2 * nn], di[2 * nn + 1], am, b, pl);
                        if (DELTA) {
                            load_b_t(b, k_s + pl * L::kTile, DK, kb * 16, c0 + nn * 16, lane);
                            mma_planes<kPlanes, kPlanes>(di[2 * nn], di[2 * nn + 1], lm, b, pl);
                        }
                    }
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
                rows[(warp >> 2) * kChunk + i] = y[r];
                rows[(2 + (warp >> 2)) * kChunk + i] = b2[r];
            }
        }
        __syncthreads();
        if (warp == 0) {
            float s = 0.f;
            for (int i = lane; i < (256 / (DK / 2)) * DK; i += 32) s += part[i];
            const float across = warp_sum(s) * expf((float)G[kChunk - 1]);
            // lane holds tokens 2 lane, 2 lane + 1
            const float y0 = rows[2 * lane] + rows[kChunk + 2 * lane], y1 = rows[2 * lane + 1] + rows[kChunk + 2 * lane + 1];
            const float w0 = rows[2 * kChunk + 2 * lane] + rows[3 * kChunk + 2 * lane];
            const float w1 = rows[2 * kChunk + 2 * lane + 1] + rows[3 * kChunk + 2 * lane + 1];
            float suf = y0 + y1, pre = w0 + w1;
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
            if (i < p.valid) a.dg[(size_t)(p.tok0 + i) * a.H + h] = across + before + (after + y1 + y0);
            if (i + 1 < p.valid) a.dg[(size_t)(p.tok0 + i + 1) * a.H + h] = across + (before + w0) + (after + y1);
        }
    } else {
        // decayed vectors, and the decay in front of / behind a token inside its block
        constexpr int kV = kChunk * SW;
        float *qs = st, *kc = qs + kV, *ps = kc + kV, *ss = ps + kV, *ks = ss + kV;
        for (int w = tid; w < 4 * DK; w += 256) {
            const int blk = w / DK, c = w % DK;
            BlockVectors<IO> o;
            block_vectors<IO, EXCL>(a, p, h, hq, DK, blk, c, true, o);
            B[blk * DK + c] = o.B;
            if (!(o.B > -kBlockDecay)) deep[blk] = 1;
            float pre = 0.f, suf = 0.f;
#pragma unroll
            for (int r = 0; r < kBlock; ++r) {
                const int i = blk * kBlock + r;
                const float gate = i < p.valid ? a.g[((size_t)(p.tok0 + i) * a.H + h) * DK + c] : 0.f;
                if (EXCL) ps[i * SW + c] = pre;
                pre += gate;
                if (!EXCL) ps[i * SW + c] = pre;
                qs[i * SW + c] = o.qs[r];
                kc[i * SW + c] = o.kc[r];
                if (DELTA) ks[i * SW + c] = o.ks[r];
            }
#pragma unroll
            for (int r = kBlock - 1; r >= 0; --r) {
                const int i = blk * kBlock + r;
                ss[i * SW + c] = suf;
                suf += i < p.valid ? a.g[((size_t)(p.tok0 + i) * a.H + h) * DK + c] : 0.f;
            }
        }
        __syncthreads();
        float acc[NT][4], dia[NT][4];
        // sum over blocks J < mt (towards the front) or I > mt (towards the back) of a row block's pairs, the decay of the
        // blocks in between multiplied in by Horner's rule, then the block's own pairs
        auto zero = [&](float (&x)[NT][4]) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) x[n][e] = 0.f;
        };
        auto times_block = [&](float (&x)[NT][4], int blk, float sign) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float2 d = *reinterpret_cast<const float2 *>(B + blk * DK + c0 + n * 8 + 2 * t);
                const float e0 = expf(sign * d.x), e1 = expf(sign * d.y);
                x[n][0] *= e0, x[n][1] *= e1, x[n][2] *= e0, x[n][3] *= e1;
            }
        };
        auto product = [&](float (&x)[NT][4], const float *mat, bool transposed, int blk, const float *vec) {
            uint32_t m[kPlanes][4];
            if (transposed) frag_a_t(m, mat, MW, blk * 16, mt * 16, lane);
            else frag_a(m, mat, MW, mt * 16, blk * 16, lane);
#pragma unroll
            for (int nn = 0; nn < NT / 2; ++nn) {
                uint32_t b[kPlanes][4];
                frag_b_t(b, vec, SW, blk * 16, c0 + nn * 16, lane);
                mma_all(x[2 * nn], x[2 * nn + 1], m, b);
            }
        };
        // a strongly decaying block's own pairs, one by one: for element (i, c) the sum over j of mat[i][j] x_jc e^(..),
        // or (transposed) over the later rows
        auto raw = [&](const void *src, int i, int c) { return i < p.valid ? to_f32(static_cast<const IO *>(src)[((size_t)(p.tok0 + i) * a.Hq + hq) * DK + c]) : 0.f; };
        auto gate_at = [&](int i, int c) { return i < p.valid ? a.g[((size_t)(p.tok0 + i) * a.H + h) * DK + c] : 0.f; };
        auto pairs_front = [&](const float *mat, int i, int c) {  // sum_(j <= i) mat_ij k_jc e^(G_i - G_j)
            float s = 0.f, x = 0.f;
            for (int j = i; j >= mt * 16; --j) {
                if (j < i && !(EXCL && j + 1 == i)) x += gate_at(j + 1, c);
                s = fmaf(mat[i * MW + j] * raw(a.k, j, c), expf(x), s);
            }
            return s;
        };
        auto pairs_back = [&](int j, int c) {  // sum_(i >= j) (dA_ij q_ic + dL'_ij k_ic) e^(G_i - G_j)
            float s = 0.f, x = 0.f;
            for (int i = j; i < mt * 16 + 16; ++i) {
                if (i > j && !EXCL) x += gate_at(i, c);
                if (EXCL && i > j + 1) x += gate_at(i - 1, c);
                float w = da_f[i * MW + j] * raw(a.q, i, c);
                if (DELTA) w = fmaf(dl_f[i * MW + j], raw(a.k, i, c), w);
                s = fmaf(w, expf(x), s);
            }
            return s;
        };
        const bool own_deep = deep[mt] != 0;
        auto chunk_front = [&](int c) {
            float s = 0.f;
            for (int m = 0; m < mt; ++m) s += B[m * DK + c];
            return s;
        };
        auto chunk_back = [&](int c) {
            float s = 0.f;
            for (int m = mt + 1; m < 4; ++m) s += B[m * DK + c];
            return s;
        };
        // dq
        zero(acc), zero(dia);
        for (int J = 0; J < mt; ++J) {
            if (J) times_block(acc, J, 1.f);
            product(acc, da_f, false, J, kc);
        }
        if (!own_deep) product(dia, da_f, false, mt, kc), times_block(dia, mt, -1.f);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = mt * 16 + g + 8 * (e >> 1), c = c0 + n * 8 + 2 * t + (e & 1);
                const float ep = expf(ps[i * SW + c]);
                float x = fmaf(expf(chunk_front(c)) * ep * a.scale, dq[n][e], ep * (acc[n][e] + dia[n][e]));
                if (own_deep) x += pairs_front(da_f, i, c);
                dq[n][e] = x;
            }
        // dk as read
        if (DELTA) {
            zero(acc), zero(dia);
            for (int J = 0; J < mt; ++J) {
                if (J) times_block(acc, J, 1.f);
                product(acc, dl_f, false, J, kc);
            }
            if (!own_deep) product(dia, dl_f, false, mt, kc), times_block(dia, mt, -1.f);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = mt * 16 + g + 8 * (e >> 1), c = c0 + n * 8 + 2 * t + (e & 1);
                    const float ep = expf(ps[i * SW + c]);
                    float x = fmaf(-expf(chunk_front(c)) * ep, dr[n][e], ep * (acc[n][e] + dia[n][e]));
                    if (own_deep) x += pairs_front(dl_f, i, c);
                    dr[n][e] = x;
                }
        }
        // dk as written: behind the chunk (dw), inside it (acc)
        zero(acc), zero(dia);
        for (int I = 3; I > mt; --I) {
            if (I < 3) times_block(acc, I, 1.f);
            product(acc, da_f, true, I, qs);
            if (DELTA) product(acc, dl_f, true, I, ks);
        }
        if (!own_deep) {
            product(dia, da_f, true, mt, qs);
            if (DELTA) product(dia, dl_f, true, mt, ks);
            times_block(dia, mt, -1.f);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int i = mt * 16 + g + 8 * r, c = c0 + n * 8 + 2 * t;
                float2 qv = make_float2(0.f, 0.f), kv = qv, q_next = qv, k_prev = qv;
                if (i < p.valid) {
                    const size_t at = ((size_t)(p.tok0 + i) * a.Hq + hq) * DK + c, row = (size_t)a.Hq * DK;
                    qv = load_pair<IO>(a.q, at), kv = load_pair<IO>(a.k, at);
                    if (EXCL && i > 0) k_prev = load_pair<IO>(a.k, at - row);
                    if (EXCL && i + 1 < p.valid) q_next = load_pair<IO>(a.q, at + row);
                }
                const float to_prev = EXCL && i > 0 ? near[i] : 0.f, from_next = EXCL && i + 1 < p.valid ? near[i + 1] : 0.f;
                float oq[2], ok[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int el = 2 * r + e;
                    const float es = expf(ss[i * SW + c + e]);
                    float in = es * (acc[n][el] + dia[n][el]);
                    if (own_deep) in += pairs_back(i, c + e);
                    const float out = expf(chunk_back(c + e)) * es * dw[n][el];
                    const float qe = e ? qv.y : qv.x, ke = e ? kv.y : kv.x;
                    // the readout of RWKV6 sees the decays in front of its token only: its term belongs to the token before
                    float y = ke * ((DELTA ? dr[n][el] : 0.f) - in);
                    if (!EXCL) y = fmaf(qe, dq[n][el], y);
                    ps[i * SW + c + e] = y;
                    ss[i * SW + c + e] = ke * out;
                    oq[e] = dq[n][el], ok[e] = out + in + (DELTA ? dr[n][el] : 0.f);
                    if (EXCL) dq[n][el] *= qe;
                    const float own = EXCL ? diag[i] * a.bonus[h * DK + c + e] : diag[i];
                    oq[e] = fmaf(own, ke, oq[e]), ok[e] = fmaf(own, qe, ok[e]);
                    if (EXCL) oq[e] = fmaf(to_prev, e ? k_prev.y : k_prev.x, oq[e]), ok[e] = fmaf(from_next, e ? q_next.y : q_next.x, ok[e]);
                }
                put(a.dq, a.dq_part, i, c, oq[0], oq[1]);
                put(a.dk, a.dk_part, i, c, ok[0], ok[1]);
            }
        if (EXCL) {  // q dq goes one token up, now that every y stands
            __syncthreads();
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = mt * 16 + g + 8 * (e >> 1), c = c0 + n * 8 + 2 * t + (e & 1);
                    if (i > 0) ps[(i - 1) * SW + c] += dq[n][e];
                }
        }
        __syncthreads();
        if (tid < DK) {
            const int c = tid;
            float x = 0.f, db = 0.f;
            for (int i = 0; i < 256 / (DK / 2); ++i) x += part[i * DK + c];
            x *= expf(B[c] + B[DK + c] + B[2 * DK + c] + B[3 * DK + c]);
            for (int i = 0; i < p.valid; ++i) {  // <dS, S> and what comes from the tokens in front, into ss
                const float w = ss[i * SW + c];
                ss[i * SW + c] = x;
                x += w;
            }
            float y = 0.f;
            for (int i = kChunk - 1; i >= 0; --i) {
                y += ps[i * SW + c];
                if (i < p.valid) a.dg[((size_t)(p.tok0 + i) * a.H + h) * DK + c] = ss[i * SW + c] + y;
            }
            if (EXCL) {
                for (int i = 0; i < p.valid; ++i) {
                    const size_t at = ((size_t)(p.tok0 + i) * a.Hq + hq) * DK + c;
                    db = fmaf(diag[i], to_f32(static_cast<const IO *>(a.q)[at]) * to_f32(static_cast<const IO *>(a.k)[at]), db);
                }
                a.dbonus_part[unit * DK + c] = db;
            }
        }
    }
}

// dq, dk of heads that several value heads share: the sum over them, in order.
template <typename IO>
__global__ void __launch_bounds__(256) scan_group_sum_kernel(const ScanArgs a, int dk) {
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
