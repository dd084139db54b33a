// What the chunks of a scan need before the chain over the states can run, one CTA per (chunk, head): the
// in-chunk matrix A, for the delta rule the triangular inverse T = (I + L)^-1 diag(beta), and the decay factors.
#pragma once

#include "scan_common.cuh"

namespace deltalog {

// The delta rule divides by beta in one place of the backward pass (E = U / beta); a beta of zero stands in as
// 1e-30, which changes U by 1e-30 E, far below the rounding of anything it is added to.
__device__ __forceinline__ float scan_beta(float b) { return fabsf(b) < 1e-30f ? copysignf(1e-30f, b) : b; }

struct ChunkPlace {
    int seq, tok0, valid;
};
// Sequence, first token and token count of a chunk; false for entries behind the last chunk and skipped rows.
__device__ __forceinline__ bool chunk_place(const ScanArgs &a, int chunk, ChunkPlace &p) {
    if (chunk >= a.max_chunks) return false;
    p.seq = a.chunk_seq[chunk];
    if (p.seq < 0) return false;
    if (a.slots) {
        const int s = a.slots[p.seq];
        if (s < 0 || s >= a.num_slots) return false;
    }
    p.tok0 = a.starts[p.seq] + (chunk - a.chunk_starts[p.seq]) * kChunk;
    p.valid = min(kChunk, a.starts[p.seq + 1] - p.tok0);
    return true;
}

constexpr int kInvStride = 65;

// T = (I + N)^-1 for the strictly lower N (64 x 64, fp32): the four diagonal 16 x 16 blocks by forward substitution,
// one column per thread, then the blocks below them, one block diagonal after the other.
__device__ __forceinline__ void invert_unit_lower(const float *N, float *T, float *X, int tid, int nthreads) {
    if (tid < kChunk) {
        const int b = tid & ~15, c = tid & 15;
        float x[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float s = r == c ? 1.f : 0.f;
#pragma unroll
            for (int k = 0; k < r; ++k) s = fmaf(-N[(b + r) * kInvStride + b + k], x[k], s);
            x[r] = s;
            T[(b + r) * kInvStride + b + c] = s;
        }
    }
    __syncthreads();
    for (int d = 1; d < 4; ++d) {
        const int count = (4 - d) * 256;
        for (int i = tid; i < count; i += nthreads) {
            const int bi = d + (i >> 8), r = (i >> 4) & 15, c = i & 15, j0 = (bi - d) * 16;
            float s = 0.f;
            for (int k = j0; k < bi * 16; ++k) s = fmaf(N[(bi * 16 + r) * kInvStride + k], T[k * kInvStride + j0 + c], s);
            X[i] = s;
        }
        __syncthreads();
        for (int i = tid; i < count; i += nthreads) {
            const int bi = d + (i >> 8), r = (i >> 4) & 15, c = i & 15, j0 = (bi - d) * 16;
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < 16; ++k) s = fmaf(-T[(bi * 16 + r) * kInvStride + bi * 16 + k], X[(i & ~255) + k * 16 + c], s);
            T[(bi * 16 + r) * kInvStride + j0 + c] = s;
        }
        __syncthreads();
    }
}

// A pair of values to the same place of kPlanes planes.
__device__ __forceinline__ void put_planes(__nv_bfloat16 *dst, size_t plane, float x, float y) {
    uint32_t w[kPlanes];
    split_pair<kPlanes>(x, y, w);
#pragma unroll
    for (int p = 0; p < kPlanes; ++p) *reinterpret_cast<uint32_t *>(dst + p * plane) = w[p];
}

// T diag(beta) as planes, zeros above the diagonal.
__device__ __forceinline__ void write_inverse(const float *T, const float *beta, __nv_bfloat16 *dst, int tid, int nthreads) {
    for (int i = tid; i < kChunk * kChunk / 2; i += nthreads) {
        const int r = i >> 5, c = (i & 31) * 2;
        const float x = c <= r ? T[r * kInvStride + c] * beta[c] : 0.f;
        const float y = c + 1 <= r ? T[r * kInvStride + c + 1] * beta[c + 1] : 0.f;
        put_planes(dst + r * kChunk + c, kChunk * kChunk, x, y);
    }
}

// Cumulative scalar log-decay of the chunk's tokens, in fp64: differences of the sums, not the sums, go into
// exponentials, and after a strong decay fp32 sums would leave the later differences few bits.  A gate below -1e4
// counts as -1e4 (its exponential is zero all the same), so that a reset (-inf) gives no inf - inf.
__device__ __forceinline__ void chunk_decay_sums(const ScanArgs &a, const ChunkPlace &p, int h, double *G, int lane) {
    double x[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int i = 2 * lane + e;
        const float g = a.g && i < p.valid ? a.g[(size_t)(p.tok0 + i) * a.H + h] : 0.f;
        x[e] = g < -1e4f ? -1e4 : (double)g;
    }
    double s = x[0] + x[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
    }
    G[2 * lane + 1] = s;
    G[2 * lane] = s - x[1];
}

template <int P, int DK>
constexpr size_t prep_scalar_smem(bool delta) {
    return (size_t)2 * P * kChunk * DK * 2 + (kChunk * 8) + kChunk * 4 + (delta ? (2 * kChunk * kInvStride + 3 * 256) * 4 : 0);
}

// Scalar decay: A and L are masked products of whole tiles, scaled entry by entry.
template <int P, int DK, bool DELTA>
__global__ void __launch_bounds__(128) scan_prep_scalar_kernel(const ScanArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, chunk = blockIdx.x, h = blockIdx.y;
    ChunkPlace p;
    if (!chunk_place(a, chunk, p)) return;
    const size_t unit = (size_t)chunk * a.H + h;
    const int hq = h / (a.H / a.Hq);
    constexpr int kTile = kChunk * DK * 2;
    const uint32_t q_s = smem_addr(smem), k_s = q_s + P * kTile;
    double *G = reinterpret_cast<double *>(smem + 2 * P * kTile);
    float *beta = reinterpret_cast<float *>(G + kChunk);
    float *N = beta + kChunk, *T = N + kChunk * kInvStride, *X = T + kChunk * kInvStride;
    const size_t off = ((size_t)p.tok0 * a.Hq + hq) * DK;
#pragma unroll
    for (int pl = 0; pl < P; ++pl) {
        load_tile(q_s + pl * kTile, a.qp + pl * a.q_plane + off, (size_t)a.Hq * DK, kChunk, DK, p.valid, tid, 128);
        load_tile(k_s + pl * kTile, a.kp + pl * a.q_plane + off, (size_t)a.Hq * DK, kChunk, DK, p.valid, tid, 128);
    }
    cp_async_commit();
    if (warp == 0) chunk_decay_sums(a, p, h, G, lane);
    if (DELTA && tid >= 64) {
        const int i = tid - 64;
        beta[i] = scan_beta(i < p.valid ? a.beta[(size_t)(p.tok0 + i) * a.H + h] : 0.f);
    }
    cp_async_wait_all();
    __syncthreads();
    if (tid < kChunk) {
        a.decay[unit * 2 * kChunk + tid] = expf((float)G[tid]);
        a.decay[unit * 2 * kChunk + kChunk + tid] = expf((float)(G[kChunk - 1] - G[tid]));
    }
    const int m0 = warp * 16;
    float qa[8][4] = {}, ka[8][4] = {};
#pragma unroll
    for (int k0 = 0; k0 < DK; k0 += 16) {
        uint32_t aq[P][4], ak[P][4];
#pragma unroll
        for (int pl = 0; pl < P; ++pl) {
            load_a(aq[pl], q_s + pl * kTile, DK, m0, k0, lane);
            if (DELTA) load_a(ak[pl], k_s + pl * kTile, DK, m0, k0, lane);
        }
#pragma unroll
        for (int nn = 0; nn < 4; ++nn) {
            if (nn > warp) break;
#pragma unroll
            for (int pl = 0; pl < P; ++pl) {
                uint32_t b[4];
                load_b(b, k_s + pl * kTile, DK, nn * 16, k0, lane);
#pragma unroll
                for (int pa = 0; pa + pl < P; ++pa) {  // P = 3: the six products that count
                    mma(qa[2 * nn], aq[pa], b[0], b[1]);
                    mma(qa[2 * nn + 1], aq[pa], b[2], b[3]);
                    if (DELTA) {
                        mma(ka[2 * nn], ak[pa], b[0], b[1]);
                        mma(ka[2 * nn + 1], ak[pa], b[2], b[3]);
                    }
                }
            }
        }
    }
    const int g = lane >> 2, t = lane & 3;
    __nv_bfloat16 *A = a.A + unit * kPlanes * kChunk * kChunk;
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = m0 + g + 8 * half, j = n * 8 + 2 * t;
            float m[2], x[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                m[e] = j + e <= i ? expf((float)(G[i] - G[j + e])) : 0.f;
                x[e] = j + e <= i ? a.scale * qa[n][2 * half + e] * m[e] : 0.f;
                if (DELTA) N[i * kInvStride + j + e] = j + e < i ? beta[i] * ka[n][2 * half + e] * m[e] : 0.f;
            }
            put_planes(A + i * kChunk + j, kChunk * kChunk, x[0], x[1]);
        }
    if (DELTA) {
        __syncthreads();
        invert_unit_lower(N, T, X, tid, 128);
        write_inverse(T, beta, a.T + unit * kPlanes * kChunk * kChunk, tid, 128);
    }
}

// ---- per-channel decay -------------------------------------------------------------------------------------
// The factor e^(G_ic - G_jc) does not leave the sum over channels, and e^(G_i), e^(-G_j) apart overflow, so a
// chunk is cut into four blocks of 16 tokens.  With p the cumulative decay from a block's start, s the decay behind
// a token up to its block's end and B a block's total, for token i of block I and j of block J < I
//     e^(G_i - G_j) = e^(p_i) e^(B_(J+1) + .. + B_(I-1)) e^(s_j),
// every exponent a sum of gates of one sign: nothing overflows and nothing cancels.  Inside a block
// e^(p_i - p_j) = e^(p_i) e^(-B) e^(s_j), which is used while -B stays below kBlockDecay (e^60 is far from the range
// of fp32 and bf16 planes); where a block decays further, its pairs are summed one by one.
constexpr int kBlock = 16;
constexpr float kBlockDecay = 60.f;

// q_i e^(p_i) (RWKV6: its readout sees the decay in front of the token), k_i e^(p_i), k_j e^(s_j) of a (block, channel).
template <typename IO>
struct BlockVectors {
    float qs[kBlock], ks[kBlock], kc[kBlock];
    float B;
};
template <typename IO, bool EXCL>
__device__ __forceinline__ void block_vectors(const ScanArgs &a, const ChunkPlace &p, int h, int hq, int DK, int blk, int c, bool with_q,
                                              BlockVectors<IO> &o) {
    float gate[kBlock];
#pragma unroll
    for (int r = 0; r < kBlock; ++r) {
        const int i = blk * kBlock + r;
        const bool ok = i < p.valid;
        gate[r] = ok ? a.g[((size_t)(p.tok0 + i) * a.H + h) * DK + c] : 0.f;
        const size_t at = ((size_t)(p.tok0 + (ok ? i : 0)) * a.Hq + hq) * DK + c;
        o.kc[r] = ok ? to_f32(static_cast<const IO *>(a.k)[at]) : 0.f;
        if (with_q) o.qs[r] = ok ? to_f32(static_cast<const IO *>(a.q)[at]) : 0.f;
    }
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < kBlock; ++r) {
        if (EXCL && with_q) o.qs[r] *= expf(s);
        s += gate[r];
        const float e = expf(s);
        if (!EXCL && with_q) o.qs[r] *= e;
        o.ks[r] = o.kc[r] * e;
    }
    s = 0.f;
#pragma unroll
    for (int r = kBlock - 1; r >= 0; --r) {
        o.kc[r] *= expf(s);
        s += gate[r];
    }
    o.B = s;
}

// fp32 tile of 64 x DK in shared memory, rows padded by four
template <int DK>
constexpr int kVecStride = DK + 4;

template <int DK>
constexpr size_t prep_vector_smem(bool delta) {
    return (size_t)(delta ? 2 : 1) * kChunk * kVecStride<DK> * 4 + kPlanes * kChunk * DK * 2 + 4 * DK * 4 + kChunk * 4 + 16 +
           (delta ? (2 * kChunk * kInvStride + 3 * 256) * 4 : 0);
}

// One pair (i, j) of a strongly decaying block: sum_c x_ic k_jc e^(g_(j+1) + .. + g_i) with the gates added up directly.
template <typename IO, bool EXCL>
__device__ __forceinline__ void pair_sums(const ScanArgs &a, const ChunkPlace &p, int h, int hq, int DK, int i, int j, float &sq, float &sk) {
    sq = sk = 0.f;
    if (i >= p.valid) return;
    const size_t ri = ((size_t)(p.tok0 + i) * a.Hq + hq) * DK, rj = ((size_t)(p.tok0 + j) * a.Hq + hq) * DK;
    for (int c = 0; c < DK; ++c) {
        float s = 0.f, last = 0.f;
        for (int m = j + 1; m <= i; ++m) {
            last = a.g[((size_t)(p.tok0 + m) * a.H + h) * DK + c];
            if (!EXCL || m < i) s += last;
        }
        const float kj = to_f32(static_cast<const IO *>(a.k)[rj + c]);
        sq = fmaf(to_f32(static_cast<const IO *>(a.q)[ri + c]) * kj, expf(s), sq);
        sk = fmaf(to_f32(static_cast<const IO *>(a.k)[ri + c]) * kj, expf(s), sk);
    }
}

// OP selects the readout (RWKV6) and the delta rule; 256 threads.
template <int OP, int DK, typename IO>
__global__ void __launch_bounds__(256) scan_prep_vector_kernel(const ScanArgs a) {
    constexpr bool DELTA = OpTraits<OP>::kDeltaRule, EXCL = OpTraits<OP>::kBonus;
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, chunk = blockIdx.x, h = blockIdx.y;
    ChunkPlace p;
    if (!chunk_place(a, chunk, p)) return;
    const size_t unit = (size_t)chunk * a.H + h;
    const int hq = h / (a.H / a.Hq);
    constexpr int VS = kVecStride<DK>;
    constexpr int kTile = kChunk * DK * 2;
    const uint32_t kc_s = smem_addr(smem);
    float *qs = reinterpret_cast<float *>(smem + kPlanes * kTile);
    float *ks = qs + kChunk * VS;                       // delta rule only
    float *B = DELTA ? ks + kChunk * VS : ks;           // [4][DK]
    float *beta = B + 4 * DK;
    int *deep = reinterpret_cast<int *>(beta + kChunk); // [4] blocks that decay too far for the factored form
    float *N = reinterpret_cast<float *>(deep + 4), *T = N + kChunk * kInvStride, *X = T + kChunk * kInvStride;
    if (tid < 4) deep[tid] = 0;
    if (DELTA && tid >= 64 && tid < 128) {
        const int i = tid - 64;
        beta[i] = scan_beta(i < p.valid ? a.beta[(size_t)(p.tok0 + i) * a.H + h] : 0.f);
    }
    __syncthreads();
    for (int w = tid; w < 4 * DK; w += 256) {
        const int blk = w / DK, c = w % DK;
        BlockVectors<IO> o;
        block_vectors<IO, EXCL>(a, p, h, hq, DK, blk, c, true, o);
        B[blk * DK + c] = o.B;
        if (!(o.B > -kBlockDecay)) deep[blk] = 1;
#pragma unroll
        for (int r = 0; r < kBlock; ++r) {
            const int i = blk * kBlock + r;
            qs[i * VS + c] = o.qs[r] * a.scale;
            if (DELTA) ks[i * VS + c] = o.ks[r];
            unsigned char *at = smem + i * DK * 2 + (((c >> 3) ^ (i & 7)) << 4) + (c & 7) * 2;
            float x = o.kc[r];
#pragma unroll
            for (int pl = 0; pl < kPlanes; ++pl) {
                const __nv_bfloat16 w = __float2bfloat16_rn(x);
                *reinterpret_cast<__nv_bfloat16 *>(at + pl * kTile) = w;
                x -= __bfloat162float(w);
            }
        }
    }
    __syncthreads();
    // decayed vectors of the whole chunk for the chain kernels
    const size_t vec = unit * kPlanes * kChunk * DK;
    for (int w = tid; w < kChunk * DK / 2; w += 256) {
        const int i = w / (DK / 2), c = (w % (DK / 2)) * 2, blk = i >> 4;
        float front[2] = {0.f, 0.f}, back[2] = {0.f, 0.f};
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float x = B[m * DK + c + e];
                if (m < blk) front[e] += x;
                if (m > blk) back[e] += x;
            }
        const float f0 = expf(front[0]), f1 = expf(front[1]);
        const size_t at = vec + (size_t)i * DK + c;
        put_planes(a.qt + at, kChunk * DK, qs[i * VS + c] * f0, qs[i * VS + c + 1] * f1);
        if (DELTA) put_planes(a.kt + at, kChunk * DK, ks[i * VS + c] * f0, ks[i * VS + c + 1] * f1);
        float x = 0.f, y = 0.f;
#pragma unroll
        for (int pl = kPlanes - 1; pl >= 0; --pl) {
            const uint32_t w2 = *reinterpret_cast<const uint32_t *>(smem + pl * kTile + i * DK * 2 + (((c >> 3) ^ (i & 7)) << 4) + (c & 7) * 2);
            x += bf16_lo(w2), y += bf16_hi(w2);
        }
        put_planes(a.kh + at, kChunk * DK, x * expf(back[0]), y * expf(back[1]));
    }
    if (tid < DK) a.decay[unit * DK + tid] = expf(B[tid] + B[DK + tid] + B[2 * DK + tid] + B[3 * DK + tid]);
    // block pairs (I, J <= I) of A and L, 16 x 16 each, one warp per pair and matrix
    __nv_bfloat16 *A = a.A + unit * kPlanes * kChunk * kChunk;
    const int g = lane >> 2, t = lane & 3;
    constexpr int kMats = DELTA ? 2 : 1;
    for (int task = warp; task < 16 * kMats; task += 8) {
        const int which = task >> 4, I = (task >> 2) & 3, J = task & 3;
        float acc[2][4] = {};
        if (J < I || (J == I && !deep[I])) {
            const float *src = which ? ks : qs;
#pragma unroll 2
            for (int k0 = 0; k0 < DK; k0 += 16) {
                float f[4];  // channels k0 + 2t + {0, 1, 8, 9}
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int c = k0 + 2 * t + (e & 1) + 8 * (e >> 1);
                    float x = 0.f;
                    if (J == I) x = -B[I * DK + c];
                    else
                        for (int m = J + 1; m < I; ++m) x += B[m * DK + c];
                    f[e] = expf(x);
                }
                uint32_t x[kPlanes][4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = I * kBlock + g + 8 * (e & 1), c = k0 + 2 * t + 8 * (e >> 1);
                    const float2 y = *reinterpret_cast<const float2 *>(src + row * VS + c);
                    uint32_t w[kPlanes];
                    split_pair<kPlanes>(y.x * f[2 * (e >> 1)], y.y * f[2 * (e >> 1) + 1], w);
#pragma unroll
                    for (int pl = 0; pl < kPlanes; ++pl) x[pl][e] = w[pl];
                }
#pragma unroll
                for (int pl = 0; pl < kPlanes; ++pl) {
                    uint32_t b[4];
                    load_b(b, kc_s + pl * kTile, DK, J * kBlock, k0, lane);
                    mma_planes<kPlanes, kPlanes>(acc[0], acc[1], x, b, pl);
                }
            }
        } else if (J == I) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = I * kBlock + g + 8 * (e >> 1), j = J * kBlock + n * 8 + 2 * t + (e & 1);
                    if (j <= i) {
                        float sq, sk;
                        pair_sums<IO, EXCL>(a, p, h, hq, DK, i, j, sq, sk);
                        acc[n][e] = which ? sk : sq * a.scale;
                    }
                }
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int i = I * kBlock + g + 8 * half, j = J * kBlock + n * 8 + 2 * t;
                float x[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const bool in = which || EXCL ? j + e < i : j + e <= i;
                    x[e] = in ? acc[n][2 * half + e] : 0.f;
                    if (which) N[i * kInvStride + j + e] = in ? beta[i] * x[e] : 0.f;
                }
                if (!which) {
                    if (EXCL && (i == j || i == j + 1) && i < p.valid) {  // the bonus term q . (bonus * k)
                        float s = 0.f;
                        const size_t r = ((size_t)(p.tok0 + i) * a.Hq + hq) * DK;
                        for (int c = 0; c < DK; ++c)
                            s = fmaf(to_f32(static_cast<const IO *>(a.q)[r + c]) * to_f32(static_cast<const IO *>(a.k)[r + c]), a.bonus[h * DK + c], s);
                        x[i - j] = s;
                    }
                    put_planes(A + i * kChunk + j, kChunk * kChunk, x[0], x[1]);
                }
            }
    }
    if (DELTA) {
        __syncthreads();
        invert_unit_lower(N, T, X, tid, 256);
        write_inverse(T, beta, a.T + unit * kPlanes * kChunk * kChunk, tid, 256);
    }
}

}  // namespace deltalog
