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

// Zeros to the rows of `out` that no chain will write, for the CTA of a chunk that has nothing to prepare: a skipped row's
// chunk clears its own tokens, and the entries behind the last chunk (with the CTA beyond the table) share those behind the last
// sequence.  No launch of its own, and nothing is written twice, as a memset of the whole tensor in front would.  (Out of line:
// inside, the code between a short prompt's instructions cost it a microsecond.)
static __device__ __noinline__ void clear_rows(void *out, int first, int last, int H, int h, int row_bytes) {
    const int lane = threadIdx.x & 31, units = row_bytes / 16;
    for (int row = first + (int)(threadIdx.x >> 5); row < last; row += (int)(blockDim.x >> 5)) {
        uint4 *dst = reinterpret_cast<uint4 *>(out) + ((size_t)row * H + h) * units;
        for (int u = lane; u < units; u += 32) dst[u] = make_uint4(0u, 0u, 0u, 0u);
    }
}
static __device__ __noinline__ void clear_unwritten(void *out, const int32_t *starts, const int32_t *chunk_starts, const int32_t *chunk_seq, int n,
                                                    int max_tokens, int max_chunks, int chunk, int H, int h, int row_bytes) {
    const int seq = chunk < max_chunks ? chunk_seq[chunk] : -1;
    if (seq >= 0) {
        const int first = starts[seq] + (chunk - chunk_starts[seq]) * kChunk;
        clear_rows(out, first, min(first + kChunk, starts[seq + 1]), H, h, row_bytes);
        return;
    }
    const int tokens = starts[n], chunks = chunk_starts[n], tail = max_tokens - tokens;
    if (tail <= 0) return;
    const int parts = max_chunks - chunks + 1, each = (tail + parts - 1) / parts;
    const long long first = tokens + (long long)each * (chunk - chunks);
    if (first < max_tokens) clear_rows(out, (int)first, (int)min(first + each, (long long)max_tokens), H, h, row_bytes);
}
template <typename IO>
__device__ __forceinline__ void clear_unwritten(const ScanArgs &a, int chunk, int h) {
    if (a.clear)
        clear_unwritten(a.out, a.starts, a.chunk_starts, a.chunk_seq, a.n, a.max_tokens, a.max_chunks, chunk, a.H, h, a.dv * (int)sizeof(IO));
}

constexpr int kInvStride = kChunk + 8;  // row of the fp32 matrices: fragment reads without bank conflicts

// T = (I + N)^-1 for the strictly lower N (64 x 64, fp32).  The four diagonal 16 x 16 blocks by forward substitution, one
// column per thread; then warp J solves column block J downwards, T_IJ = -T_II sum_(J <= K < I) N_IK T_KJ, on the tensor
// cores and transposed: the accumulators of a block are the A operand of the next.  (With fp32 FMAs in place of the
// products this step took two thirds of the kernel.)
__device__ __forceinline__ void invert_unit_lower(const float *N, float *T, int tid) {
    const int lane = tid & 31, J = tid >> 5;
    if (tid < kChunk) {
        const int b = tid & ~15, c = tid & 15;
        float x[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float s0 = r == c ? 1.f : 0.f, s1 = 0.f;
#pragma unroll
            for (int k = 0; k < r; k += 2) {
                const float2 n = *reinterpret_cast<const float2 *>(N + (b + r) * kInvStride + b + k);
                s0 = fmaf(-n.x, x[k], s0);
                if (k + 1 < r) s1 = fmaf(-n.y, x[k + 1], s1);
            }
            x[r] = s0 + s1;
            T[(b + r) * kInvStride + b + c] = x[r];
        }
    }
    __syncthreads();
    if (J < 3) {
        const int g = lane >> 2, t = lane & 3;
        uint32_t f[3][kPlanes][4];  // blocks (J + r, J) of T, transposed, as A operands
        frag_a_t(f[0], T, kInvStride, J * 16, J * 16, lane);
#pragma unroll
        for (int r = 1; r < 4; ++r) {
            const int I = J + r;
            if (I > 3) break;
            float x[2][4] = {}, y[2][4] = {};
            uint32_t b[kPlanes][4], w[kPlanes][4];
#pragma unroll
            for (int k = 0; k < r; ++k) {
                frag_b(b, N, kInvStride, I * 16, (J + k) * 16, lane);
                mma_all(x[0], x[1], f[k], b);
            }
            acc_to_a<kPlanes>(x[0], x[1], w);
            frag_b(b, T, kInvStride, I * 16, I * 16, lane);
            mma_all(y[0], y[1], w, b);
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y[n][e] = -y[n][e];
                    T[(I * 16 + n * 8 + 2 * t + (e & 1)) * kInvStride + J * 16 + g + 8 * (e >> 1)] = y[n][e];
                }
            if (r < 3) acc_to_a<kPlanes>(y[0], y[1], f[r]);
        }
    }
    __syncthreads();
}

// A pair of values to the same place of kPlanes planes; `all` false: of the first two (what only a bf16 output sees).
__device__ __forceinline__ void put_planes(__nv_bfloat16 *dst, size_t plane, float x, float y, bool all = true) {
    uint32_t w[kPlanes];
    split_pair<kPlanes>(x, y, w);
#pragma unroll
    for (int p = 0; p < kPlanes; ++p)
        if (p < 2 || all) *reinterpret_cast<uint32_t *>(dst + p * plane) = w[p];
}

// T diag(beta) as planes.  Of A and T the 16 x 16 blocks above the diagonal are neither written nor read.
__device__ __forceinline__ void write_inverse(const float *T, const float *beta, __nv_bfloat16 *dst, int tid, int nthreads) {
    for (int i = tid; i < 10 * 128; i += nthreads) {  // ten blocks of 128 pairs
        const int blk = i >> 7, I = blk < 1 ? 0 : blk < 3 ? 1 : blk < 6 ? 2 : 3, J = blk - I * (I + 1) / 2;
        const int r = I * 16 + ((i >> 3) & 15), c = J * 16 + (i & 7) * 2;
        const float2 x = *reinterpret_cast<const float2 *>(T + r * kInvStride + c);
        put_planes(dst + image_at(r, c), kChunk * kChunk, c <= r ? x.x * beta[c] : 0.f, c + 1 <= r ? x.y * beta[c + 1] : 0.f);
    }
}

// Cumulative scalar log-decay of the chunk's tokens, in fp64: differences of the sums, not the sums, go into
// exponentials, and after a strong decay fp32 sums would leave the later differences few bits (so a sum is kept as two
// floats).  A gate below -1e4
// counts as -1e4 (its exponential is zero all the same), so that a reset (-inf) gives no inf - inf.
__device__ __forceinline__ void chunk_decay_sums(const ScanArgs &a, const ChunkPlace &p, int h, float2 *G, int lane) {
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
#pragma unroll
    for (int e = 1; e >= 0; --e) {
        const float hi = (float)s;
        G[2 * lane + e] = make_float2(hi, (float)(s - hi));
        s -= x[e];
    }
}
__device__ __forceinline__ float decay_between(const float2 &i, const float2 &j) { return (i.x - j.x) + (i.y - j.y); }

// Rows of the plan, the longest first (sorted by chunks, those of 511 and more together): what the chain kernels run
// through.  A chain's time is its length, and the longest one started last would run alone at the end.
__device__ __forceinline__ void order_rows(const ScanArgs &a, int *bins, int tid, int nthreads) {  // bins: 512, shared
    for (int i = tid; i < 512; i += nthreads) bins[i] = 0;
    __syncthreads();
    auto bin = [&](int i) { return 511 - min(511, a.chunk_starts[i + 1] - a.chunk_starts[i]); };
    for (int i = tid; i < a.n; i += nthreads) atomicAdd(bins + bin(i), 1);
    __syncthreads();
    if (tid < 32) {  // exclusive scan, sixteen bins a lane
        int sum = 0, own[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) own[i] = bins[tid * 16 + i], sum += own[i];
        int s = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, s, o);
            if (tid >= o) s += y;
        }
        s -= sum;
#pragma unroll
        for (int i = 0; i < 16; ++i) bins[tid * 16 + i] = s, s += own[i];
    }
    __syncthreads();
    for (int i = tid; i < a.n; i += nthreads) a.order[atomicAdd(bins + bin(i), 1)] = i;
}

template <int P, int DK>
struct PrepScalarSmem {
    static constexpr int kTile = kChunk * DK * 2;
    static constexpr int kMat = kChunk * kInvStride * 4;
    // q and k, in whose place N and T come later
    static constexpr int small(bool delta) { return delta && 2 * kMat > 2 * P * kTile ? 2 * kMat : 2 * P * kTile; }
    static constexpr size_t bytes(bool delta) { return small(delta) + kChunk * 8 + kChunk * 4; }
};

// Scalar decay: A and L are masked products of whole tiles, scaled entry by entry.  Five CTAs share an SM: the steps of
// one chunk depend on each other, and only other chunks fill the gaps.  bf16, 32 heads of 128: 36k tokens 336 us, 8k tokens 79 us
// (2.8 TB/s of DRAM traffic).
template <int P, int DK, bool DELTA, typename IO>
__global__ void __launch_bounds__(128, P == 1 ? 5 : 3) scan_prep_scalar_kernel(const ScanArgs a) {
    using L = PrepScalarSmem<P, DK>;
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, chunk = blockIdx.x, h = blockIdx.y;
    scan_kernel_begin();
    if (chunk == a.max_chunks) {  // one CTA beyond the chunks
        if (h == 0) order_rows(a, reinterpret_cast<int *>(smem), tid, 128);
        clear_unwritten<IO>(a, chunk, h);
        return;
    }
    ChunkPlace p;
    if (!chunk_place(a, chunk, p)) {
        clear_unwritten<IO>(a, chunk, h);
        return;
    }
    const size_t unit = (size_t)chunk * a.H + h;
    const int hq = h / (a.H / a.Hq);
    constexpr int kTile = L::kTile;
    const uint32_t q_s = smem_addr(smem), k_s = q_s + P * kTile;
    float *N = reinterpret_cast<float *>(smem), *T = reinterpret_cast<float *>(smem + L::kMat);
    constexpr int kSmall = DELTA && 2 * L::kMat > 2 * P * kTile ? 2 * L::kMat : 2 * P * kTile;
    float2 *G = reinterpret_cast<float2 *>(smem + kSmall);
    float *beta = reinterpret_cast<float *>(G + kChunk);
    const size_t off = ((size_t)p.tok0 * a.Hq + hq) * DK, stride = (size_t)a.Hq * DK;
    if constexpr (sizeof(IO) == 2) {
        load_tile<DK>(q_s, static_cast<const IO *>(a.q) + off, stride, p.valid, tid, 128);
        load_tile<DK>(k_s, static_cast<const IO *>(a.k) + off, stride, p.valid, tid, 128);
        cp_async_commit();
    } else {
#pragma unroll 1
        for (int i0 = 0; i0 < kChunk * DK / 2; i0 += 128 * 8) {
            float2 q[8], k[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int i = i0 + u * 128 + tid;
                const size_t at = off + min(i / (DK / 2), p.valid - 1) * stride + i % (DK / 2) * 2;
                q[u] = *reinterpret_cast<const float2 *>(static_cast<const IO *>(a.q) + at), k[u] = *reinterpret_cast<const float2 *>(static_cast<const IO *>(a.k) + at);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int i = i0 + u * 128 + tid, row = i / (DK / 2), c = i % (DK / 2) * 2;
                const bool ok = row < p.valid;
                __nv_bfloat16 *dst = reinterpret_cast<__nv_bfloat16 *>(smem) + image_at(row, c);
                put_planes(dst, kTile / 2, ok ? q[u].x : 0.f, ok ? q[u].y : 0.f);
                put_planes(dst + P * kTile / 2, kTile / 2, ok ? k[u].x : 0.f, ok ? k[u].y : 0.f);
            }
        }
    }
    if (warp == 0) chunk_decay_sums(a, p, h, G, lane);
    if (DELTA && tid >= 64) {
        const int i = tid - 64;
        beta[i] = scan_beta(i < p.valid ? a.beta[(size_t)(p.tok0 + i) * a.H + h] : 0.f);
    }
    cp_async_wait_all();
    __syncthreads();
    if (tid < kChunk) {
        a.decay[unit * 2 * kChunk + tid] = expf(G[tid].x + G[tid].y);
        a.decay[unit * 2 * kChunk + kChunk + tid] = expf(decay_between(G[kChunk - 1], G[tid]));
    }
    if (P > 1 && h % (a.H / a.Hq) == 0) {  // the tiles as they are: the chain kernels' operands
        const size_t at = ((size_t)chunk * a.Hq + hq) * P * kTile / 16;
        const uint4 *src = reinterpret_cast<const uint4 *>(smem);
        for (int i = tid; i < P * kTile / 16; i += 128) {
            reinterpret_cast<uint4 *>(a.qi)[at + i] = src[i];
            reinterpret_cast<uint4 *>(a.ki)[at + i] = src[P * kTile / 16 + i];
        }
    }
    const int m0 = warp * 16;
    float qa[8][4] = {}, ka[8][4] = {};
#pragma unroll
    for (int k0 = 0; k0 < DK; k0 += 16) {
        uint32_t aq[P][4], ak[P][4];
#pragma unroll
        for (int pl = 0; pl < P; ++pl) {
            load_a(aq[pl], q_s + pl * kTile, m0, k0, lane);
            if (DELTA) load_a(ak[pl], k_s + pl * kTile, m0, k0, lane);
        }
#pragma unroll
        for (int nn = 0; nn < 4; ++nn) {
            if (nn > warp) break;
            {
                uint32_t b[P][4];
#pragma unroll
                for (int pl = 0; pl < P; ++pl) load_b(b[pl], k_s + pl * kTile, nn * 16, k0, lane);
                mma_all(qa[2 * nn], qa[2 * nn + 1], aq, b);
                if (DELTA) mma_all(ka[2 * nn], ka[2 * nn + 1], ak, b);
            }
        }
    }
    const int g = lane >> 2, t = lane & 3;
    __nv_bfloat16 *A = a.A + unit * kPlanes * kChunk * kChunk;
    const float2 Gi[2] = {G[m0 + g], G[m0 + g + 8]};
    const bool all = sizeof(IO) == 4 || a.keep;  // planes of A
    if (DELTA) __syncthreads();  // the tiles make room for N
#pragma unroll
    for (int n = 0; n < 8; ++n) {
        if (n > 2 * warp + 1) break;
        const int j = n * 8 + 2 * t;
        const float2 G0 = G[j], G1 = G[j + 1];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = m0 + g + 8 * half;
            const float d0 = j <= i ? decay_exp(decay_between(Gi[half], G0)) : 0.f, d1 = j + 1 <= i ? decay_exp(decay_between(Gi[half], G1)) : 0.f;
            // (selected, not multiplied: a product above the diagonal may be anything)
            put_planes(A + image_at(i, j), kChunk * kChunk, j <= i ? a.scale * qa[n][2 * half] * d0 : 0.f,
                       j + 1 <= i ? a.scale * qa[n][2 * half + 1] * d1 : 0.f, all);
            if (DELTA)
                *reinterpret_cast<float2 *>(N + i * kInvStride + j) = make_float2(j < i ? beta[i] * ka[n][2 * half] * d0 : 0.f,
                                                                                  j + 1 < i ? beta[i] * ka[n][2 * half + 1] * d1 : 0.f);
        }
    }
    if (DELTA) {
        __syncthreads();
        invert_unit_lower(N, T, tid);
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
// of fp32 and bf16 planes); where a block decays further, its pairs are summed one by one.  There the factor e^(-B) brings
// small weights back up to one, and what counts is their relative error.  Exponentials of sums rounded to fp32 are off by |x| 2^-24
// each: up to 2.4e-5 of a pair's weight at gates of -3.5.  So the weights of a block are running products of e^(gate): of
// a pair's weight the tokens outside of it cancel, up to one rounding of 2^-24 per product.
constexpr int kBlock = 16;
constexpr float kBlockDecay = 60.f;

// The decayed vectors of one block and one pair of neighbouring channels: q_i e^(p_i) (RWKV6: the decay in front of the
// token), k_i e^(p_i), k_j e^(s_j), and the block's total B.
struct BlockVectors {
    float2 qs[kBlock], ks[kBlock], kc[kBlock];
    float2 B, E;  // and e^B as the product that the weights are made of
};
template <typename IO, bool EXCL, bool DELTA>
__device__ __forceinline__ void block_vectors(const ScanArgs &a, const ChunkPlace &p, int h, int hq, int DK, int blk, int c, BlockVectors &o) {
    float2 gate[kBlock];
#pragma unroll
    for (int r = 0; r < kBlock; ++r) {
        // (rows behind the last token read it again and are cleared below: loads without branches go out together)
        const size_t i = p.tok0 + min(blk * kBlock + r, p.valid - 1), at = (i * a.Hq + hq) * DK + c;
        float x[2];
        gate[r] = *reinterpret_cast<const float2 *>(a.g + (i * a.H + h) * DK + c);
        load_vec<IO, 2>(static_cast<const IO *>(a.k) + at, x);
        o.kc[r] = make_float2(x[0], x[1]);
        load_vec<IO, 2>(static_cast<const IO *>(a.q) + at, x);
        o.qs[r] = make_float2(x[0], x[1]);
    }
#pragma unroll
    for (int r = 0; r < kBlock; ++r)
        if (blk * kBlock + r >= p.valid) gate[r] = o.kc[r] = o.qs[r] = make_float2(0.f, 0.f);
    float2 s = make_float2(0.f, 0.f), e = make_float2(1.f, 1.f);
#pragma unroll
    for (int r = 0; r < kBlock; ++r) {
        if (EXCL) o.qs[r].x *= e.x, o.qs[r].y *= e.y;
        s.x += gate[r].x, s.y += gate[r].y;
        gate[r] = make_float2(expf(gate[r].x), expf(gate[r].y));
        e.x *= gate[r].x, e.y *= gate[r].y;
        if (!EXCL) o.qs[r].x *= e.x, o.qs[r].y *= e.y;
        if (DELTA) o.ks[r] = make_float2(o.kc[r].x * e.x, o.kc[r].y * e.y);
    }
    o.B = s, o.E = e;
    e = make_float2(1.f, 1.f);
#pragma unroll
    for (int r = kBlock - 1; r >= 0; --r) {
        o.kc[r].x *= e.x, o.kc[r].y *= e.y;
        e.x *= gate[r].x, e.y *= gate[r].y;
    }
}

template <int DK>
struct PrepVectorSmem {
    static constexpr int kVS = DK + 8;                    // row of the fp32 vectors
    static constexpr int kVec = kChunk * kVS * 4;
    // q e^p, k e^s, (delta rule) k e^p, in whose place N and T come later; factors between blocks.  Two CTAs share an SM.
    __host__ __device__ static constexpr int factors(bool delta) { return (delta ? 3 : 2) * kVec; }
    __host__ __device__ static constexpr int small(bool delta) { return factors(delta) + 19 * DK * 4; }
    static constexpr size_t bytes(bool delta) { return small(delta) + kChunk * 4 + 16; }
};

// One pair (i, j) of a strongly decaying block: sum_c x_ic k_jc e^(g_(j+1) + .. + g_i) with the gates added up directly,
// for x = q and x = k.  (Out of line: rarely taken, large.)  Slow: one lane per pair.  A whole scan of KDA, 3.9k tokens of 5 rows, 32 heads
// of 128, takes 315 us with ordinary gates, 2.4 ms with a reset in every chunk and 4.3 ms with a tenth of the channels at -5 a token, where
// every block decays that far (training, with pairs_front and pairs_back of the gradients: 1.0, 4.3 and 6.7 ms).
template <typename IO, bool EXCL>
__device__ __noinline__ float2 pair_sums(const IO *q, const IO *k, int stride, const float *gate, int g_stride, int valid, int DK, int i, int j) {
    float sq = 0.f, sk = 0.f;
    if (i >= valid) return make_float2(0.f, 0.f);
    for (int c = 0; c < DK; ++c) {
        float s = 0.f;
        for (int m = j + 1; m <= (EXCL ? i - 1 : i); ++m) s += gate[(size_t)m * g_stride + c];
        const float kj = to_f32(k[(size_t)j * stride + c]);
        sq = fmaf(to_f32(q[(size_t)i * stride + c]) * kj, expf(s), sq);
        sk = fmaf(to_f32(k[(size_t)i * stride + c]) * kj, expf(s), sk);
    }
    return make_float2(sq, sk);
}

// OP selects the readout (RWKV6) and the delta rule; one thread per block and channel pair, so 256 or 128.
// Bound by latency at 16 warps per SM (a block's vectors take 96 registers of a thread, the chunk's 104 KB of an SM).
// bf16: KDA, 32 heads of 128, 13k tokens 532 us (2.1 TB/s of DRAM traffic); RWKV6, 64 heads of 64, 17k tokens 468 us.
template <int OP, int DK, typename IO>
__global__ void __launch_bounds__(2 * DK, 256 / DK) scan_prep_vector_kernel(const ScanArgs a) {
    constexpr bool DELTA = OpTraits<OP>::kDeltaRule, EXCL = OpTraits<OP>::kBonus;
    using L = PrepVectorSmem<DK>;
    constexpr int VS = L::kVS;
    extern __shared__ __align__(128) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, chunk = blockIdx.x, h = blockIdx.y;
    scan_kernel_begin();
    if (chunk == a.max_chunks) {  // one CTA beyond the chunks
        if (h == 0) order_rows(a, reinterpret_cast<int *>(smem), tid, 2 * DK);
        clear_unwritten<IO>(a, chunk, h);
        return;
    }
    ChunkPlace p;
    if (!chunk_place(a, chunk, p)) {
        clear_unwritten<IO>(a, chunk, h);
        return;
    }
    const size_t unit = (size_t)chunk * a.H + h;
    const int hq = h / (a.H / a.Hq);
    float *qs = reinterpret_cast<float *>(smem), *kc = qs + kChunk * VS, *ks = kc + kChunk * VS;
    float *B = reinterpret_cast<float *>(smem + L::factors(DELTA));  // [4][DK] block decays
    float *F = B + 4 * DK;                                          // [7][DK] e^(-B_I), e^(B_1), e^(B_2), e^(B_1 + B_2)
    float *W = F + 7 * DK;                                          // [2][4][DK] decay of the chunk in front of / behind a block
    float *beta = reinterpret_cast<float *>(smem + L::small(DELTA));
    int *deep = reinterpret_cast<int *>(beta + kChunk);             // [4] blocks that decay too far for the factored form
    float *T = reinterpret_cast<float *>(smem), *N = T + kChunk * kInvStride;
    if (tid < 4) deep[tid] = 0;
    if (DELTA && tid < kChunk) beta[tid] = scan_beta(tid < p.valid ? a.beta[(size_t)(p.tok0 + tid) * a.H + h] : 0.f);
    __syncthreads();
    // a thread's block and channel pair: the block's vectors into shared memory, then, with the other blocks' decays at hand,
    // the whole chunk's to the chain kernels
    const bool all = sizeof(IO) == 4 || a.keep;  // planes of A and of q e^G
    constexpr int kPairs = DK / 2, kThreads = 4 * kPairs, kWarps = kThreads / 32;
    const int blk = tid / kPairs, c = (tid % kPairs) * 2;
    float2 E;
    {
        BlockVectors o;
        block_vectors<IO, EXCL, DELTA>(a, p, h, hq, DK, blk, c, o);
        *reinterpret_cast<float2 *>(B + blk * DK + c) = o.B;
        E = o.E;
        if (!(o.B.x > -kBlockDecay && o.B.y > -kBlockDecay)) deep[blk] = 1;
#pragma unroll
        for (int r = 0; r < kBlock; ++r) {
            const int at = (blk * kBlock + r) * VS + c;
            o.qs[r].x *= a.scale, o.qs[r].y *= a.scale;
            *reinterpret_cast<float2 *>(qs + at) = o.qs[r];
            *reinterpret_cast<float2 *>(kc + at) = o.kc[r];
            if (DELTA) *reinterpret_cast<float2 *>(ks + at) = o.ks[r];
        }
    }
    __syncthreads();
    {
        float2 front = make_float2(0.f, 0.f), back = front;
        for (int m = 0; m < 4; ++m) {
            const float2 x = *reinterpret_cast<const float2 *>(B + m * DK + c);
            if (m < blk) front.x += x.x, front.y += x.y;
            if (m > blk) back.x += x.x, back.y += x.y;
        }
        *reinterpret_cast<float2 *>(W + blk * DK + c) = make_float2(decay_exp(front.x), decay_exp(front.y));
        *reinterpret_cast<float2 *>(W + (4 + blk) * DK + c) = make_float2(decay_exp(back.x), decay_exp(back.y));
        const float2 b = *reinterpret_cast<const float2 *>(B + blk * DK + c);
        *reinterpret_cast<float2 *>(F + blk * DK + c) = make_float2(1.f / E.x, 1.f / E.y);  // (not read where E may be 0)
        if (blk == 1 || blk == 2) *reinterpret_cast<float2 *>(F + (3 + blk) * DK + c) = make_float2(decay_exp(b.x), decay_exp(b.y));
        if (blk == 1) {
            const float2 x = *reinterpret_cast<const float2 *>(B + 2 * DK + c);
            *reinterpret_cast<float2 *>(F + 6 * DK + c) = make_float2(decay_exp(b.x + x.x), decay_exp(b.y + x.y));
        }
    }
    __syncthreads();
    // the whole chunk's decayed vectors, eight channels of a token at a time: 16-byte stores, one per plane
    {
        const size_t base = unit * kPlanes * kChunk * DK;
        auto write = [&](__nv_bfloat16 *dst, const float *vec, const float *factor, int i, int c8, bool three) {
            uint32_t w[kPlanes][4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 x = *reinterpret_cast<const float4 *>(vec + i * VS + c8 + 4 * j), y = *reinterpret_cast<const float4 *>(factor + (i >> 4) * DK + c8 + 4 * j);
                uint32_t z[kPlanes];
                split_pair<kPlanes>(x.x * y.x, x.y * y.y, z);
#pragma unroll
                for (int pl = 0; pl < kPlanes; ++pl) w[pl][2 * j] = z[pl];
                split_pair<kPlanes>(x.z * y.z, x.w * y.w, z);
#pragma unroll
                for (int pl = 0; pl < kPlanes; ++pl) w[pl][2 * j + 1] = z[pl];
            }
#pragma unroll
            for (int pl = 0; pl < kPlanes; ++pl)
                if (pl < 2 || three) *reinterpret_cast<uint4 *>(dst + base + pl * kChunk * DK + image_at(i, c8)) = make_uint4(w[pl][0], w[pl][1], w[pl][2], w[pl][3]);
        };
#pragma unroll 1
        for (int n = tid; n < kChunk * DK / 8; n += kThreads) {
            const int i = n / (DK / 8), c8 = n % (DK / 8) * 8;
            write(a.qt, qs, W, i, c8, all);
            if (DELTA) write(a.kt, ks, W, i, c8, true);
            write(a.kh, kc, W + 4 * DK, i, c8, true);
        }
    }
    if (tid < DK) a.decay[unit * DK + tid] = expf(B[tid] + B[DK + tid] + B[2 * DK + tid] + B[3 * DK + tid]);
    // block pairs (I, J <= I) of A and L, 16 x 16 each, one warp per pair
    __nv_bfloat16 *A = a.A + unit * kPlanes * kChunk * kChunk;
    const int g = lane >> 2, t = lane & 3;
    constexpr int kPairsAll = 10, kRounds = (kPairsAll + kWarps - 1) / kWarps, kMats = DELTA ? 2 : 1;
    float acc[kRounds][kMats][2][4] = {};
#pragma unroll
    for (int round = 0; round < kRounds; ++round) {
        const int pair = warp + kWarps * round;
        if (pair >= kPairsAll) break;
        const int I = pair < 1 ? 0 : pair < 3 ? 1 : pair < 6 ? 2 : 3, J = pair - I * (I + 1) / 2;
        if (J < I || !deep[I]) {
            const float *f = J == I ? F + I * DK : I - J == 3 ? F + 6 * DK : F + (3 + J + 1) * DK;  // (not read for I = J + 1)
#pragma unroll 2
            for (int k0 = 0; k0 < DK; k0 += 16) {
                uint32_t b[kPlanes][4];
                frag_b(b, kc, VS, J * kBlock, k0, lane);
                float2 w[2] = {make_float2(1.f, 1.f), make_float2(1.f, 1.f)};
                if (I != J + 1) w[0] = *reinterpret_cast<const float2 *>(f + k0 + 2 * t), w[1] = *reinterpret_cast<const float2 *>(f + k0 + 2 * t + 8);
#pragma unroll
                for (int m = 0; m < kMats; ++m) {
                    const float *src = (m ? ks : qs) + (I * kBlock + g) * VS + k0 + 2 * t;
                    uint32_t x[kPlanes][4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 y = *reinterpret_cast<const float2 *>(src + (e & 1) * 8 * VS + (e >> 1) * 8);
                        frag_pair(x, e, y.x * w[e >> 1].x, y.y * w[e >> 1].y);
                    }
                    // (A of bf16 tensors meets bf16 values only: its steps straight into the sum)
                    if (m == 0 && sizeof(IO) == 2) mma_all<false>(acc[round][m][0], acc[round][m][1], x, b);
                    else mma_all(acc[round][m][0], acc[round][m][1], x, b);
                }
            }
        } else {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i = I * kBlock + g + 8 * (e >> 1), j = J * kBlock + n * 8 + 2 * t + (e & 1);
                    if (j <= i) {
                        const size_t at = ((size_t)p.tok0 * a.Hq + hq) * DK;
                        const float2 x = pair_sums<IO, EXCL>(static_cast<const IO *>(a.q) + at, static_cast<const IO *>(a.k) + at, a.Hq * DK,
                                                             a.g + ((size_t)p.tok0 * a.H + h) * DK, a.H * DK, p.valid, DK, i, j);
                        acc[round][0][n][e] = x.x * a.scale;
                        if (DELTA) acc[round][kMats - 1][n][e] = x.y;
                    }
                }
        }
    }
    if (DELTA) __syncthreads();  // the vectors make room for N
#pragma unroll
    for (int round = 0; round < kRounds; ++round) {
        const int pair = warp + kWarps * round;
        if (pair >= kPairsAll) break;
        const int I = pair < 1 ? 0 : pair < 3 ? 1 : pair < 6 ? 2 : 3, J = pair - I * (I + 1) / 2;
#pragma unroll
        for (int m = 0; m < kMats; ++m)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int i = I * kBlock + g + 8 * half, j = J * kBlock + n * 8 + 2 * t;
                    const int last = m || EXCL ? i - 1 : i;  // A: j <= i (RWKV6: j < i), L: j < i
                    const float x = j <= last ? acc[round][m][n][2 * half] : 0.f, y = j + 1 <= last ? acc[round][m][n][2 * half + 1] : 0.f;
                    if (m) *reinterpret_cast<float2 *>(N + i * kInvStride + j) = make_float2(beta[i] * x, beta[i] * y);
                    else put_planes(A + image_at(i, j), kChunk * kChunk, x, y, all);
                }
    }
    if (EXCL) {
        // the diagonal's bonus term q . (bonus * k), `kEach` threads per token
        constexpr int kEach = kThreads / kChunk;
        __syncthreads();  // (the zeros above are in place)
        const int i = tid / kEach;
        float s = 0.f;
        if (i < p.valid) {
            const size_t r = ((size_t)(p.tok0 + i) * a.Hq + hq) * DK;
#pragma unroll 4
            for (int d = (tid % kEach) * 2; d < DK; d += 2 * kEach) {
                float x[2], y[2];
                load_vec<IO, 2>(static_cast<const IO *>(a.q) + r + d, x);
                load_vec<IO, 2>(static_cast<const IO *>(a.k) + r + d, y);
                s = fmaf(x[0] * y[0], a.bonus[h * DK + d], s), s = fmaf(x[1] * y[1], a.bonus[h * DK + d + 1], s);
            }
        }
#pragma unroll
        for (int o = 1; o < kEach; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (tid % kEach == 0)
#pragma unroll
            for (int pl = 0; pl < kPlanes; ++pl) {
                const __nv_bfloat16 w = __float2bfloat16_rn(s);
                A[pl * kChunk * kChunk + image_at(i, i)] = w;
                s -= __bfloat162float(w);
            }
    }
    if (DELTA) {
        __syncthreads();
        invert_unit_lower(N, T, tid);
        write_inverse(T, beta, a.T + unit * kPlanes * kChunk * kChunk, tid, kThreads);
    }
}

}  // namespace deltalog
