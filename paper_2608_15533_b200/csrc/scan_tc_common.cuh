// tcgen05 pieces of the scan's chain kernels for d_v = 128: bf16 products whose A operand is in tensor memory.
#pragma once

#include "decode_pipelined.cuh"  // mbarriers, bulk copies, bounded waits
#include "scan_common.cuh"

namespace deltalog {

constexpr int kTcThreads = 512;
constexpr int kTmemCols = 512;
// CTAs of the tcgen05 kernels take all of an SM's tensor memory: the request keeps a second one off the SM.
constexpr size_t kTcMinSmem = 120 * 1024;

// Shared-memory descriptor of an image (128-byte swizzle).  K-major: rows are n, eight rows every 1024 bytes.  MN-major:
// rows are k, eight rows every 1024 bytes, the next 64 columns of n `half` bytes on.
__device__ __forceinline__ uint64_t image_desc(uint32_t addr, int half = kChunk * 128) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(half >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) |
           ((uint64_t)2 << 61);
}
// Instruction descriptor: fp32 accumulators, bf16 A (K-major) and B, M = 128.
__device__ __forceinline__ constexpr uint32_t tc_idesc(int n, bool b_mn_major) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}
// D[tmem] (+)= A[tmem] B for one step of K = 16.
__device__ __forceinline__ void tc_mma(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
        : "memory");
}
// One lane of a convergent warp.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n .reg .pred q;\n elect.sync _|q, 0xffffffff;\n selp.u32 %0, 1, 0, q;\n}\n" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }

// 16 consecutive columns of the thread's lane.  The load and the wait for it are one statement: the registers hold nothing
// before the wait, and between two statements the compiler may move or spill them.
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float (&x)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};\n" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
                 "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }
// 32 or 16 values as N planes of packed pairs: plane p to columns addr + p * plane onwards.
template <int N, int COUNT>
__device__ __forceinline__ void tmem_st_planes(uint32_t addr, int plane, const float (&x)[COUNT]) {
#pragma unroll
    for (int j = 0; j < COUNT; j += 16) {
        uint32_t w[N][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t y[N];
            split_pair<N>(x[j + 2 * i], x[j + 2 * i + 1], y);
#pragma unroll
            for (int p = 0; p < N; ++p) w[p][i] = y[p];
        }
#pragma unroll
        for (int p = 0; p < N; ++p) tmem_st8(addr + p * plane + j / 2, w[p]);
    }
}

// The plane products (index sum LO <= pa + pb < HI) of A (planes A_PLANE columns apart) with the image planes PB0 .. PB1 - 1
// of B (`b`: plane PB0), issued by one thread.  Everything but the addresses is a constant and the loops unroll: a product of
// 128 x 64 x 16 takes the tensor core 32 cycles, and with descriptors put together for each the issuing thread needed 60.
// The smallest products go first, where the sum is still small: the tensor cores cut an accumulator's last bits (see mma_planes), and behind
// the leading products the others cut the sum forty times more (states 6e-7 off instead of 8e-8).
// K-major B (rows are n): a step of 16 is 32 bytes of a row, 64 columns per image half.  MN-major B (rows are k): 16 rows.
// SPLIT: B's rows are two operands of N / 2 = 64, and D's first half is a sum already while the second starts here.
template <int PA, int PB0, int PB1, int LO, int HI, bool MN, int STEPS, int N, int A_PLANE, int B_PLANE, int HALF = kChunk * 128, bool SPLIT = false>
__device__ __forceinline__ void tc_product(uint32_t d, uint32_t a, uint32_t b, bool first = true) {
    const uint64_t desc = image_desc(b, HALF);
    bool clear = first, split = SPLIT;
#pragma unroll
    for (int order = PA + PB1 - 2; order >= 0; --order)
#pragma unroll
        for (int pb = PB0; pb < PB1; ++pb) {
            const int pa = order - pb;
            if (pa < 0 || pa >= PA || order < LO || order >= HI) continue;
#pragma unroll
            for (int k = 0; k < STEPS; ++k) {
                const int off = (pb - PB0) * B_PLANE + (MN ? k * 2048 : (k >> 2) * HALF + (k & 3) * 32);
                if (split) {
                    tc_mma(d, a + pa * A_PLANE + k * 8, desc + (off >> 4), tc_idesc(N / 2, MN), true);
                    tc_mma(d + N / 2, a + pa * A_PLANE + k * 8, desc + ((off + kChunk * 128) >> 4), tc_idesc(N / 2, MN), false);
                    split = false;
                } else {
                    tc_mma(d, a + pa * A_PLANE + k * 8, desc + (off >> 4), tc_idesc(N, MN), !clear);
                }
                clear = false;
            }
        }
}
// The same with a lower-triangular 64 x 64 matrix, D[., i] += sum_j A[., j] M[i, j]: step k (16 j) reaches the columns i >= 16 k.
template <int PA, int PB, int LIMIT, int A_PLANE>
__device__ __forceinline__ void tc_product_lower(uint32_t d, uint32_t a, uint32_t b) {
    const uint64_t desc = image_desc(b);
    bool clear = true;
#pragma unroll
    for (int order = LIMIT - 1; order >= 0; --order)
#pragma unroll
        for (int pb = 0; pb < PB; ++pb) {
            const int pa = order - pb;
            if (pa < 0 || pa >= PA) continue;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int off = pb * (kChunk * kChunk * 2) + k * 2048 + k * 32;
                tc_mma(d + 16 * k, a + pa * A_PLANE + k * 8, desc + (off >> 4), tc_idesc(64 - 16 * k, false), !clear);
                clear = false;
            }
        }
}
// And with its transpose, D[., j] += sum_i A[., i] M[i, j]: step k (16 i) reaches the columns j < 16 (k + 1).  Steps go down so
// that the first one covers all of D.
template <int PA, int PB, int LIMIT, int A_PLANE>
__device__ __forceinline__ void tc_product_upper(uint32_t d, uint32_t a, uint32_t b, bool first = true) {
    const uint64_t desc = image_desc(b);
    bool clear = first;
#pragma unroll
    for (int order = LIMIT - 1; order >= 0; --order)
#pragma unroll
        for (int pb = 0; pb < PB; ++pb) {
            const int pa = order - pb;
            if (pa < 0 || pa >= PA) continue;
#pragma unroll
            for (int k = 3; k >= 0; --k) {
                const int off = pb * (kChunk * kChunk * 2) + k * 2048;
                tc_mma(d, a + pa * A_PLANE + k * 8, desc + (off >> 4), tc_idesc(16 * (k + 1), true), !clear);
                clear = false;
            }
        }
}

// A chain CTA's barriers and tensor memory: set up by the whole CTA, taken down by it.
struct TcBlock {
    uint32_t tmem;
    uint32_t bars;          // shared address of the mbarriers
    volatile int *abort_flag;
};
// words: [0, 12) mbarriers, 12 tensor-memory slot, 14 abort flag, 15 flag of the waits after an abort
constexpr int kTcControlBytes = 128;
__device__ __forceinline__ TcBlock tc_setup(unsigned char *control, int bars, int tid) {
    TcBlock b;
    uint32_t *slot = reinterpret_cast<uint32_t *>(control + 96);
    b.bars = smem_addr(control);
    b.abort_flag = reinterpret_cast<volatile int *>(control + 104);
    if (tid < 32) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_addr(slot)), "r"(kTmemCols));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::);
    }
    if (tid == 0) {
        for (int i = 0; i < bars; ++i) mbar_init(b.bars + 8u * i, 1);
        b.abort_flag[0] = b.abort_flag[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    b.tmem = __shfl_sync(0xffffffffu, *slot, 0);
    return b;
}
__device__ __forceinline__ void tc_teardown(const TcBlock &b, int tid) {
    tc_fence_before();
    __syncthreads();
    if (tid < 32) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(b.tmem), "r"(kTmemCols));
}

// ---- what the chains keep for the per-chunk gradients (bf16 io) ------------------------------------------------
// Two planes take fp32's room and are operands as they stand.  States: [plane][c / 8][v][c % 8], 16 bytes a unit: the lanes of a
// chain's warp are neighbouring v, so a warp's store is four whole lines.  (As rows v of 128 bytes, swizzled, every lane wrote
// into a line of its own, 32 cycles a store: 4k of the 14k cycles of a chunk.)  U: an image of 64 tokens by 128 columns v.
// dV: rows of 128 columns.
constexpr int kKeptGroup = 128 * 16;  // bytes of eight channels of a state
__device__ __forceinline__ int kept_state_at(int c, int v) { return (c >> 3) * kKeptGroup + v * 16 + (c & 7) * 2; }
template <int DK, int HC>
__device__ __forceinline__ void keep_state_planes(void *dst, const float (&s)[HC], int v, int c0) {
    unsigned char *base = static_cast<unsigned char *>(dst);
#pragma unroll
    for (int i = 0; i < HC; i += 8) {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t w[2];
            split_pair<2>(s[i + 2 * j], s[i + 2 * j + 1], w);
            hi[j] = w[0], lo[j] = w[1];
        }
        unsigned char *at = base + kept_state_at(c0 + i, v);
        *reinterpret_cast<uint4 *>(at) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        *reinterpret_cast<uint4 *>(at + DK * 256) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
}
// D[., c] = sum_v A[., v] S[v][c] with the two planes of a kept state: c-major without a swizzle, core matrices of 8 v by 16
// bytes, the next v 128 bytes on, the next c a group.
template <int PA, int DK>
__device__ __forceinline__ void tc_product_state(uint32_t d, uint32_t a, uint32_t b) {
    const uint64_t desc = (uint64_t)((b & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 16) | ((uint64_t)(kKeptGroup >> 4) << 32) | ((uint64_t)1 << 46);
    bool clear = true;
#pragma unroll
    for (int order = 1; order >= 0; --order)
#pragma unroll
        for (int pb = 0; pb < 2; ++pb) {
            const int pa = order - pb;
            if (pa < 0 || pa >= PA) continue;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                tc_mma(d, a + pa * 64 + k * 8, desc + ((pb * DK * 256 + k * 256) >> 4), tc_idesc(DK, true), !clear);
                clear = false;
            }
        }
}
// Place of (token, column v) in U's image / dV's rows, in bytes.
__device__ __forceinline__ int kept_u_at(int tok, int v) { return (v >> 6) * (kChunk * 128) + tok * 128 + ((((v >> 3) & 7) ^ (tok & 7)) << 4) + (v & 7) * 2; }
__device__ __forceinline__ int kept_dv_at(int tok, int v) { return tok * 256 + v * 2; }
// Values of column v for COUNT tokens from t0 on as planes.  Lanes in pairs: the even one takes a pair's first token, the odd
// one its second, two neighbouring columns each.
template <bool IMAGE, int COUNT>
__device__ __forceinline__ void keep_value_planes(void *dst, const float (&u)[COUNT], int t0, int v) {
    const bool odd = v & 1;
#pragma unroll
    for (int i = 0; i < COUNT; i += 2) {
        const float got = __shfl_xor_sync(0xffffffffu, odd ? u[i] : u[i + 1], 1);
        uint32_t w[2];
        split_pair<2>(odd ? got : u[i], odd ? u[i + 1] : got, w);
        const int tok = t0 + i + (odd ? 1 : 0), at = IMAGE ? kept_u_at(tok, v & ~1) : kept_dv_at(tok, v & ~1);
        unsigned char *p = static_cast<unsigned char *>(dst) + at;
        *reinterpret_cast<uint32_t *>(p) = w[0];
        *reinterpret_cast<uint32_t *>(p + kChunk * 256) = w[1];
    }
}

__device__ __forceinline__ void l2_prefetch(const void *p, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;\n" ::"l"(p), "r"(bytes) : "memory");
}
// 16 lanes x 8 N columns in the accumulator layout of mma.sync: x[n][0..1] lane t/4, columns 8 n + 2 (t % 4) + {0, 1}, x[n][2..3]
// lane t/4 + 8.
__device__ __forceinline__ void tmem_ld_frag(uint32_t addr, float (&x)[4][4]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i >> 2][i & 3] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_ld_frag(uint32_t addr, float (&x)[2][4]) {
    uint32_t r[8];
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
        : "r"(addr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i >> 2][i & 3] = __uint_as_float(r[i]);
}

// A tile of 64 tokens x 128 columns of a bf16 tensor to and from shared memory, rows of 256 bytes.
__device__ __forceinline__ void tc_load_rows(uint32_t dst, const __nv_bfloat16 *src, size_t stride, int valid, int tid) {
#pragma unroll
    for (int i = 0; i < kChunk * 16 / kTcThreads; ++i) {
        const int r = (i * kTcThreads + tid) >> 4, u = tid & 15;
        const bool ok = r < valid;
        cp_async16_zfill(dst + r * 256 + u * 16, src + (ok ? (size_t)r * stride + u * 8 : 0), ok);
    }
}
// A chunk's q or k of a bf16 tensor as an operand: column halves HALF bytes apart.
template <int DK, int HALF>
__device__ __forceinline__ void tc_load_operand(uint32_t dst, const void *src, size_t at, size_t stride, int valid, int tid) {
    constexpr int kUnits = DK / 8;
    const __nv_bfloat16 *p = static_cast<const __nv_bfloat16 *>(src) + at;
#pragma unroll
    for (int i = 0; i < kChunk * kUnits / kTcThreads; ++i) {
        const int r = (i * kTcThreads + tid) / kUnits, u = tid % kUnits;
        const bool ok = r < valid;
        cp_async16_zfill(dst + (u >> 3) * HALF + r * 128 + (((u & 7) ^ (r & 7)) << 4), p + (ok ? (size_t)r * stride + u * 8 : 0), ok);
    }
}
// Row `r` of the tile, asynchronously, by one thread (the tile's writers have fenced towards the async proxy and met at a
// barrier).  Every warp's first four lanes take a row each: a warp issues such copies one after the other.
__device__ __forceinline__ void tc_store_row(__nv_bfloat16 *dst, size_t stride, int valid, uint32_t src, int r) {
    if (r < valid)
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], 256;\n" ::"l"(dst + (size_t)r * stride), "r"(src + r * 256) : "memory");
    asm volatile("cp.async.bulk.commit_group;\n" ::: "memory");
}
__device__ __forceinline__ void tc_stores_read() { asm volatile("cp.async.bulk.wait_group.read 0;\n" ::: "memory"); }
__device__ __forceinline__ void tc_stores_done() { asm volatile("cp.async.bulk.wait_group 0;\n" ::: "memory"); }
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }

}  // namespace deltalog
