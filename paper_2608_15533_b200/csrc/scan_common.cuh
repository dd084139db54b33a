// Shared pieces of the chunked scan: the arguments of its kernels, the warp-level matrix helpers and the
// split of fp32 operands into bf16 planes.
//
// A sequence is cut into chunks of kChunk tokens.  With G the cumulative log-decay inside a chunk (inclusive;
// a readout of RWKV6 sees the exclusive one) the token recurrence becomes, per chunk and head,
//     A_ij = scale sum_c q_ic k_jc e^(G_ic - G_jc)  (j <= i)      T = (I + L)^-1 diag(beta)
//     L_ij = beta_i sum_c k_ic k_jc e^(G_ic - G_jc) (j < i)       U = T (V - (k e^G) S_0)      (or U = V)
//     O = scale (q e^G) S_0 + A U          S_1 = e^(G_end) S_0 + (k e^(G_end - G))^T U
// A and T of every chunk come from one parallel kernel (scan_prep_kernel), the chain over S from a sequential
// one (scan_forward_kernel).  The backward pass mirrors it: scan_backward_kernel carries dS from the last
// chunk to the first, scan_grad_kernel forms the gradients of q, k, g and beta chunk by chunk in parallel.
//
// Precision: a bf16 value enters the tensor cores exactly.  An fp32 operand enters as three bf16 planes x = x0 + x1 + x2
// (to 2^-26 of its size), and of a product of two such operands the six plane products with i + j <= 2 are summed in
// fp32 accumulators, so a product is as good as one in fp32.  Two planes (three products) leave 2^-18 per operand: the
// states and gate gradients then came out 3e-6 to 4e-5 off, against 5e-8 to 3e-7 of an fp32 computation.  Results that are
// rounded to bf16 and feed nothing else take two planes: 2^-18 vanishes beside their own 2^-9.
#pragma once

#include "common.cuh"

namespace deltalog {

constexpr int kChunk = DELTALOG_SCAN_CHUNK;
constexpr int kPlanes = 3;  // of an fp32 operand
static_assert(kChunk == 64, "the kernels' tiles are written for 64 tokens");

struct ScanArgs {
    // the plan
    const int32_t *starts, *chunk_starts, *chunk_seq;
    const int32_t *slots;  // state index of each row; NULL: the row itself, every row takes part
    int32_t n, max_chunks, max_tokens, num_slots;
    int32_t *status;
    // the problem
    int32_t H, Hq, dv;
    float scale;
    const void *q, *k, *v;  // io dtype
    const float *g, *beta, *bonus;
    const void *dout;
    // workspace, unit = chunk * H + head
    int32_t *order;              // [n] rows, the longest first: the order in which the chain kernels' CTAs take them
    __nv_bfloat16 *qi, *ki;      // scalar decay, fp32 io: images of q and k [chunk * Hq + head][3][64][d_k]
    __nv_bfloat16 *A, *T;        // images [unit][3][64][64]
    float *decay;                // scalar decay: [unit][2][64] e^(G_i), e^(G_end - G_i); per channel: [unit][d_k] e^(G_end)
    __nv_bfloat16 *qt, *kt, *kh; // per-channel decay: images [unit][3][64][d_k]
    float *U, *dV;               // [unit][64][d_v]
    float *S, *dS;               // [unit][d_v][d_k], state in front of the chunk / gradient behind it (transposed)
    // states
    const void *S_in;            // [.., H, d_k, d_v]
    void *S_out;
    int32_t in_bf16, out_bf16;
    const int32_t *fresh;        // rows that start from zero, or NULL
    int32_t *log_len;            // [num_slots, H], emptied for the rows that ran, or NULL
    int32_t keep;                // forward: write S and U for a backward pass
    void *out;                   // [tokens, H, d_v], or NULL
    int32_t clear;               // zeros to the rows of out below max_tokens that no row writes
    // backward
    const float *dS_final;
    float *dS_init;
    void *dq, *dk, *dv_out;
    float *dq_part, *dk_part;    // [tokens, H, d_k] where several value heads share one query / key head
    float *dg, *dbeta, *dbonus_part;
    int32_t wave;                // CTAs of one wave
    // split of long rows (d_v = 128; see ScanSegment): segments per row at most, which of the two passes, the pieces' states
    int32_t split, pass;
    float *pieces;               // [n * H][2 * split - 3][d_k][d_v]
};

// Few rows leave most of the device idle while one chain runs, so long rows are cut into segments.  A segment is an affine map
// of the state in front of it, S_end = M S + E: pass 1 runs the first segment as it is and, for each one behind it but
// the last, two chains side by side -- E from a zero state, and M from the identity with v = 0 (its columns are as many as a
// state's, so it is the same kernel).  scan_join_kernel then carries the state over the segments, and pass 2 runs all but
// the first from the state they really start with.  Two passes of 1 / segments of the row each.
constexpr int kMinSegment = 8;    // chunks
constexpr int kSplitCtas = 148;   // CTAs of pass 1 at most: one per SM, and the same on every host
inline __host__ __device__ int scan_segments(int chunks, int most) {
    const int p = chunks / kMinSegment < most ? chunks / kMinSegment : most;
    return p < 3 ? 1 : p;  // two segments would run one behind the other
}
inline __host__ __device__ int scan_pieces(int segments) { return 2 * segments - 3; }
// Where the state in front of segment s >= 1 is among the pieces: behind the first segment, then in E's place.
__device__ __forceinline__ int scan_piece_of_start(int s) { return s == 1 ? 0 : 2 * s - 3; }

// What a chain CTA runs: chunks [first, end) of its row, from and to where.
struct ScanSegment {
    int seq, h, first, end;
    int from, to;   // piece; -1: the call's own states; to: -2 for nothing
    bool map;       // the chain for M
    bool emit;      // output and what the backward pass reads
};
__device__ __forceinline__ bool scan_segment(const ScanArgs &a, int block, ScanSegment &g) {
    const int each = a.split <= 1 ? 1 : a.pass == 1 ? scan_pieces(a.split) : a.split - 1;
    g.h = block % a.H;
    const int i = block / a.H % each;
    g.seq = a.order[block / a.H / each];
    const int chunks = a.chunk_starts[g.seq + 1] - a.chunk_starts[g.seq];
    const int segments = a.split <= 1 ? 1 : scan_segments(chunks, a.split);
    const int s = a.split <= 1 ? 0 : a.pass == 1 ? (i + 1) / 2 : i + 1;
    if (s >= segments || (a.pass == 1 && s > 0 && s == segments - 1)) return false;
    g.first = (int)((long long)chunks * s / segments), g.end = (int)((long long)chunks * (s + 1) / segments);
    const bool last = s == segments - 1, early = a.pass == 1 && s > 0;  // early: ahead of the state it starts with
    g.map = early && i == 2 * s;
    g.emit = !early;
    g.from = s == 0 || early ? -1 : scan_piece_of_start(s);
    g.to = last ? -1 : a.pass == 1 || a.split <= 1 ? i : -2;
    if (early) g.from = -2;
    return true;
}

// The scan's kernels follow one another on the stream and are launched so that a kernel's CTAs may be set up while the one in
// front retires (a microsecond or two per kernel, which short prompts notice).  First thing, each waits until
// everything in front of it is complete and visible, and then lets its successor be set up.  A kernel that writes states
// does not: a decode step that may start early (DELTALOG_HINT_BASE_UNTOUCHED) lets its own successor start before it has
// itself waited, and that one reads base tiles at once; all that keeps it off these is that the first one starts late.
__device__ __forceinline__ void scan_kernel_begin(bool writes_states = false) {
    asm volatile("griddepcontrol.wait;\n" ::: "memory");
    if (!writes_states) asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
}

// Row and slot of a (sequence, head) unit; false when the unit has nothing to do.
__device__ __forceinline__ bool scan_slot(const ScanArgs &a, int seq, int tid, int &slot) {
    if (!a.slots) {
        slot = seq;
        return true;
    }
    return resolve_slot(a.slots, seq, a.num_slots, a.status, tid, slot);
}

// e^x for x <= 0 that weighs a term as it is: the argument's rounding costs |x| 2^-24 of the weight e^x, at most 2^-25 of the
// largest weight.  (Not for a weight that a factor above one brings back up: see block_vectors.)
__device__ __forceinline__ float decay_exp(float x) { return __expf(x); }

// ---- bf16 planes -------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t pack_bf16(float lo_elem, float hi_elem) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo_elem, hi_elem);
    return *reinterpret_cast<const uint32_t *>(&p);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// x, y -> their packed planes 0 .. N-1, each the bf16 rounding of what the planes in front of it leave.  (Rounded, not cut:
// cutting costs as many instructions, leaves twice as much, and always with the same sign -- sums over long contractions
// were ten times further off.)
template <int N>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t (&w)[N]) {
    float2 r = make_float2(x, y);
#pragma unroll
    for (int p = 0; p < N; ++p) {
        w[p] = pack_bf16(r.x, r.y);
        if (p + 1 < N) r = __ffma2_rn(make_float2(bf16_lo(w[p]), bf16_hi(w[p])), make_float2(-1.f, -1.f), r);
    }
}

// ---- warp-level products -----------------------------------------------------------------------------------
// c += a b, m16n8k16.  Accumulator layout: c[0..1] row lane/4, columns 2(lane%4)+{0,1}; c[2..3] row lane/4 + 8.
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two neighbouring accumulator tiles (16 columns) as the A operand of the next product, in N planes.
template <int N>
__device__ __forceinline__ void acc_to_a(const float (&c0)[4], const float (&c1)[4], uint32_t (&f)[N][4]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float x = r < 2 ? c0[2 * r] : c1[2 * r - 4], y = r < 2 ? c0[2 * r + 1] : c1[2 * r - 3];
        uint32_t w[N];
        split_pair<N>(x, y, w);
#pragma unroll
        for (int p = 0; p < N; ++p) f[p][r] = w[p];
    }
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void stsm4_t(uint32_t addr, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};\n" ::"r"(addr), "r"(r0), "r"(r1), "r"(r2), "r"(r3)
                 : "memory");
}

// The tensor cores cut an accumulator's last bits instead of rounding them: every addition into a sum loses half a unit 2^-23 of
// the partial sum on average, always towards zero.  So the plane products of one step of K = 16 are summed by themselves, the smallest
// first and the leading one last, and what they come to is added to the running sum by an ordinary, rounded addition.  (One
// after the other into the running sum, an fp32 contraction over 128 channels was cut 48 times: 1.2e-6 of a sum of positive
// terms, ten times what fp32 arithmetic leaves.)  That is done for fp32 tensors and, with bf16 ones, for L and
// its inverse.  The order alone leaves states of bf16 tensors 1e-7 to 2e-7 off; with every step apart the chains for d_v = 64 took 2 to 20
// % longer (fp32 tensors: 9 to 15 %).  A sum of several products of planes starts here ...
template <int N>
__device__ __forceinline__ void add_to(float (&c)[N], const float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] += x[i];
}
// ... and c0, c1 += a b adds a k16 x n16 operand b in plane `pb` to it (callers go from the last plane to the first): the planes of
// a whose product with it counts (index sum below LIMIT).
template <int PA, int LIMIT>
__device__ __forceinline__ void mma_planes(float (&c0)[4], float (&c1)[4], const uint32_t (&a)[PA][4], const uint32_t (&b)[4], int pb) {
#pragma unroll
    for (int pa = PA - 1; pa >= 0; --pa)
        if (pa + pb < LIMIT) mma(c0, a[pa], b[0], b[1]), mma(c1, a[pa], b[2], b[3]);
}

// The same for two n16 operands side by side, four accumulators in turn: a product waits 22 cycles
// for the one before it into the same accumulator, and one is issued every eight.
template <int PA, int LIMIT>
__device__ __forceinline__ void mma_planes2(float (&c0)[4], float (&c1)[4], float (&d0)[4], float (&d1)[4], const uint32_t (&a)[PA][4],
                                            const uint32_t (&b)[4], const uint32_t (&e)[4], int pb) {
#pragma unroll
    for (int pa = PA - 1; pa >= 0; --pa)
        if (pa + pb < LIMIT) mma(c0, a[pa], b[0], b[1]), mma(c1, a[pa], b[2], b[3]), mma(d0, a[pa], e[0], e[1]), mma(d1, a[pa], e[2], e[3]);
}

// ---- shared-memory tiles -----------------------------------------------------------------------------------
// A bf16 tile of `kChunk` rows (w = 64 or 128 columns): 64 columns at a time, rows of 128 bytes, the 16-byte units of a
// row permuted by the row's low three bits.  Eight rows at one unit fall into eight different bank groups, and it is the
// 128-byte swizzle of the tensor cores' descriptors.  The workspace holds tiles in this very form ("images"), so a
// chain kernel's load is a plain copy.
__device__ __forceinline__ uint32_t tile_offset(int row, int unit) {
    return (uint32_t)(((unit >> 3) * kChunk + row) * 128 + (((unit & 7) ^ (row & 7)) << 4));
}
__device__ __forceinline__ uint32_t tile_addr(uint32_t base, int row, int unit) { return base + tile_offset(row, unit); }
// Place of element (row, column c) of an image, in elements.
__device__ __forceinline__ int image_at(int row, int c) { return (int)(tile_offset(row, c >> 3) >> 1) + (c & 7); }
// The same for the per-warp slices of 16 columns (32-byte rows).
__device__ __forceinline__ uint32_t slice_addr(uint32_t base, int row, int unit) {
    return base + (uint32_t)(row * 32 + ((unit ^ ((row >> 2) & 1)) << 4));
}

// Operand B (k16 x n16, two n8 tiles: r[0..1], r[2..3]) of a tile stored [n][k] ...
__device__ __forceinline__ void load_b(uint32_t (&r)[4], uint32_t base, int n0, int k0, int lane) {
    const int m = lane >> 3, x = lane & 7;
    ldsm4(r, tile_addr(base, n0 + (m >> 1) * 8 + x, (k0 >> 3) + (m & 1)));
}
// ... and of a tile stored [k][n].
__device__ __forceinline__ void load_b_t(uint32_t (&r)[4], uint32_t base, int k0, int n0, int lane) {
    const int m = lane >> 3, x = lane & 7;
    ldsm4_t(r, tile_addr(base, k0 + (m & 1) * 8 + x, (n0 >> 3) + (m >> 1)));
}
// Operand A (m16 x k16) of a tile stored [m][k] ...
__device__ __forceinline__ void load_a(uint32_t (&r)[4], uint32_t base, int m0, int k0, int lane) {
    const int m = lane >> 3, x = lane & 7;
    ldsm4(r, tile_addr(base, m0 + (m & 1) * 8 + x, (k0 >> 3) + (m >> 1)));
}
// ... and of a tile stored [k][m].
__device__ __forceinline__ void load_a_t(uint32_t (&r)[4], uint32_t base, int k0, int m0, int lane) {
    const int m = lane >> 3, x = lane & 7;
    ldsm4_t(r, tile_addr(base, k0 + (m >> 1) * 8 + x, (m0 >> 3) + (m & 1)));
}
// Operand A of a 16-column slice stored [token k][16]; read as accumulator tiles it is the slice's transpose:
// r[0] row lane/4 tokens k0..7, r[1] row lane/4 + 8, r[2], r[3] the same for tokens k0 + 8..15.
__device__ __forceinline__ void load_slice_t(uint32_t (&r)[4], uint32_t base, int k0, int lane) {
    const int m = lane >> 3, x = lane & 7;
    ldsm4_t(r, slice_addr(base, k0 + (m >> 1) * 8 + x, m & 1));
}

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
template <int N>
__device__ __forceinline__ void frag_a(uint32_t (&f)[N][4], const float *tile, int w, int m0, int k0, int lane) {
    const float *p = tile + (m0 + (lane >> 2)) * w + k0 + 2 * (lane & 3);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float2 x = *reinterpret_cast<const float2 *>(p + (r & 1) * 8 * w + (r >> 1) * 8);
        frag_pair(f, r, x.x, x.y);
    }
}
// ... and of a tile [k][m].
template <int N>
__device__ __forceinline__ void frag_a_t(uint32_t (&f)[N][4], const float *tile, int w, int k0, int m0, int lane) {
    const float *p = tile + (k0 + 2 * (lane & 3)) * w + m0 + (lane >> 2);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float *q = p + (r >> 1) * 8 * w + (r & 1) * 8;
        frag_pair(f, r, q[0], q[w]);
    }
}
// Operand B (k16 x n16) of a tile [n][k] ...
template <int N>
__device__ __forceinline__ void frag_b(uint32_t (&f)[N][4], const float *tile, int w, int n0, int k0, int lane) {
    const float *p = tile + (n0 + (lane >> 2)) * w + k0 + 2 * (lane & 3);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float2 x = *reinterpret_cast<const float2 *>(p + (r >> 1) * 8 * w + (r & 1) * 8);
        frag_pair(f, r, x.x, x.y);
    }
}
// ... and of a tile [k][n] (w = 4 mod 16: no bank conflicts).
template <int N>
__device__ __forceinline__ void frag_b_t(uint32_t (&f)[N][4], const float *tile, int w, int k0, int n0, int lane) {
    const float *p = tile + (k0 + 2 * (lane & 3)) * w + n0 + (lane >> 2);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float *q = p + (r & 1) * 8 * w + (r >> 1) * 8;
        frag_pair(f, r, q[0], q[w]);
    }
}
// c0, c1 += a b over all plane products that count: index sums below the larger number of planes.  APART: summed by themselves
// first.
template <bool APART = true, int PA, int PB>
__device__ __forceinline__ void mma_all(float (&c0)[4], float (&c1)[4], const uint32_t (&a)[PA][4], const uint32_t (&b)[PB][4]) {
    constexpr int kLimit = PA > PB ? PA : PB;
    if constexpr (!APART || kLimit == 1) {
#pragma unroll
        for (int pb = PB - 1; pb >= 0; --pb) mma_planes<PA, kLimit>(c0, c1, a, b[pb], pb);
    } else {
        float x0[4] = {}, x1[4] = {};
#pragma unroll
        for (int pb = PB - 1; pb >= 0; --pb) mma_planes<PA, kLimit>(x0, x1, a, b[pb], pb);
        add_to(c0, x0), add_to(c1, x1);
    }
}

// Asynchronous 16-byte copy that writes zeros when `ok` is false (the source is then not read).
__device__ __forceinline__ void cp_async16_zfill(uint32_t dst, const void *src, bool ok) {
    const int n = ok ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory");
}
// kChunk x w tile of rows `stride` elements apart; rows at and behind `valid` become zeros.
template <int W>
__device__ __forceinline__ void load_tile(uint32_t dst, const __nv_bfloat16 *src, size_t stride, int valid, int tid, int nthreads) {
    constexpr int kUnits = W / 8;
    for (int i = tid; i < kChunk * kUnits; i += nthreads) {
        const int row = i / kUnits, unit = i % kUnits;
        const bool ok = row < valid;
        cp_async16_zfill(tile_addr(dst, row, unit), src + (ok ? (size_t)row * stride + unit * 8 : 0), ok);
    }
}
// An image, `bytes` long.
__device__ __forceinline__ void load_image(uint32_t dst, const void *src, int bytes, int tid, int nthreads) {
    for (int i = tid * 16; i < bytes; i += nthreads * 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst + i), "l"(static_cast<const char *>(src) + i) : "memory");
}
// A warp's 64 x 16 slice of rows `stride` elements apart.
__device__ __forceinline__ void load_slice(uint32_t dst, const __nv_bfloat16 *src, size_t stride, int valid, int lane) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 16 + (lane >> 1), unit = lane & 1;
        const bool ok = row < valid;
        cp_async16_zfill(slice_addr(dst, row, unit), src + (ok ? (size_t)row * stride + unit * 8 : 0), ok);
    }
}
// q or k of a chunk with scalar decay: from the tensor (bf16 io), or the image that prep made of it (fp32 io).
template <int P, int DK>
__device__ __forceinline__ void load_vectors_tile(uint32_t dst, const void *raw, const __nv_bfloat16 *image, const ScanArgs &a, int tok, int chunk, int hq,
                                                  int valid, int tid, int nthreads) {
    if constexpr (P == 1)
        load_tile<DK>(dst, static_cast<const __nv_bfloat16 *>(raw) + ((size_t)tok * a.Hq + hq) * DK, (size_t)a.Hq * DK, valid, tid, nthreads);
    else
        load_image(dst, image + ((size_t)chunk * a.Hq + hq) * P * kChunk * DK, P * kChunk * DK * 2, tid, nthreads);
}

// Transposed accumulators x[8][4] (16 columns of d_v x 64 tokens) to a tensor of rows `stride` elements apart: bf16
// through the warp's staging slice, fp32 directly (eight lanes write one 32-byte sector).
__device__ __forceinline__ void store_slice(__nv_bfloat16 *dst, size_t stride, int valid, const float (&x)[8][4], uint32_t stage, int lane) {
    __syncwarp();
#pragma unroll
    for (int n = 0; n < 8; n += 2) {
        const int m = lane >> 3, r = lane & 7;
        stsm4_t(slice_addr(stage, n * 8 + (m >> 1) * 8 + r, m & 1), pack_bf16(x[n][0], x[n][1]), pack_bf16(x[n][2], x[n][3]),
                pack_bf16(x[n + 1][0], x[n + 1][1]), pack_bf16(x[n + 1][2], x[n + 1][3]));
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = i * 16 + (lane >> 1), unit = lane & 1;
        if (row < valid) {
            uint4 w;
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];\n" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(slice_addr(stage, row, unit)) : "memory");
            *reinterpret_cast<uint4 *>(dst + (size_t)row * stride + unit * 8) = w;
        }
    }
}
__device__ __forceinline__ void store_slice(float *dst, size_t stride, int valid, const float (&x)[8][4], uint32_t, int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int tok = n * 8 + 2 * t + (e & 1);
            if (tok < valid) dst[(size_t)tok * stride + g + (e >> 1) * 8] = x[n][e];
        }
}
// Tokens 16 kb .. + 15 of the warp's 16 columns in the accumulator layout x[2][4]: from the warp's slice of a bf16
// tensor, or straight from an fp32 one.
__device__ __forceinline__ void read_slice(float (&x)[2][4], const __nv_bfloat16 *, size_t, int, uint32_t slice, int kb, int lane) {
    uint32_t f[4];
    load_slice_t(f, slice, kb * 16, lane);
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int r = 0; r < 2; ++r) x[n][2 * r] = bf16_lo(f[2 * n + r]), x[n][2 * r + 1] = bf16_hi(f[2 * n + r]);
}
__device__ __forceinline__ void read_slice(float (&x)[2][4], const float *src, size_t stride, int valid, uint32_t, int kb, int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int tok = kb * 16 + n * 8 + 2 * t + (e & 1);
            x[n][e] = tok < valid ? __ldg(src + (size_t)tok * stride + g + (e >> 1) * 8) : 0.f;
        }
}

// A state tile of this warp: s[n][e] = S[c = 8n + 2t + (e & 1)][v0 + g + 8 (e >> 1)], rows of S d_v apart.
template <int NT>
__device__ __forceinline__ void load_state(float (&s)[NT][4], const void *src, bool is_bf16, size_t off, int dv, int v0, int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const size_t i = off + (size_t)(8 * n + 2 * t + (e & 1)) * dv + v0 + g + 8 * (e >> 1);
            s[n][e] = is_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(src)[i]) : static_cast<const float *>(src)[i];
        }
}
template <int NT>
__device__ __forceinline__ void store_state(const float (&s)[NT][4], void *dst, bool is_bf16, size_t off, int dv, int v0, int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const size_t i = off + (size_t)(8 * n + 2 * t + (e & 1)) * dv + v0 + g + 8 * (e >> 1);
            if (is_bf16) static_cast<__nv_bfloat16 *>(dst)[i] = __float2bfloat16_rn(s[n][e]);
            else static_cast<float *>(dst)[i] = s[n][e];
        }
}
// A state tile to the workspace, transposed [d_v][8 NT], fp32.
template <int NT>
__device__ __forceinline__ void keep_state(float *dst, const float (&s)[NT][4], int v0, int lane) {
    const int g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < 2; ++r)
            *reinterpret_cast<float2 *>(dst + (size_t)(v0 + g + 8 * r) * (8 * NT) + 8 * n + 2 * t) = make_float2(s[n][2 * r], s[n][2 * r + 1]);
}

}  // namespace deltalog
