// Launches of the scan's per-chunk preparation.
#include "scan_launch.cuh"
#include "scan_prep_kernel.cuh"

namespace deltalog {
namespace {

// An fp32 tensor as bf16 planes.
__global__ void __launch_bounds__(256) split_planes_kernel(const float *x, __nv_bfloat16 *out, size_t pairs) {
    for (size_t i = blockIdx.x * 256ull + threadIdx.x; i < pairs; i += gridDim.x * 256ull) {
        const float2 v = reinterpret_cast<const float2 *>(x)[i];
        put_planes(out + 2 * i, 2 * pairs, v.x, v.y);
    }
}

template <int P, int DK, bool DELTA>
int launch_scalar(const ScanArgs &a, cudaStream_t s) {
    auto kernel = scan_prep_scalar_kernel<P, DK, DELTA>;
    const size_t smem = PrepScalarSmem<P, DK>::bytes(DELTA);
    if (int rc = ensure_smem(kernel, smem)) return rc;
    kernel<<<dim3(a.max_chunks, a.H), 128, smem, s>>>(a);
    return finish_launch();
}

template <int OP, int DK, typename IO>
int launch_vector(const ScanArgs &a, cudaStream_t s) {
    auto kernel = scan_prep_vector_kernel<OP, DK, IO>;
    const size_t smem = PrepVectorSmem<DK>::bytes(OpTraits<OP>::kDeltaRule);
    if (int rc = ensure_smem(kernel, smem)) return rc;
    kernel<<<dim3(a.max_chunks, a.H), 2 * DK, smem, s>>>(a);
    return finish_launch();
}

template <int OP>
int launch_vector_op(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s) {
    if (d->io_dtype == DELTALOG_F32) return d->d_k == 128 ? launch_vector<OP, 128, float>(a, s) : launch_vector<OP, 64, float>(a, s);
    return d->d_k == 128 ? launch_vector<OP, 128, __nv_bfloat16>(a, s) : launch_vector<OP, 64, __nv_bfloat16>(a, s);
}

}  // namespace

int launch_scan_split(const float *x, __nv_bfloat16 *planes, size_t elements, cudaStream_t s) {
    const size_t pairs = elements / 2, ctas = (pairs + 255) / 256;
    if (pairs == 0) return DELTALOG_OK;
    split_planes_kernel<<<(unsigned)(ctas < 4096 ? ctas : 4096), 256, 0, s>>>(x, planes, pairs);
    return finish_launch();
}

int launch_scan_prep(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s) {
    if (d->op == DELTALOG_KDA) return launch_vector_op<DELTALOG_KDA>(d, a, s);
    if (d->op == DELTALOG_RWKV6) return launch_vector_op<DELTALOG_RWKV6>(d, a, s);
    if (d->op == DELTALOG_GLA) return launch_vector_op<DELTALOG_GLA>(d, a, s);
#define CALL_PREP(VEC, P, DK, DELTA, IO) return launch_scalar<P, DK, DELTA>(a, s)
    if (op_delta_rule(d->op)) DELTALOG_SCAN_IO(d, CALL_PREP, false, true);
    else DELTALOG_SCAN_IO(d, CALL_PREP, false, false);
#undef CALL_PREP
    return DELTALOG_ERR_UNSUPPORTED_SHAPE;
}

}  // namespace deltalog
