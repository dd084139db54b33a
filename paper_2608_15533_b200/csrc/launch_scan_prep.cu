// Launches of the scan's per-chunk preparation.
#include "scan_launch.cuh"
#include "scan_prep_kernel.cuh"

namespace deltalog {
namespace {

template <int P, int DK, bool DELTA, typename IO>
int launch_scalar(const ScanArgs &a, cudaStream_t s) {
    auto kernel = scan_prep_scalar_kernel<P, DK, DELTA, IO>;
    const size_t smem = PrepScalarSmem<P, DK>::bytes(DELTA);
    if (int rc = ensure_smem(kernel, smem)) return rc;
    return launch_chained(kernel, dim3(a.max_chunks + 1, a.H), 128, smem, s, a);
}

template <int OP, int DK, typename IO>
int launch_vector(const ScanArgs &a, cudaStream_t s) {
    auto kernel = scan_prep_vector_kernel<OP, DK, IO>;
    const size_t smem = PrepVectorSmem<DK>::bytes(OpTraits<OP>::kDeltaRule);
    if (int rc = ensure_smem(kernel, smem)) return rc;
    return launch_chained(kernel, dim3(a.max_chunks + 1, a.H), 2 * DK, smem, s, a);
}

template <int OP>
int launch_vector_op(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s) {
    if (d->io_dtype == DELTALOG_F32) return d->d_k == 128 ? launch_vector<OP, 128, float>(a, s) : launch_vector<OP, 64, float>(a, s);
    return d->d_k == 128 ? launch_vector<OP, 128, __nv_bfloat16>(a, s) : launch_vector<OP, 64, __nv_bfloat16>(a, s);
}

}  // namespace

int launch_scan_prep(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s) {
    if (d->op == DELTALOG_KDA) return launch_vector_op<DELTALOG_KDA>(d, a, s);
    if (d->op == DELTALOG_RWKV6) return launch_vector_op<DELTALOG_RWKV6>(d, a, s);
    if (d->op == DELTALOG_GLA) return launch_vector_op<DELTALOG_GLA>(d, a, s);
#define CALL_PREP(VEC, P, DK, DELTA, IO) return launch_scalar<P, DK, DELTA, IO>(a, s)
    if (op_delta_rule(d->op)) DELTALOG_SCAN_IO(d, CALL_PREP, false, true);
    else DELTALOG_SCAN_IO(d, CALL_PREP, false, false);
#undef CALL_PREP
    return DELTALOG_ERR_UNSUPPORTED_SHAPE;
}

}  // namespace deltalog
