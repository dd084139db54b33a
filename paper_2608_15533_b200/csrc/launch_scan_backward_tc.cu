// Launches of the scan's backward chain for d_v = 128 (tcgen05).
#include "scan_backward_tc_kernel.cuh"
#include "scan_launch.cuh"

namespace deltalog {
namespace {

template <bool VEC, int P, int DK, bool DELTA, typename IO>
int launch_chain(const ScanArgs &a, cudaStream_t s) {
    auto kernel = scan_backward_tc_kernel<VEC, P, DK, DELTA, IO>;
    constexpr size_t smem = BackwardTcSmem<VEC, P, DK, DELTA, IO>::bytes;
    static_assert(smem <= 227 * 1024, "shared memory of one SM");
    if (int rc = ensure_smem(kernel, smem)) return rc;
    return launch_chained(kernel, dim3(a.n * a.H), kTcThreads, smem, s, a);
}

}  // namespace

int launch_scan_backward_tc(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s) {
#define CALL_CHAIN(VEC, P, DK, DELTA, IO) return launch_chain<VEC, P, DK, DELTA, IO>(a, s)
    DELTALOG_SCAN_DISPATCH(d, CALL_CHAIN);
#undef CALL_CHAIN
    return DELTALOG_ERR_UNSUPPORTED_SHAPE;
}

}  // namespace deltalog
