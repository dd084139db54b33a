// Launches of the scan's forward chain.
#include "scan_forward_kernel.cuh"
#include "scan_launch.cuh"

namespace deltalog {
namespace {

template <bool VEC, int P, int DK, bool DELTA, typename IO>
int launch_chain(const ScanArgs &a, cudaStream_t s) {
    auto kernel = scan_forward_kernel<VEC, P, DK, DELTA, IO>;
    const int warps = scan_chain_warps(a.n * a.H);
    const size_t smem = ForwardSmem<VEC, P, DK, DELTA, IO>::bytes(warps);
    if (int rc = ensure_smem(kernel, smem)) return rc;
    return launch_chained(kernel, dim3(a.n * a.H, 4 / warps), warps * 32, smem, s, a);
}

}  // namespace

int launch_scan_forward(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s) {
    if (a.dv == 128) return launch_scan_forward_tc(d, a, s);
#define CALL_CHAIN(VEC, P, DK, DELTA, IO) return launch_chain<VEC, P, DK, DELTA, IO>(a, s)
    DELTALOG_SCAN_DISPATCH(d, CALL_CHAIN);
#undef CALL_CHAIN
    return DELTALOG_ERR_UNSUPPORTED_SHAPE;
}

}  // namespace deltalog
