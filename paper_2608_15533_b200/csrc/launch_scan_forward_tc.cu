// Launches of the scan's forward chain for d_v = 128 (tcgen05).
#include "scan_forward_tc_kernel.cuh"
#include "scan_launch.cuh"

namespace deltalog {
namespace {

template <bool VEC, int P, int DK, bool DELTA, typename IO, bool KEEP>
int launch_chain(const ScanArgs &a, cudaStream_t s) {
    auto kernel = scan_forward_tc_kernel<VEC, P, DK, DELTA, IO, KEEP>;
    constexpr size_t smem = ForwardTcSmem<VEC, P, DK, DELTA, IO>::bytes;
    static_assert(smem <= 227 * 1024, "shared memory of one SM");
    if (int rc = ensure_smem(kernel, smem)) return rc;
    if (a.split <= 1) return launch_chained(kernel, dim3(a.n * a.H), kTcThreads, smem, s, a);
    ScanArgs b = a;
    b.pass = 1;
    if (int rc = launch_chained(kernel, dim3(a.n * a.H * scan_pieces(a.split)), kTcThreads, smem, s, b)) return rc;
    constexpr size_t join_smem = JoinSmem<DK>::bytes;
    if (int rc = ensure_smem(scan_join_kernel<DK>, join_smem)) return rc;
    if (int rc = launch_chained(scan_join_kernel<DK>, dim3(a.n * a.H, 128 / kJoinCols), DK, join_smem, s, a)) return rc;
    b.pass = 2;
    return launch_chained(kernel, dim3(a.n * a.H * (a.split - 1)), kTcThreads, smem, s, b);
}

}  // namespace

int launch_scan_forward_tc(const deltalog_desc *d, const ScanArgs &a, cudaStream_t s) {
#define CALL_CHAIN(VEC, P, DK, DELTA, IO) return a.keep ? launch_chain<VEC, P, DK, DELTA, IO, true>(a, s) : launch_chain<VEC, P, DK, DELTA, IO, false>(a, s)
    DELTALOG_SCAN_DISPATCH(d, CALL_CHAIN);
#undef CALL_CHAIN
    return DELTALOG_ERR_UNSUPPORTED_SHAPE;
}

}  // namespace deltalog
