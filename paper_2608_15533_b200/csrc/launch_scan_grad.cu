// Launches of the scan's per-chunk gradients and of the sums behind them.
#include "scan_grad_kernel.cuh"
#include "scan_launch.cuh"

namespace deltalog {
namespace {

template <int OP, int P, int DK, typename IO, bool TC>
int launch_grad(const deltalog_desc *d, const ScanArgs &args, int rows, float *dbonus, cudaStream_t s) {
    ScanArgs a = args;
    a.wave = device_info().sms;
    auto kernel = scan_grad_kernel<OP, P, DK, IO, TC>;
    const size_t smem = GradSmem<OP, P, DK, IO, TC>::bytes;
    if (int rc = ensure_smem(kernel, smem)) return rc;
    if (int rc = launch_chained(kernel, dim3(a.max_chunks, a.H), kGradThreads, smem, s, a)) return rc;
    const int sms = device_info().sms;
    if (a.H != a.Hq) {
        if (int rc = launch_chained(scan_group_sum_kernel<IO>, dim3(sms * 8), 256, 0, s, a, DK)) return rc;
    }
    if (OP == DELTALOG_RWKV6) {
        if (int rc = launch_chained(scan_bonus_sum_kernel, dim3(a.H), 256, 0, s, a, DK, dbonus)) return rc;
    }
    const int e = (int)sizeof(IO), gate = op_has_gate(d->op) ? 4 * a.H * (op_vec_decay(d->op) ? DK : 1) : 0;
    return launch_chained(scan_tail_kernel, dim3(sms), 256, 0, s, a, rows, a.Hq * DK * e, a.H * a.dv * e, gate, op_delta_rule(d->op) ? 4 * a.H : 0);
}

template <int OP>
int launch_grad_op(const deltalog_desc *d, const ScanArgs &a, int rows, float *dbonus, cudaStream_t s) {
    if (d->io_dtype == DELTALOG_F32)
        return d->d_k == 128 ? launch_grad<OP, 3, 128, float, false>(d, a, rows, dbonus, s) : launch_grad<OP, 3, 64, float, false>(d, a, rows, dbonus, s);
    if (a.dv == 128)  // as the chains: what they keep is laid out for this
        return d->d_k == 128 ? launch_grad<OP, 1, 128, __nv_bfloat16, true>(d, a, rows, dbonus, s)
                             : launch_grad<OP, 1, 64, __nv_bfloat16, true>(d, a, rows, dbonus, s);
    return d->d_k == 128 ? launch_grad<OP, 1, 128, __nv_bfloat16, false>(d, a, rows, dbonus, s)
                         : launch_grad<OP, 1, 64, __nv_bfloat16, false>(d, a, rows, dbonus, s);
}

}  // namespace

int launch_scan_grad(const deltalog_desc *d, const ScanArgs &a, int rows, float *dbonus, cudaStream_t s) {
    switch (d->op) {
        case DELTALOG_GDN: return launch_grad_op<DELTALOG_GDN>(d, a, rows, dbonus, s);
        case DELTALOG_KDA: return launch_grad_op<DELTALOG_KDA>(d, a, rows, dbonus, s);
        case DELTALOG_RWKV6: return launch_grad_op<DELTALOG_RWKV6>(d, a, rows, dbonus, s);
        case DELTALOG_GLA: return launch_grad_op<DELTALOG_GLA>(d, a, rows, dbonus, s);
        default: return launch_grad_op<DELTALOG_RETNET>(d, a, rows, dbonus, s);  // linear attention: null gate
    }
}

}  // namespace deltalog
