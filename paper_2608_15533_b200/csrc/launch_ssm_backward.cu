// Launches of the state space scan's backward pass.
#include "ssm_backward_kernel.cuh"
#include "ssm_launch.cuh"

namespace deltalog {

namespace {

template <typename IO, int N>
int backward(const SsmArgs &a, cudaStream_t s) {
    static_assert(SsmBackward<IO, N, false>::kCtas == ssm_on_sm(sizeof(IO) == 4, N, kSsmBack), "a wave is what the cuts take it for");
    const unsigned cols = (unsigned)(a.G * a.blocks);
    if (a.spans > 1) {
        auto local = ssm_backward_kernel<IO, N, true>;
        const size_t smem = sizeof(typename SsmBackward<IO, N, true>::Shared);
        if (int rc = ensure_smem(local, smem)) return rc;
        local<<<dim3(cols, (unsigned)a.parts), kSsmThreads, smem, s>>>(a);
        if (int rc = finish_launch()) return rc;
        if (int rc = launch_ssm_join<true>(a, N, s)) return rc;
    }
    const unsigned rest = a.dS_init ? ssm_empty_ctas(a.rows.n) : 0;
    if (a.spans + rest > 0) {
        auto kernel = ssm_backward_kernel<IO, N, false>;
        const size_t smem = sizeof(typename SsmBackward<IO, N, false>::Shared);
        if (int rc = ensure_smem(kernel, smem)) return rc;
        kernel<<<dim3(cols, (unsigned)a.spans + rest), kSsmThreads, smem, s>>>(a);
        if (int rc = finish_launch()) return rc;
    }
    const long long token_blocks = ssm_ceil((long long)a.total_rows * a.G * (2 * N / 4), 64), param_blocks = ssm_ceil((long long)a.D_ * (N + 2), 256);
    if (token_blocks + param_blocks > 0x7fffffffll) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    ssm_sums_kernel<IO, N><<<(unsigned)(token_blocks + param_blocks), 256, 0, s>>>(a, token_blocks);
    return finish_launch();
}

}  // namespace

int launch_ssm_backward(const deltalog_ssm_desc *d, const SsmArgs &a, cudaStream_t s) {
#define CALL(IO, N) return backward<IO, N>(a, s)
    SSM_DISPATCH(d, CALL);
#undef CALL
}

}  // namespace deltalog
