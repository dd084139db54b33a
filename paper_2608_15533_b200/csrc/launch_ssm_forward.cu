// Launches of the state space scan's forward pass and of its single-token form.
#include "ssm_forward_kernel.cuh"
#include "ssm_launch.cuh"

namespace deltalog {

namespace {

template <typename IO, int N, bool WIDE>
int forward(const SsmArgs &a, cudaStream_t s) {
    static_assert(SsmForward<IO, N, WIDE>::kCtas == ssm_on_sm(sizeof(IO) == 4, N, WIDE ? kSsmWide : kSsmNarrow), "a wave is what the cuts take it for");
    const size_t smem = sizeof(typename SsmForward<IO, N, WIDE>::Shared);
    const unsigned cols = (unsigned)(a.G * a.blocks);
    if (a.spans > 1) {
        auto local = ssm_forward_kernel<IO, N, true, WIDE>;
        if (int rc = ensure_smem(local, smem)) return rc;
        local<<<dim3(cols, (unsigned)((a.spans - 1) * (a.span / a.part))), kSsmThreads, smem, s>>>(a);
        if (int rc = finish_launch()) return rc;
        if (int rc = launch_ssm_join<false>(a, N, s)) return rc;
    }
    auto kernel = ssm_forward_kernel<IO, N, false, WIDE>;
    if (int rc = ensure_smem(kernel, smem)) return rc;
    // more CTAs behind them for the rows without tokens, whose states a training call hands on
    const unsigned rest = a.S_out && !a.slots ? ssm_empty_ctas(a.rows.n) : 0;
    if (a.spans + rest == 0) return DELTALOG_OK;
    kernel<<<dim3(cols, (unsigned)a.spans + rest), kSsmThreads, smem, s>>>(a);
    return finish_launch();
}

template <typename IO, int N>
int step(const SsmArgs &a, cudaStream_t s) {
    const int cols = (int)ssm_ceil(a.D_, kSsmWarps * 32 / (N / 8));
    constexpr int run = 4;  // 125 rows of 4096 channels with 2, 4, 8, 16 rows a CTA: 17.1, 16.3, 15.8, 20.6 us
    const long long grid = ssm_ceil(a.total_rows, run) * cols;
    if (grid > 0x7fffffffll) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    ssm_step_kernel<IO, N><<<(unsigned)grid, kSsmThreads, 0, s>>>(a, cols, run);
    return finish_launch();
}

}  // namespace

int launch_ssm_forward(const deltalog_ssm_desc *d, const SsmArgs &a, cudaStream_t s) {
#define CALL(IO, N) return a.wide ? forward<IO, N, true>(a, s) : forward<IO, N, false>(a, s)
    SSM_DISPATCH(d, CALL);
#undef CALL
}

int launch_ssm_step(const deltalog_ssm_desc *d, const SsmArgs &a, cudaStream_t s) {
#define CALL(IO, N) return step<IO, N>(a, s)
    SSM_DISPATCH(d, CALL);
#undef CALL
}

}  // namespace deltalog
