// deltalog_build_plan.
#include "launch_common.cuh"
#include "plan_kernel.cuh"

using namespace deltalog;

extern "C" int deltalog_build_plan(const int32_t *lens, const int32_t *slots, const int32_t *log_len, int32_t H, int32_t cap, int32_t num_slots,
                                   int32_t decode_rows, const deltalog_plan *plan, void *stream) {
    if (int rc = validate_plan(plan)) return rc;
    if (plan->n > 0 && !lens) return DELTALOG_ERR_INVALID_ARG;
    if (!plan->totals || !aligned16(plan->totals) || (plan->token_seq && !aligned16(plan->token_seq))) return DELTALOG_ERR_INVALID_ARG;
    if (log_len && (H <= 0 || num_slots <= 0)) return DELTALOG_ERR_INVALID_ARG;
    if (log_len && (cap < 1 || cap > kMaxCapHost)) return DELTALOG_ERR_CAP_RANGE;
    PlanArgs a{lens, slots, log_len, plan->n, H, cap, num_slots, decode_rows, plan->max_tokens, scan_max_chunks(plan->n, plan->max_tokens),
               plan->starts, plan->chunk_starts, plan->chunk_seq, plan->token_seq, plan->scan_slots, plan->append_slots, plan->merge_slots,
               plan->totals};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    // a thread's share of the tables: four tokens and a row or so each, one wave of CTAs at most
    const long long work = (plan->token_seq ? (plan->max_tokens + 3ll) / 4 : 0) + a.n + a.max_chunks;
    const long long ctas = (work + kPlanThreads - 1) / kPlanThreads;
    if (a.n <= kPlanShared) {
        // few rows: fewer threads meet at the barriers sooner; many: more share the scan that every CTA runs.  us per call, back
        // to back in a graph, with 256 / 512 / 1024 threads: 64 requests 4.3 / 4.6 / 5.5, 512 requests (51k tokens) 5.0 / 5.1 / 6.3,
        // 2048 requests 6.7 / 6.4 / 7.4, 4096 requests 9.3 / 7.5 / 8.2, 8192 requests 13.8 / 10.5 / 9.9, 20k documents 40 / 25 / 19
        const int threads = a.n <= 512 ? 256 : a.n <= 4096 ? 512 : kPlanThreads;
        const long long need = (work + threads - 1) / threads;
        const int grid = (int)(need < 1 ? 1 : need > device_info().sms ? device_info().sms : need);
        const size_t smem = (size_t)2 * (a.n + 1) * sizeof(int32_t);
        if (int rc = ensure_smem(plan_kernel, smem)) return rc;
        plan_kernel<<<grid, threads, smem, s>>>(a);
        return finish_launch();
    }
    plan_offsets_kernel<<<1, 1024, 0, s>>>(a);
    if (int rc = finish_launch()) return rc;
    const int grid = (int)(ctas > device_info().sms ? device_info().sms : ctas);
    plan_tables_kernel<<<grid, kPlanThreads, 0, s>>>(a);
    return finish_launch();
}
