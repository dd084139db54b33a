// deltalog_conv_*: argument checks, grids, launches.
#include "conv_kernel.cuh"
#include "launch_common.cuh"
#include "validate.h"

using namespace deltalog;

namespace {

int validate_conv(const deltalog_conv_desc *d, const void *x, int64_t x_stride, const float *weight, const float *bias) {
    if (!d || d->channels <= 0 || (d->io_dtype != DELTALOG_F32 && d->io_dtype != DELTALOG_BF16)) return DELTALOG_ERR_INVALID_ARG;
    if (d->channels % 8 || d->width < 2 || d->width > 4) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    if (!x || !weight || !aligned16(x) || !aligned16(weight) || !aligned16(bias)) return DELTALOG_ERR_INVALID_ARG;
    if (x_stride < d->channels || x_stride % (d->io_dtype == DELTALOG_F32 ? 4 : 8)) return DELTALOG_ERR_INVALID_ARG;
    return DELTALOG_OK;
}

int conv_columns(const deltalog_conv_desc *d) { return (d->channels / kConvVec + 31) / 32; }

ConvArgs conv_args(const deltalog_conv_desc *d, const void *x, int64_t x_stride, const float *weight, const float *bias) {
    ConvArgs a = {};
    a.x = x, a.x_stride = x_stride, a.w = weight, a.bias = bias;
    a.C = d->channels, a.silu = d->silu != 0, a.num_slots = d->num_slots;
    return a;
}

void conv_plan(ConvArgs &a, const deltalog_plan *p) {
    a.rows = Rows{p->starts, p->token_seq, p->n};
    a.max_tokens = p->max_tokens;
}

// A run reads inputs that another run owns: the output must not lie over them.
bool conv_overlaps(const deltalog_conv_desc *d, const void *x, int64_t x_stride, const void *out, int32_t tokens) {
    const uint64_t size = d->io_dtype == DELTALOG_F32 ? 4 : 2, t = tokens;
    const uint64_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(out);
    return t > 0 && a < b + t * d->channels * size && b < a + ((t - 1) * x_stride + d->channels) * size;
}

constexpr int kWarpsPerCta = kConvThreads / 32;
long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// FN<io type, width>
#define CONV_DISPATCH(d, CALL)                                                        \
    do {                                                                              \
        if ((d)->io_dtype == DELTALOG_F32) { CONV_WIDTH(float, d, CALL); }            \
        else { CONV_WIDTH(__nv_bfloat16, d, CALL); }                                  \
    } while (0)
#define CONV_WIDTH(IO, d, CALL)                                                       \
    if ((d)->width == 2) { CALL(IO, 2); } else if ((d)->width == 3) { CALL(IO, 3); } else { CALL(IO, 4); }

int conv_packed(const deltalog_conv_desc *d, ConvArgs &a, cudaStream_t s) {
    const int cols = conv_columns(d);
    // A run of 8 tokens reads 3 more than it owns and looks its row up: the longer the better, as long as every SM has sixty
    // warps to take (three waves).
    const long long warps = (long long)cols * a.max_tokens / (60ll * device_info().sms);
    a.run = warps >= 128 ? 128 : warps >= 64 ? 64 : warps >= 32 ? 32 : 8;
    const long long heads = ceil_div(a.rows.n, kWarpsPerCta), runs = ceil_div(ceil_div(a.max_tokens, a.run), kWarpsPerCta);
    const long long grid = (heads + runs) * cols;
    if (grid > 0x7fffffffll) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
#define CALL(IO, W) conv_forward_kernel<IO, W><<<(unsigned)grid, kConvThreads, 0, s>>>(a, cols, heads)
    CONV_DISPATCH(d, CALL);
#undef CALL
    return finish_launch();
}

// Tokens per warp of the backward pass and the blocks that they make: sixteen blocks an SM, so that the partial sums stay a
// few percent of the tokens' bytes however long the sequences are.
struct ConvSplit { int run; long long groups; };
ConvSplit conv_split(const deltalog_conv_desc *d, int32_t rows) {
    // (148 SMs whatever the device: the workspace's size must not depend on which device is current)
    const long long most = ceil_div(148 * 16, conv_columns(d));
    const long long run = ceil_div(rows, most * kWarpsPerCta);
    ConvSplit c;
    c.run = (int)(run < 16 ? 16 : run);
    c.groups = ceil_div(rows, (long long)c.run * kWarpsPerCta);
    return c;
}

}  // namespace

extern "C" {

int deltalog_conv_step(const deltalog_conv_desc *desc, void *window, const void *x, int64_t x_stride, const float *weight, const float *bias,
                       const int32_t *slot_idx, int32_t B, void *out, int32_t *status, void *stream) {
    if (int rc = validate_conv(desc, x, x_stride, weight, bias)) return rc;
    if (desc->num_slots <= 0 || B < 0 || !window || !out || !aligned16(window) || !aligned16(out)) return DELTALOG_ERR_INVALID_ARG;
    if (!slot_idx && B > desc->num_slots) return DELTALOG_ERR_INVALID_ARG;
    if (B == 0) return DELTALOG_OK;
    ConvArgs a = conv_args(desc, x, x_stride, weight, bias);
    a.init = window, a.final = window, a.out = out, a.slots = slot_idx, a.status = status, a.total_rows = B;
    const int cols = conv_columns(desc);
    a.run = 4;  // in flight together; 250 rows of 12288 channels with 1, 2, 4, 8, 16 rows a warp: 24, 19, 16.6, 19, 18.6 us
    const long long grid = ceil_div(ceil_div(B, a.run), kWarpsPerCta) * cols;
    if (grid > 0x7fffffffll) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
#define CALL(IO, W) conv_step_kernel<IO, W><<<(unsigned)grid, kConvThreads, 0, s>>>(a, cols)
    CONV_DISPATCH(desc, CALL);
#undef CALL
    return finish_launch();
}

int deltalog_conv_prefill(const deltalog_conv_desc *desc, void *window, const deltalog_plan *plan, const void *x, int64_t x_stride, const float *weight,
                          const float *bias, const int32_t *fresh, void *out, int32_t *status, void *stream) {
    if (int rc = validate_conv(desc, x, x_stride, weight, bias)) return rc;
    if (int rc = validate_plan(plan)) return rc;
    if (desc->num_slots <= 0 || !window || !out || !aligned16(window) || !aligned16(out)) return DELTALOG_ERR_INVALID_ARG;
    if (conv_overlaps(desc, x, x_stride, out, plan->max_tokens)) return DELTALOG_ERR_INVALID_ARG;
    if (plan->n == 0) return DELTALOG_OK;
    ConvArgs a = conv_args(desc, x, x_stride, weight, bias);
    conv_plan(a, plan);
    a.init = window, a.final = window, a.slots = plan->scan_slots, a.fresh = fresh, a.out = out, a.status = status;
    a.clear = (desc->hints & DELTALOG_HINT_ZERO_UNWRITTEN) != 0;
    return conv_packed(desc, a, static_cast<cudaStream_t>(stream));
}

int deltalog_conv_forward(const deltalog_conv_desc *desc, const deltalog_plan *plan, const void *init, const void *x, int64_t x_stride,
                          const float *weight, const float *bias, void *out, void *final, void *stream) {
    if (int rc = validate_conv(desc, x, x_stride, weight, bias)) return rc;
    if (int rc = validate_plan(plan)) return rc;
    if (!out || !aligned16(out) || !aligned16(init) || !aligned16(final)) return DELTALOG_ERR_INVALID_ARG;
    if (conv_overlaps(desc, x, x_stride, out, plan->max_tokens)) return DELTALOG_ERR_INVALID_ARG;
    if (plan->n == 0) return DELTALOG_OK;
    ConvArgs a = conv_args(desc, x, x_stride, weight, bias);
    conv_plan(a, plan);
    a.init = init, a.final = final, a.out = out;
    a.clear = (desc->hints & DELTALOG_HINT_ZERO_UNWRITTEN) != 0;
    return conv_packed(desc, a, static_cast<cudaStream_t>(stream));
}

size_t deltalog_conv_workspace_bytes(const deltalog_conv_desc *desc, int32_t rows) {
    if (!desc || desc->channels <= 0 || desc->channels % 8 || desc->width < 2 || desc->width > 4 || rows < 0) return 0;
    // (room for the most blocks that this many rows or fewer make)
    const long long most = ceil_div(148 * 16, conv_columns(desc)), blocks = ceil_div(rows, 16 * kWarpsPerCta);
    const size_t groups = (size_t)(blocks < 1 ? 1 : blocks < most ? blocks : most);
    return groups * (desc->width + 1) * desc->channels * sizeof(float);
}

int deltalog_conv_backward(const deltalog_conv_desc *desc, const deltalog_plan *plan, const void *init, const void *x, int64_t x_stride,
                           const float *weight, const float *bias, const void *dout, const void *dfinal, const deltalog_conv_grads *grads,
                           int32_t rows, void *workspace, size_t workspace_bytes, void *stream) {
    if (int rc = validate_conv(desc, x, x_stride, weight, bias)) return rc;
    if (int rc = validate_plan(plan)) return rc;
    if (!dout || !grads || !grads->x || !grads->weight || rows < plan->max_tokens) return DELTALOG_ERR_INVALID_ARG;
    if (rows > 0x7fffffff - 64) return DELTALOG_ERR_UNSUPPORTED_SHAPE;  // a run walks W - 1 tokens beyond its last one, in 32 bits
    if (!aligned16(init) || !aligned16(dout) || !aligned16(dfinal) || !aligned16(grads->x) || !aligned16(grads->init)) return DELTALOG_ERR_INVALID_ARG;
    if (!workspace || !aligned16(workspace) || workspace_bytes < deltalog_conv_workspace_bytes(desc, rows)) return DELTALOG_ERR_INVALID_ARG;
    if (conv_overlaps(desc, x, x_stride, grads->x, rows) || conv_overlaps(desc, dout, desc->channels, grads->x, rows)) return DELTALOG_ERR_INVALID_ARG;
    if (plan->n == 0) return DELTALOG_OK;
    ConvArgs a = conv_args(desc, x, x_stride, weight, bias);
    conv_plan(a, plan);
    const ConvSplit split = conv_split(desc, rows);
    a.init = init, a.dout = dout, a.dfinal = dfinal, a.dx = grads->x, a.dinit = grads->init;
    a.total_rows = rows, a.run = split.run, a.partial = static_cast<float *>(workspace);
    const int cols = conv_columns(desc);
    const long long heads = grads->init ? ceil_div(plan->n, kWarpsPerCta) : 0, grid = (heads + split.groups) * cols;
    if (grid > 0x7fffffffll) return DELTALOG_ERR_UNSUPPORTED_SHAPE;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (grid > 0) {
#define CALL(IO, W) conv_backward_kernel<IO, W><<<(unsigned)grid, kConvThreads, 0, s>>>(a, cols, heads)
        CONV_DISPATCH(desc, CALL);
#undef CALL
        if (int rc = finish_launch()) return rc;
    }
    conv_reduce_kernel<<<((desc->width + 1) * desc->channels + 31) / 32, 256, 0, s>>>(a.partial, split.groups, a.C, desc->width, grads->weight, grads->bias);
    return finish_launch();
}

}  // extern "C"
