// C ABI of the operators around the layer (norms, gated feed-forward network, microscaled values and products, gradient clipping): argument checks.
// Host code only.
#include <math.h>

#include <algorithm>
#include <initializer_list>
#include <memory>
#include <new>

#include "block_norm.h"
#include "clip.h"
#include "gated_ffn.h"
#include "mx.h"
#include "mx_gemm.h"
#include "norm.h"

namespace slicemoe {

static bool misaligned(const void *p, size_t a) { return ((uintptr_t)p % a) != 0; }
static bool storage_ok(int dtype) { return dtype == SLICEMOE_F32 || dtype == SLICEMOE_BF16; }
static slicemoe_status status_of(hipError_t e) { return e == hipSuccess ? SLICEMOE_OK : SLICEMOE_ERR_HIP; }

static slicemoe_status validate(const slicemoe_norm_config *c)
{
    if (!c || c->T < 0 || c->d < 1 || !storage_ok(c->dtype)) return SLICEMOE_ERR_INVALID_ARG;
    if (!(c->eps >= 0.f) || isinf(c->eps)) return SLICEMOE_ERR_INVALID_ARG;
    return c->d > kNormMaxWidth ? SLICEMOE_ERR_UNSUPPORTED : SLICEMOE_OK;
}

static slicemoe_status validate(const slicemoe_gated_config *c)
{
    if (!c || c->T < 0 || c->d < 1 || c->H < 1 || !storage_ok(c->dtype)) return SLICEMOE_ERR_INVALID_ARG;
    // row offsets inside a tile are 32 bits, the contraction over T counts its bytes and the step beyond them in 31, tiles are counted in 31
    if (c->T > 1 << 29 || c->d > 1 << 20 || c->H > 1 << 20) return SLICEMOE_ERR_UNSUPPORTED;
    return (long long)c->T * std::max(c->d, c->H) > 1ll << 40 ? SLICEMOE_ERR_UNSUPPORTED : SLICEMOE_OK;
}
static slicemoe_status validate_quantized(const slicemoe_gated_config *c)
{
    const slicemoe_status st = validate(c);
    if (st != SLICEMOE_OK) return st;
    return c->dtype != SLICEMOE_BF16 || c->d % 16 != 0 ? SLICEMOE_ERR_UNSUPPORTED : SLICEMOE_OK;
}

static slicemoe_status validate(const slicemoe_block_norm_config *c)
{
    if (!c || c->T < 0 || c->d < 1 || !storage_ok(c->dtype)) return SLICEMOE_ERR_INVALID_ARG;
    if (!(c->eps >= 0.f) || isinf(c->eps) || !(fabsf(c->residual_scale) < INFINITY)) return SLICEMOE_ERR_INVALID_ARG;
    if (c->gate != SLICEMOE_GATE_NONE && c->gate != SLICEMOE_GATE_CHANNEL && c->gate != SLICEMOE_GATE_TOKEN) return SLICEMOE_ERR_INVALID_ARG;
    return c->d > kNormMaxWidth ? SLICEMOE_ERR_UNSUPPORTED : SLICEMOE_OK;
}

static bool bits_ok(int bits) { return bits == 4 || bits == 8; }
static slicemoe_status validate(const slicemoe_mx_config *c)
{
    if (!c || c->rows < 0 || c->cols < 1 || !bits_ok(c->bits) || !storage_ok(c->dtype)) return SLICEMOE_ERR_INVALID_ARG;
    if (c->transposed != 0 && c->transposed != 1) return SLICEMOE_ERR_INVALID_ARG;
    return c->cols > 1 << 20 || c->rows > 1 << 30 || (long long)c->rows * c->cols > 1ll << 40 ? SLICEMOE_ERR_UNSUPPORTED : SLICEMOE_OK;
}
constexpr long long kMxMost = 1ll << 36;   // (a launch ends below 2^32 threads: 2^24 blocks of 128 x 64 results)
static slicemoe_status validate(const slicemoe_mx_product_config *c)
{
    if (!c || c->T < 0 || c->K < 1 || c->N < 1 || !bits_ok(c->bits) || !storage_ok(c->dtype)) return SLICEMOE_ERR_INVALID_ARG;
    if (c->T > 1 << 24 || c->K > 1 << 20 || c->N > 1 << 20) return SLICEMOE_ERR_UNSUPPORTED;
    return (long long)c->T * std::max(c->K, c->N) > kMxMost ? SLICEMOE_ERR_UNSUPPORTED : SLICEMOE_OK;
}
static slicemoe_status validate_mx(const slicemoe_gated_config *c, int bits)
{
    const slicemoe_status st = validate(c);
    if (st != SLICEMOE_OK) return st;
    if (!bits_ok(bits)) return SLICEMOE_ERR_INVALID_ARG;
    return c->dtype != SLICEMOE_BF16 || c->T > 1 << 24 || (long long)c->T * std::max(c->d, c->H) > kMxMost ? SLICEMOE_ERR_UNSUPPORTED : SLICEMOE_OK;
}
// Whether p (may be null) is none of the others.
static bool apart(const void *p, std::initializer_list<const void *> others)
{
    return !p || std::find(others.begin(), others.end(), p) == others.end();
}
// A workspace of at least `need` bytes on the alignment every workspace has.
static slicemoe_status check_workspace(const void *ws, size_t bytes, size_t need)
{
    if (!ws || bytes < need) return SLICEMOE_ERR_WORKSPACE;
    return misaligned(ws, 256) ? SLICEMOE_ERR_INVALID_ARG : SLICEMOE_OK;
}

static slicemoe_status validate(const slicemoe_grad *g, int32_t count)
{
    if (count < 0 || (count > 0 && !g)) return SLICEMOE_ERR_INVALID_ARG;
    double total = 0;
    for (int32_t i = 0; i < count; ++i) {
        if (!storage_ok(g[i].dtype) || g[i].n < 0) return SLICEMOE_ERR_INVALID_ARG;
        const size_t el = g[i].dtype == SLICEMOE_BF16 ? 2 : 4;
        if (g[i].n > 0 && (!g[i].grad || misaligned(g[i].grad, el) || misaligned(g[i].out, el))) return SLICEMOE_ERR_INVALID_ARG;
        total += (double)g[i].n;
    }
    return total > 1e12 || count > 1 << 20 ? SLICEMOE_ERR_UNSUPPORTED : SLICEMOE_OK;
}

struct Range {
    uintptr_t begin, end;
    bool written;
};
constexpr int kOnStack = 512;   // tensors whose ranges (two each) are sorted on the stack, 24 KB; longer lists take host memory

// Whether an array that is written overlaps any other array of the call but the very one it replaces.  r: room for 2 count ranges.
static bool writes_overlap(const slicemoe_grad *g, int32_t count, Range *r)
{
    Range *last = r;
    for (int32_t i = 0; i < count; ++i) {
        if (g[i].n == 0) continue;
        const uintptr_t bytes = (uintptr_t)g[i].n * (g[i].dtype == SLICEMOE_BF16 ? 2 : 4);
        const uintptr_t a = (uintptr_t)g[i].grad, o = (uintptr_t)g[i].out;
        *last++ = {a, a + bytes, o == a};
        if (o && o != a) *last++ = {o, o + bytes, true};
    }
    std::sort(r, last, [](const Range &x, const Range &y) { return x.begin < y.begin; });
    uintptr_t read_end = 0, write_end = 0;   // of the ranges so far
    for (const Range *x = r; x < last; ++x) {
        if (x->begin < write_end || (x->written && x->begin < read_end)) return true;
        (x->written ? write_end : read_end) = std::max(x->written ? write_end : read_end, x->end);
    }
    return false;
}
static slicemoe_status check_overlaps(const slicemoe_grad *g, int32_t count)
{
    if (count <= kOnStack) {
        Range r[2 * kOnStack];
        return writes_overlap(g, count, r) ? SLICEMOE_ERR_INVALID_ARG : SLICEMOE_OK;
    }
    const std::unique_ptr<Range[]> r(new (std::nothrow) Range[2 * (size_t)count]);
    if (!r) return SLICEMOE_ERR_HIP;
    return writes_overlap(g, count, r.get()) ? SLICEMOE_ERR_INVALID_ARG : SLICEMOE_OK;
}

}  // namespace slicemoe

using namespace slicemoe;

extern "C" {

slicemoe_status slicemoe_add_rmsnorm(const slicemoe_norm_config *cfg, const void *x, const void *residual, const void *weight, void *sum,
                                     void *y, void *y_quantized, float *y_scale, slicemoe_stream_t stream)
{
    const slicemoe_status st = validate(cfg);
    if (st != SLICEMOE_OK) return st;
    if (!weight || (cfg->T > 0 && (!x || (!y && !y_quantized) || (y_quantized && !y_scale)))) return SLICEMOE_ERR_INVALID_ARG;
    for (const void *p : {x, residual, weight, (const void *)sum, (const void *)y, (const void *)y_quantized})
        if (misaligned(p, 16)) return SLICEMOE_ERR_INVALID_ARG;
    if (misaligned(y_scale, 4) || (y && y == sum)) return SLICEMOE_ERR_INVALID_ARG;
    return status_of(launch_add_rmsnorm(*cfg, x, residual, weight, sum, y, (uint8_t *)y_quantized, y_scale, (hipStream_t)stream));
}

size_t slicemoe_add_rmsnorm_backward_workspace_bytes(const slicemoe_norm_config *cfg)
{
    if (validate(cfg) != SLICEMOE_OK) return 0;
    return align_up((size_t)norm_backward_blocks(*cfg) * cfg->d * 4, 256);
}

slicemoe_status slicemoe_add_rmsnorm_backward(const slicemoe_norm_config *cfg, const void *sum, const void *weight, const void *d_y,
                                              const void *d_sum, void *d_x, float *d_weight, void *workspace, size_t workspace_bytes,
                                              slicemoe_stream_t stream)
{
    slicemoe_status st = validate(cfg);
    if (st != SLICEMOE_OK) return st;
    if (!weight || !d_weight || (cfg->T > 0 && (!sum || !d_y || !d_x))) return SLICEMOE_ERR_INVALID_ARG;
    for (const void *p : {sum, weight, d_y, d_sum, (const void *)d_x})
        if (misaligned(p, 16)) return SLICEMOE_ERR_INVALID_ARG;
    if (misaligned(d_weight, 4) || (d_x && d_x == sum)) return SLICEMOE_ERR_INVALID_ARG;
    st = check_workspace(workspace, workspace_bytes, slicemoe_add_rmsnorm_backward_workspace_bytes(cfg));
    if (st != SLICEMOE_OK) return st;
    return status_of(launch_add_rmsnorm_backward(*cfg, sum, weight, d_y, d_sum, d_x, d_weight, (float *)workspace, (hipStream_t)stream));
}

size_t slicemoe_gated_ffn_workspace_bytes(const slicemoe_gated_config *cfg)
{
    return validate(cfg) == SLICEMOE_OK ? gated_plan(*cfg, false, false).total : 0;
}
size_t slicemoe_gated_ffn_backward_workspace_bytes(const slicemoe_gated_config *cfg)
{
    return validate(cfg) == SLICEMOE_OK ? gated_plan(*cfg, true, false).total : 0;
}
size_t slicemoe_gated_ffn_quantized_workspace_bytes(const slicemoe_gated_config *cfg)
{
    return validate_quantized(cfg) == SLICEMOE_OK ? gated_plan(*cfg, false, true).total : 0;
}

slicemoe_status slicemoe_gated_ffn(const slicemoe_gated_config *cfg, const void *x, const slicemoe_gated_weights *w, const void *addend,
                                   void *y, void *workspace, size_t workspace_bytes, slicemoe_stream_t stream)
{
    slicemoe_status st = validate(cfg);
    if (st != SLICEMOE_OK) return st;
    if (!w || !w->Wg || !w->Wu || !w->Wd || (cfg->T > 0 && (!x || !y))) return SLICEMOE_ERR_INVALID_ARG;
    for (const void *p : {x, addend, (const void *)y, w->Wg, w->Wu, w->Wd})
        if (misaligned(p, 16)) return SLICEMOE_ERR_INVALID_ARG;
    const GatedPlan plan = gated_plan(*cfg, false, false);
    st = check_workspace(workspace, workspace_bytes, plan.total);
    if (st != SLICEMOE_OK) return st;
    return status_of(launch_gated_ffn(*cfg, plan, x, *w, addend, y, (char *)workspace, (hipStream_t)stream));
}

slicemoe_status slicemoe_gated_ffn_backward(const slicemoe_gated_config *cfg, const void *x, const slicemoe_gated_weights *w, const void *d_y,
                                            const void *addend, void *d_x, const slicemoe_gated_weight_grads *grads, void *workspace,
                                            size_t workspace_bytes, slicemoe_stream_t stream)
{
    slicemoe_status st = validate(cfg);
    if (st != SLICEMOE_OK) return st;
    if (!w || !w->Wg || !w->Wu || !w->Wd || !grads || !grads->Wg || !grads->Wu || !grads->Wd) return SLICEMOE_ERR_INVALID_ARG;
    if (cfg->T > 0 && (!x || !d_y || !d_x)) return SLICEMOE_ERR_INVALID_ARG;
    for (const void *p : {x, d_y, addend, (const void *)d_x, w->Wg, w->Wu, w->Wd, (const void *)grads->Wg, (const void *)grads->Wu,
                          (const void *)grads->Wd})
        if (misaligned(p, 16)) return SLICEMOE_ERR_INVALID_ARG;
    const GatedPlan plan = gated_plan(*cfg, true, false);
    st = check_workspace(workspace, workspace_bytes, plan.total);
    if (st != SLICEMOE_OK) return st;
    return status_of(launch_gated_ffn_backward(*cfg, plan, x, *w, d_y, addend, d_x, *grads, (char *)workspace, (hipStream_t)stream));
}

slicemoe_status slicemoe_gated_ffn_quantized(const slicemoe_gated_config *cfg, const void *x_quantized, const float *x_scale,
                                             const slicemoe_gated_weights_quantized *w, const void *addend, void *y, void *workspace,
                                             size_t workspace_bytes, slicemoe_stream_t stream)
{
    slicemoe_status st = validate_quantized(cfg);
    if (st != SLICEMOE_OK) return st;
    if (!w || !w->Wg || !w->Wu || !w->Wd || !w->Wg_scale || !w->Wu_scale) return SLICEMOE_ERR_INVALID_ARG;
    if (cfg->T > 0 && (!x_quantized || !x_scale || !y)) return SLICEMOE_ERR_INVALID_ARG;
    for (const void *p : {x_quantized, addend, (const void *)y, w->Wg, w->Wu, w->Wd})
        if (misaligned(p, 16)) return SLICEMOE_ERR_INVALID_ARG;
    if (misaligned(x_scale, 4) || misaligned(w->Wg_scale, 4) || misaligned(w->Wu_scale, 4)) return SLICEMOE_ERR_INVALID_ARG;
    const GatedPlan plan = gated_plan(*cfg, false, true);
    st = check_workspace(workspace, workspace_bytes, plan.total);
    if (st != SLICEMOE_OK) return st;
    return status_of(launch_gated_ffn_quantized(*cfg, plan, (const uint8_t *)x_quantized, x_scale, *w, addend, y, (char *)workspace,
                                                (hipStream_t)stream));
}

slicemoe_status slicemoe_gated_ffn_quantize_weights(const slicemoe_gated_config *cfg, const slicemoe_gated_weights *w, void *Wg,
                                                    float *Wg_scale, void *Wu, float *Wu_scale, slicemoe_stream_t stream)
{
    const slicemoe_status st = validate_quantized(cfg);
    if (st != SLICEMOE_OK) return st;
    if (!w || !w->Wg || !w->Wu || !Wg || !Wu || !Wg_scale || !Wu_scale) return SLICEMOE_ERR_INVALID_ARG;
    for (const void *p : {w->Wg, w->Wu, (const void *)Wg, (const void *)Wu})
        if (misaligned(p, 16)) return SLICEMOE_ERR_INVALID_ARG;
    if (misaligned(Wg_scale, 4) || misaligned(Wu_scale, 4)) return SLICEMOE_ERR_INVALID_ARG;
    return status_of(launch_gated_quantize_weights(*cfg, *w, (uint8_t *)Wg, Wg_scale, (uint8_t *)Wu, Wu_scale, (hipStream_t)stream));
}

size_t slicemoe_clip_grads_workspace_bytes(const slicemoe_grad *grads, int32_t count)
{
    if (validate(grads, count) != SLICEMOE_OK) return 0;
    return align_up((size_t)clip_plan(grads, count).chunks * 8 + 1, 256);
}

slicemoe_status slicemoe_clip_grads(const slicemoe_grad *grads, int32_t count, float max_norm, float *norm, void *workspace,
                                    size_t workspace_bytes, slicemoe_stream_t stream)
{
    slicemoe_status st = validate(grads, count);
    if (st != SLICEMOE_OK) return st;
    if (!(max_norm >= 0.f) || !norm || misaligned(norm, 4)) return SLICEMOE_ERR_INVALID_ARG;
    const ClipPlan plan = clip_plan(grads, count);
    st = check_workspace(workspace, workspace_bytes, align_up((size_t)plan.chunks * 8 + 1, 256));
    if (st != SLICEMOE_OK) return st;
    st = check_overlaps(grads, count);
    if (st != SLICEMOE_OK) return st;
    return status_of(launch_clip_grads(grads, count, plan, max_norm, norm, (double *)workspace, (hipStream_t)stream));
}

slicemoe_status slicemoe_block_norm(const slicemoe_block_norm_config *cfg, const void *x, const void *post_weight, const void *gate,
                                    const void *residual, const void *pre_weight, void *sum, void *y, void *y_mx, int32_t y_bits,
                                    float *stats, slicemoe_stream_t stream)
{
    const slicemoe_status st = validate(cfg);
    if (st != SLICEMOE_OK) return st;
    if ((gate != nullptr) != (cfg->gate != SLICEMOE_GATE_NONE) && cfg->T > 0) return SLICEMOE_ERR_INVALID_ARG;
    if (cfg->T > 0 && (!x || !residual || !sum)) return SLICEMOE_ERR_INVALID_ARG;
    if (pre_weight ? cfg->T > 0 && !y && !y_mx : y || y_mx) return SLICEMOE_ERR_INVALID_ARG;
    if (y_mx && (!bits_ok(y_bits) || misaligned(y_mx, 256))) return SLICEMOE_ERR_INVALID_ARG;
    const slicemoe_mx_config rows = {cfg->T, cfg->d, y_bits, cfg->dtype, 0};
    if (y_mx && validate(&rows) != SLICEMOE_OK) return SLICEMOE_ERR_UNSUPPORTED;
    for (const void *p : {x, post_weight, gate, residual, pre_weight, (const void *)sum, (const void *)y})
        if (misaligned(p, 16)) return SLICEMOE_ERR_INVALID_ARG;
    if (misaligned(stats, 8) || (y && y == sum)) return SLICEMOE_ERR_INVALID_ARG;
    for (const void *p : {post_weight, gate, pre_weight, (const void *)y_mx})   // what every row reads, and a third output
        if (p && (p == sum || p == y)) return SLICEMOE_ERR_INVALID_ARG;
    for (const void *p : {x, post_weight, gate, residual, pre_weight})
        if (y_mx && p == y_mx) return SLICEMOE_ERR_INVALID_ARG;
    if (!apart(stats, {x, post_weight, gate, residual, pre_weight, sum, y, y_mx})) return SLICEMOE_ERR_INVALID_ARG;
    return status_of(launch_block_norm(*cfg, x, post_weight, gate, residual, pre_weight, sum, y, (uint8_t *)y_mx, y_bits, stats, (hipStream_t)stream));
}

size_t slicemoe_block_norm_backward_workspace_bytes(const slicemoe_block_norm_config *cfg)
{
    if (validate(cfg) != SLICEMOE_OK) return 0;
    return align_up((size_t)block_norm_backward_blocks(*cfg) * cfg->d * 8, 256);
}

slicemoe_status slicemoe_block_norm_backward(const slicemoe_block_norm_config *cfg, const void *x, const void *post_weight, const void *gate,
                                             const void *sum, const void *pre_weight, const float *stats, const void *d_y, const void *d_sum,
                                             void *d_x, void *d_residual, float *d_post_weight, void *d_gate, float *d_pre_weight,
                                             void *workspace, size_t workspace_bytes, slicemoe_stream_t stream)
{
    slicemoe_status st = validate(cfg);
    if (st != SLICEMOE_OK) return st;
    const bool token = cfg->gate == SLICEMOE_GATE_TOKEN, some = cfg->T > 0;
    if (!pre_weight || !d_pre_weight || (post_weight && !d_post_weight)) return SLICEMOE_ERR_INVALID_ARG;
    if ((gate != nullptr) != (cfg->gate != SLICEMOE_GATE_NONE) && (some || cfg->gate == SLICEMOE_GATE_CHANNEL)) return SLICEMOE_ERR_INVALID_ARG;
    if (cfg->gate != SLICEMOE_GATE_NONE && !d_gate && (some || !token)) return SLICEMOE_ERR_INVALID_ARG;
    if (some && (!x || !sum || !stats || !d_y || !d_x || !d_residual)) return SLICEMOE_ERR_INVALID_ARG;
    for (const void *p : {x, post_weight, gate, sum, pre_weight, d_y, d_sum, (const void *)d_x, (const void *)d_residual})
        if (misaligned(p, 16)) return SLICEMOE_ERR_INVALID_ARG;
    if (misaligned(stats, 8) || misaligned(d_post_weight, 4) || misaligned(d_pre_weight, 4) || misaligned(d_gate, token ? 16 : 4)) return SLICEMOE_ERR_INVALID_ARG;
    // the outputs of rows are apart from one another and from the inputs that the row's other outputs need
    if (some) {
        const void *in[] = {x, sum};
        for (const void *p : in)
            if (d_x == p || d_residual == p || (token && d_gate == p)) return SLICEMOE_ERR_INVALID_ARG;
        if (d_x == d_residual || (token && (d_gate == d_x || d_gate == d_residual || d_gate == d_y || d_gate == d_sum || d_gate == gate || d_x == gate || d_residual == gate)))
            return SLICEMOE_ERR_INVALID_ARG;
    }
    st = check_workspace(workspace, workspace_bytes, slicemoe_block_norm_backward_workspace_bytes(cfg));
    if (st != SLICEMOE_OK) return st;
    // what every row reads, and the workspace, stay as they are until the end; sums over the rows are apart from everything
    const void *row_gate = token ? d_gate : nullptr, *column_gate = cfg->gate == SLICEMOE_GATE_CHANNEL ? d_gate : nullptr, *column_post = post_weight ? d_post_weight : nullptr;
    for (const void *p : {(const void *)d_x, (const void *)d_residual, row_gate})
        if (some && !apart(p, {post_weight, gate, pre_weight, stats, workspace})) return SLICEMOE_ERR_INVALID_ARG;
    for (const void *p : {column_post, column_gate, (const void *)d_pre_weight})
        if (!apart(p, {post_weight, gate, pre_weight, workspace}) || (some && !apart(p, {x, sum, stats, d_y, d_sum, d_x, d_residual, row_gate}))) return SLICEMOE_ERR_INVALID_ARG;
    if (!apart(column_post, {column_gate, d_pre_weight}) || !apart(column_gate, {d_pre_weight})) return SLICEMOE_ERR_INVALID_ARG;
    if (!apart(workspace, {x, post_weight, gate, sum, pre_weight, stats, d_y, d_sum})) return SLICEMOE_ERR_INVALID_ARG;
    return status_of(launch_block_norm_backward(*cfg, x, post_weight, gate, sum, pre_weight, stats, d_y, d_sum, d_x, d_residual,
                                                post_weight ? d_post_weight : nullptr, d_gate, d_pre_weight, (float *)workspace, (hipStream_t)stream));
}

size_t slicemoe_mx_bytes(const slicemoe_mx_config *cfg)
{
    return validate(cfg) == SLICEMOE_OK ? std::max<size_t>(256, mx_total_bytes(cfg->rows, cfg->cols, cfg->bits)) : 0;
}

slicemoe_status slicemoe_mx_quantize(const slicemoe_mx_config *cfg, const void *x, void *mx, slicemoe_stream_t stream)
{
    const slicemoe_status st = validate(cfg);
    if (st != SLICEMOE_OK) return st;
    if (cfg->rows > 0 && (!x || !mx)) return SLICEMOE_ERR_INVALID_ARG;
    if (misaligned(x, 16) || misaligned(mx, 256)) return SLICEMOE_ERR_INVALID_ARG;
    return status_of(launch_mx_quantize(*cfg, x, (uint8_t *)mx, (hipStream_t)stream));
}

slicemoe_status slicemoe_mx_dequantize(const slicemoe_mx_config *cfg, const void *mx, void *x, slicemoe_stream_t stream)
{
    const slicemoe_status st = validate(cfg);
    if (st != SLICEMOE_OK) return st;
    if (cfg->rows > 0 && (!x || !mx)) return SLICEMOE_ERR_INVALID_ARG;
    if (misaligned(x, 16) || misaligned(mx, 256)) return SLICEMOE_ERR_INVALID_ARG;
    return status_of(launch_mx_dequantize(*cfg, (const uint8_t *)mx, x, (hipStream_t)stream));
}

size_t slicemoe_mx_product_workspace_bytes(const slicemoe_mx_product_config *cfg)
{
    return validate(cfg) == SLICEMOE_OK ? mx_product_workspace(*cfg) : 0;
}

slicemoe_status slicemoe_mx_product(const slicemoe_mx_product_config *cfg, const void *x_mx, const void *w_mx, const void *addend, void *y,
                                    void *workspace, size_t workspace_bytes, slicemoe_stream_t stream)
{
    slicemoe_status st = validate(cfg);
    if (st != SLICEMOE_OK) return st;
    if (!w_mx || (cfg->T > 0 && (!x_mx || !y))) return SLICEMOE_ERR_INVALID_ARG;
    if (misaligned(x_mx, 256) || misaligned(w_mx, 256) || misaligned(addend, 16) || misaligned(y, 16)) return SLICEMOE_ERR_INVALID_ARG;
    const size_t need = mx_product_workspace(*cfg);
    if (need > 0) st = check_workspace(workspace, workspace_bytes, need);
    if (st != SLICEMOE_OK) return st;
    return status_of(launch_mx_product(*cfg, (const uint8_t *)x_mx, (const uint8_t *)w_mx, addend, y, (char *)workspace, (hipStream_t)stream));
}

size_t slicemoe_gated_ffn_mx_workspace_bytes(const slicemoe_gated_config *cfg, int32_t bits)
{
    return validate_mx(cfg, bits) == SLICEMOE_OK ? gated_mx_workspace(*cfg, bits) : 0;
}

slicemoe_status slicemoe_gated_ffn_mx(const slicemoe_gated_config *cfg, int32_t bits, const void *x_mx, const slicemoe_gated_weights_mx *w,
                                      const void *addend, void *y, void *workspace, size_t workspace_bytes, slicemoe_stream_t stream)
{
    slicemoe_status st = validate_mx(cfg, bits);
    if (st != SLICEMOE_OK) return st;
    if (!w || !w->Wg || !w->Wu || !w->Wd || (cfg->T > 0 && (!x_mx || !y))) return SLICEMOE_ERR_INVALID_ARG;
    for (const void *p : {x_mx, w->Wg, w->Wu, w->Wd})
        if (misaligned(p, 256)) return SLICEMOE_ERR_INVALID_ARG;
    if (misaligned(addend, 16) || misaligned(y, 16)) return SLICEMOE_ERR_INVALID_ARG;
    st = check_workspace(workspace, workspace_bytes, gated_mx_workspace(*cfg, bits));
    if (st != SLICEMOE_OK) return st;
    return status_of(launch_gated_mx(*cfg, bits, (const uint8_t *)x_mx, *w, addend, y, (char *)workspace, (hipStream_t)stream));
}

}  // extern "C"
