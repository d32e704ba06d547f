// C ABI of the operators around an output layer: argument checks, plans and launches. See include/lfmmi.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>
#include <vector>

#include "checks.h"
#include "layers.h"
#include "status.h"

using namespace lfmmi;

namespace {

constexpr int32_t kMostWidth = 1 << 24;  // of a row; eight values make a chunk, whose number times eight has 32 bits

// Whether an array of so many bytes is written past the caches: it would drive out what is read, and be gone before it is
// read itself. (Past them and otherwise, replayed: dropout of 268 MB of bf16 80 and 101 us; rows of a table of 134 MB 28 and 31; the
// gradient of a table of 268 MB with its sorting 108 and 124; dropout of 82 MB, which the caches hold, 31.9 and 29.2 called in turn.)
bool past_caches(int64_t bytes) { return bytes > kCacheBytes / 2; }

lfmmi_status fail_aligned() { return fail(LFMMI_ERR_INVALID_ARG, "an array is not aligned to its elements"); }
lfmmi_status fail_overlap() { return fail(LFMMI_ERR_INVALID_ARG, "an array that is written overlaps another one"); }
lfmmi_status fail_workspace()
{
    return fail(LFMMI_ERR_INVALID_ARG, "workspace is null, too small or not aligned to 16 bytes");
}

lfmmi_status check_width(int32_t D)
{
    if (D < 1) return fail(LFMMI_ERR_INVALID_ARG, "D must be >= 1");
    if (D > kMostWidth) return fail(LFMMI_ERR_UNSUPPORTED, "D exceeds 2^24");
    return LFMMI_OK;
}

lfmmi_status check_batch(int32_t B, int32_t T, const int32_t* lengths)
{
    if (B < 0 || T < 0) return fail(LFMMI_ERR_INVALID_ARG, "B and T must be >= 0");
    if ((int64_t)B * T > INT32_MAX) return fail(LFMMI_ERR_UNSUPPORTED, "B * T exceeds 2^31 - 1");
    return check_lengths(lengths, B, T);
}

lfmmi_status check_scale(float scale)
{
    if (!(scale >= 1e-6f && scale <= 1e6f)) return fail(LFMMI_ERR_INVALID_ARG, "scale outside [1e-6, 1e6]");
    return LFMMI_OK;
}

lfmmi_status make_draw(float p, uint64_t seed, uint64_t offset, const int64_t* step, Draw* d)
{
    if (!(p >= 0.f && p <= 1.f)) return fail(LFMMI_ERR_INVALID_ARG, "p outside [0, 1]");
    if (step && !aligned(step, 8)) return fail_aligned();
    const int threshold = (int)std::nearbyint((double)p * 65536.0);
    *d = {seed, offset, step, threshold, threshold < 65536 ? (float)(65536.0 / (65536 - threshold)) : 0.f};
    return LFMMI_OK;
}

// Arrays of a call, and whether one that is written overlaps another.
struct Spans {
    std::vector<Span> all;
    void add(const void* p, int64_t bytes, bool written)
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(p);
        if (p && bytes > 0) all.push_back({a, a + (uintptr_t)bytes, written});
    }
    void rows(const void* p, int64_t stride_b, int64_t stride_t, int64_t B, int64_t T, int64_t D, int64_t size)
    {
        add(p, ((B - 1) * stride_b + (T - 1) * stride_t + D) * size, false);
    }
    bool meet() { return overlap(all); }
};

// Whether rows (b, t) follow each other without gaps.
bool in_order(int64_t stride_b, int64_t stride_t, int32_t B, int32_t T, int32_t D)
{
    return (T == 1 || stride_t == D) && (B == 1 || stride_b == (int64_t)T * D);
}

}  // namespace

extern "C" {

lfmmi_status lfmmi_embed_tokens(const void* table, int32_t dtype, int32_t V, int32_t D, int64_t stride,
                                const void* tokens, int32_t token_bytes, int32_t B, int32_t T,
                                const int32_t* lengths, float scale, void* out, int32_t* status,
                                void* hip_stream)
try {
    if (!known(dtype)) return fail(LFMMI_ERR_INVALID_ARG, "unknown dtype");
    if (V < 1) return fail(LFMMI_ERR_INVALID_ARG, "V must be >= 1");
    lfmmi_status st = check_width(D);
    if (st == LFMMI_OK) st = check_batch(B, T, lengths);
    if (st == LFMMI_OK) st = check_strides(stride, 0, V, 1);
    if (st == LFMMI_OK) st = check_scale(scale);
    if (st != LFMMI_OK) return st;
    if (token_bytes != 4 && token_bytes != 8) return fail(LFMMI_ERR_INVALID_ARG, "token_bytes must be 4 or 8");
    if (B == 0 || T == 0) return LFMMI_OK;
    if (!table || !tokens || !out) return fail(LFMMI_ERR_INVALID_ARG, "table / tokens / out is null");
    const int64_t size = (int64_t)dtype_size(dtype), N = (int64_t)B * T;
    if (!aligned(table, size) || !aligned(out, size) || !aligned(tokens, token_bytes) || !aligned(status, 4))
        return fail_aligned();
    Spans spans;
    spans.rows(table, stride, 0, V, 1, D, size);
    spans.add(tokens, N * token_bytes, false);
    spans.add(out, N * D * size, true);
    spans.add(status, N * 4, true);
    if (spans.meet()) return fail_overlap();
    for (int32_t b = 0; b < B;) {
        SeqLengths lens;
        const int32_t n = fill_lengths(lengths, b, B, &lens);
        const int64_t row = (int64_t)b * T;
        const EmbedParams p{table, stride, at_bytes(tokens, row * token_bytes), token_bytes, n, T, V, D, scale,
                            at_bytes(out, row * D * size), at(status, row), past_caches(N * D * size)};
        const hipError_t e = launch_embed(p, lens, dtype, static_cast<hipStream_t>(hip_stream));
        if (e != hipSuccess) return fail_hip(e, "kernel launch");
        b += n;
    }
    return LFMMI_OK;
} catch (...) {
    return fail_memory();
}

lfmmi_status lfmmi_embed_tokens_workspace(int32_t V, int32_t D, int32_t B, int32_t T, int64_t* bytes)
{
    if (!bytes) return fail(LFMMI_ERR_INVALID_ARG, "bytes is null");
    if (V < 1) return fail(LFMMI_ERR_INVALID_ARG, "V must be >= 1");
    lfmmi_status st = check_width(D);
    if (st == LFMMI_OK) st = check_batch(B, T, nullptr);
    if (st != LFMMI_OK) return st;
    *bytes = (int64_t)plan_embed((int64_t)B * T, V, D).bytes;
    return LFMMI_OK;
}

lfmmi_status lfmmi_embed_tokens_backward(const void* grad_out, int32_t dtype, int32_t V, int32_t D,
                                         int64_t stride_b, int64_t stride_t, const void* tokens,
                                         int32_t token_bytes, int32_t B, int32_t T, const int32_t* lengths,
                                         float scale, int accumulate, void* grad, void* workspace,
                                         int64_t workspace_bytes, void* hip_stream)
try {
    if (!known(dtype)) return fail(LFMMI_ERR_INVALID_ARG, "unknown dtype");
    if (V < 1) return fail(LFMMI_ERR_INVALID_ARG, "V must be >= 1");
    lfmmi_status st = check_width(D);
    if (st == LFMMI_OK) st = check_batch(B, T, lengths);
    if (st == LFMMI_OK) st = check_strides(stride_b, stride_t, B, T);
    if (st == LFMMI_OK) st = check_scale(scale);
    if (st != LFMMI_OK) return st;
    if (token_bytes != 4 && token_bytes != 8) return fail(LFMMI_ERR_INVALID_ARG, "token_bytes must be 4 or 8");
    const int64_t size = (int64_t)dtype_size(dtype), N = (int64_t)B * T;
    if (!grad || (N > 0 && (!grad_out || !tokens)))
        return fail(LFMMI_ERR_INVALID_ARG, "grad_out / tokens / grad is null");
    if (!aligned(grad_out, size) || !aligned(grad, size) || !aligned(tokens, token_bytes)) return fail_aligned();
    EmbedGradParams p{grad_out, stride_b, stride_t, tokens, token_bytes, B, T, V, D, scale, accumulate != 0, grad,
                      workspace, plan_embed(N, V, D), past_caches((int64_t)V * D * size)};
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < (int64_t)p.plan.bytes) return fail_workspace();
    Spans spans;
    if (N > 0) spans.rows(grad_out, stride_b, stride_t, B, T, D, size);
    spans.add(tokens, N * token_bytes, false);
    spans.add(grad, (int64_t)V * D * size, true);
    spans.add(workspace, (int64_t)p.plan.bytes, true);
    if (spans.meet()) return fail_overlap();
    if (N == 0 && accumulate) return LFMMI_OK;
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    SeqLengths lens;
    lens.n = 0;
    const bool at_once = !lengths || B <= kLengthsPerLaunch;
    if (at_once) fill_lengths(lengths, 0, B, &lens);
    for (int32_t b = 0; !at_once && b < B && T > 0;) {
        const int32_t n = fill_lengths(lengths, b, B, &lens);
        const hipError_t e = launch_embed_keys(p, lens, b, n, stream);
        if (e != hipSuccess) return fail_hip(e, "kernel launch");
        b += n;
    }
    const hipError_t e = launch_embed_grad(p, at_once ? &lens : nullptr, dtype, stream);
    return e == hipSuccess ? LFMMI_OK : fail_hip(e, "kernel launch");
} catch (...) {
    return fail_memory();
}

lfmmi_status lfmmi_dropout(const void* x, int32_t dtype, int32_t R, int32_t D, int64_t stride, float p,
                           uint64_t seed, uint64_t offset, const int64_t* step, void* y, void* hip_stream)
try {
    if (!known(dtype)) return fail(LFMMI_ERR_INVALID_ARG, "unknown dtype");
    if (R < 0 || D < 0) return fail(LFMMI_ERR_INVALID_ARG, "R and D must be >= 0");
    if (D > (1 << 30)) return fail(LFMMI_ERR_UNSUPPORTED, "D exceeds 2^30");
    lfmmi_status st = check_strides(stride, 0, R, 1);
    DropoutParams q{x, y, stride, y == x ? stride : (int64_t)D, R, D, {}, false};
    if (st == LFMMI_OK) st = make_draw(p, seed, offset, step, &q.draw);
    if (st != LFMMI_OK) return st;
    if (R == 0 || D == 0) return LFMMI_OK;
    if (!x || !y) return fail(LFMMI_ERR_INVALID_ARG, "x / y is null");
    const int64_t size = (int64_t)dtype_size(dtype);
    if (!aligned(x, size) || !aligned(y, size)) return fail_aligned();
    if (y == x && R > 1 && stride < D) return fail(LFMMI_ERR_INVALID_ARG, "rows that overlap cannot be written");
    Spans spans;
    if (y != x) spans.rows(x, stride, 0, R, 1, D, size);
    spans.add(y, ((int64_t)(R - 1) * q.stride_y + D) * size, true);
    spans.add(step, 8, false);
    if (spans.meet()) return fail_overlap();
    q.once = past_caches((int64_t)R * D * size);
    const hipError_t e = launch_dropout(q, dtype, static_cast<hipStream_t>(hip_stream));
    return e == hipSuccess ? LFMMI_OK : fail_hip(e, "kernel launch");
} catch (...) {
    return fail_memory();
}

lfmmi_status lfmmi_add_rms_norm(const void* x, int64_t stride_b, int64_t stride_t, const void* residual,
                                int64_t residual_stride_b, int64_t residual_stride_t, int32_t dtype, int32_t B,
                                int32_t T, int32_t D, const int32_t* lengths, const void* weight,
                                int32_t weight_dtype, float eps, float p, uint64_t seed, uint64_t offset,
                                const int64_t* step, void* sum, void* y, float* rstd, void* q, float* q_scale,
                                void* hip_stream)
try {
    if (!known(dtype)) return fail(LFMMI_ERR_INVALID_ARG, "unknown dtype");
    if (weight && weight_dtype != dtype && weight_dtype != LFMMI_F32)
        return fail(LFMMI_ERR_INVALID_ARG, "weight_dtype must be dtype or LFMMI_F32");
    lfmmi_status st = check_width(D);
    if (st == LFMMI_OK) st = check_batch(B, T, lengths);
    if (st == LFMMI_OK) st = check_strides(stride_b, stride_t, B, T);
    if (st == LFMMI_OK && residual) st = check_strides(residual_stride_b, residual_stride_t, B, T);
    NormParams a{};
    if (st == LFMMI_OK) st = make_draw(p, seed, offset, step, &a.draw);
    if (st != LFMMI_OK) return st;
    if (!(eps >= 1e-30f && eps <= 1e20f)) return fail(LFMMI_ERR_INVALID_ARG, "eps outside [1e-30, 1e20]");
    if (B == 0 || T == 0) return LFMMI_OK;
    if (!x) return fail(LFMMI_ERR_INVALID_ARG, "x is null");
    if (!sum && (residual || a.draw.threshold > 0))
        return fail(LFMMI_ERR_INVALID_ARG, "sum is null, with a residual or dropout");
    if ((q == nullptr) != (q_scale == nullptr)) return fail(LFMMI_ERR_INVALID_ARG, "q and q_scale go together");
    const int64_t size = (int64_t)dtype_size(dtype), N = (int64_t)B * T, wsize = weight_dtype == LFMMI_F32 ? 4 : size;
    if (!aligned(x, size) || !aligned(residual, size) || !aligned(weight, wsize) || !aligned(sum, size) ||
        !aligned(y, size) || !aligned(rstd, 4) || !aligned(q_scale, 4))
        return fail_aligned();
    // the sum may take the place of an input whose rows follow each other: a lane reads what it writes first
    const bool over_x = sum == x && in_order(stride_b, stride_t, B, T, D);
    const bool over_r = residual && sum == residual && in_order(residual_stride_b, residual_stride_t, B, T, D);
    Spans spans;
    if (!over_x && !(over_r && x == residual && in_order(stride_b, stride_t, B, T, D)))
        spans.rows(x, stride_b, stride_t, B, T, D, size);
    if (residual && !over_r && !(over_x && x == residual && in_order(residual_stride_b, residual_stride_t, B, T, D)))
        spans.rows(residual, residual_stride_b, residual_stride_t, B, T, D, size);
    spans.add(weight, (int64_t)D * wsize, false);
    spans.add(step, 8, false);
    spans.add(sum, N * D * size, true);
    spans.add(y, N * D * size, true);
    spans.add(rstd, N * 4, true);
    spans.add(q, N * D, true);
    spans.add(q_scale, N * 4, true);
    if (spans.meet()) return fail_overlap();
    for (int32_t b = 0; b < B;) {
        SeqLengths lens;
        const int32_t n = fill_lengths(lengths, b, B, &lens);
        const int64_t row = (int64_t)b * T;
        a.x = at_bytes(x, b * stride_b * size);
        a.residual = at_bytes(residual, b * residual_stride_b * size);
        a.x_stride_b = stride_b;
        a.x_stride_t = stride_t;
        a.r_stride_b = residual_stride_b;
        a.r_stride_t = residual_stride_t;
        a.B = n;
        a.T = T;
        a.D = D;
        a.row = row;
        a.weight = weight;
        a.weight_f32 = weight_dtype == LFMMI_F32;
        a.eps = eps;
        a.sum = at_bytes(sum, row * D * size);
        a.y = at_bytes(y, row * D * size);
        a.rstd = at(rstd, row);
        a.q = at(static_cast<uint8_t*>(q), row * D);
        a.q_scale = at(q_scale, row);
        a.once = past_caches(N * D * size);
        const hipError_t e = launch_norm(a, lens, dtype, static_cast<hipStream_t>(hip_stream));
        if (e != hipSuccess) return fail_hip(e, "kernel launch");
        b += n;
    }
    return LFMMI_OK;
} catch (...) {
    return fail_memory();
}

lfmmi_status lfmmi_add_rms_norm_workspace(int32_t B, int32_t T, int32_t D, int64_t* bytes)
{
    if (!bytes) return fail(LFMMI_ERR_INVALID_ARG, "bytes is null");
    lfmmi_status st = check_width(D);
    if (st == LFMMI_OK) st = check_batch(B, T, nullptr);
    if (st != LFMMI_OK) return st;
    const int64_t N = (int64_t)B * T;
    *bytes = (int64_t)std::max(norm_blocks(N, D, LFMMI_F32), norm_blocks(N, D, LFMMI_BF16)) * D * 4;
    return LFMMI_OK;
}

lfmmi_status lfmmi_add_rms_norm_backward(const void* sum, int64_t stride_b, int64_t stride_t, int32_t dtype,
                                         int32_t B, int32_t T, int32_t D, const int32_t* lengths,
                                         const void* weight, int32_t weight_dtype, const float* rstd,
                                         const void* grad_y, const void* grad_sum, float p, uint64_t seed,
                                         uint64_t offset, const int64_t* step, void* grad_x, void* grad_residual,
                                         void* grad_weight, void* workspace, int64_t workspace_bytes,
                                         void* hip_stream)
try {
    if (!known(dtype)) return fail(LFMMI_ERR_INVALID_ARG, "unknown dtype");
    if ((weight || grad_weight) && weight_dtype != dtype && weight_dtype != LFMMI_F32)
        return fail(LFMMI_ERR_INVALID_ARG, "weight_dtype must be dtype or LFMMI_F32");
    lfmmi_status st = check_width(D);
    if (st == LFMMI_OK) st = check_batch(B, T, lengths);
    if (st == LFMMI_OK) st = check_strides(stride_b, stride_t, B, T);
    NormGradParams a{};
    if (st == LFMMI_OK) st = make_draw(p, seed, offset, step, &a.draw);
    if (st != LFMMI_OK) return st;
    const int64_t size = (int64_t)dtype_size(dtype), N = (int64_t)B * T, wsize = weight_dtype == LFMMI_F32 ? 4 : size;
    if (N > 0 && (!sum || !rstd)) return fail(LFMMI_ERR_INVALID_ARG, "sum / rstd is null");
    if (N > 0 && !grad_y && !grad_sum) return fail(LFMMI_ERR_INVALID_ARG, "grad_y and grad_sum are null");
    if (!aligned(sum, size) || !aligned(weight, wsize) || !aligned(rstd, 4) || !aligned(grad_y, size) ||
        !aligned(grad_sum, size) || !aligned(grad_x, size) || !aligned(grad_residual, size) ||
        !aligned(grad_weight, wsize))
        return fail_aligned();
    a.blocks = norm_blocks(N, D, dtype);
    const int64_t need = grad_weight ? (int64_t)a.blocks * D * 4 : 0;
    if (need > 0 && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return fail_workspace();
    const int64_t all = N * D * size;
    // a gradient may take the place of one that comes in: a lane reads what it writes first
    const auto written = [&](const void* g) { return g && (g == grad_x || g == grad_residual); };
    Spans spans;
    if (N > 0) spans.rows(sum, stride_b, stride_t, B, T, D, size);
    spans.add(weight, (int64_t)D * wsize, false);
    spans.add(rstd, N * 4, false);
    spans.add(step, 8, false);
    if (!written(grad_y)) spans.add(grad_y, all, false);
    if (!written(grad_sum) && grad_sum != grad_y) spans.add(grad_sum, all, false);
    spans.add(grad_x, all, true);
    spans.add(grad_residual, all, true);
    spans.add(grad_weight, (int64_t)D * wsize, true);
    spans.add(workspace, need, true);
    if (spans.meet()) return fail_overlap();
    const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    for (int32_t b = 0; b < B && T > 0;) {
        SeqLengths lens;
        const int32_t n = fill_lengths(lengths, b, B, &lens);
        const int64_t row = (int64_t)b * T;
        a.h = at_bytes(sum, b * stride_b * size);
        a.stride_b = stride_b;
        a.stride_t = stride_t;
        a.B = n;
        a.T = T;
        a.D = D;
        a.row = row;
        a.weight = weight;
        a.weight_f32 = weight_dtype == LFMMI_F32;
        a.rstd = rstd + row;
        a.grad_y = at_bytes(grad_y, row * D * size);
        a.grad_sum = at_bytes(grad_sum, row * D * size);
        a.grad_x = at_bytes(grad_x, row * D * size);
        a.grad_residual = at_bytes(grad_residual, row * D * size);
        a.partials = grad_weight ? static_cast<float*>(workspace) : nullptr;
        a.add = b > 0;
        a.once = past_caches(all);
        const hipError_t e = launch_norm_grad(a, lens, dtype, stream);
        if (e != hipSuccess) return fail_hip(e, "kernel launch");
        b += n;
    }
    if (grad_weight) {
        const hipError_t e = launch_norm_weight(static_cast<const float*>(workspace), a.blocks, D, grad_weight,
                                                weight_dtype, stream);
        if (e != hipSuccess) return fail_hip(e, "kernel launch");
    }
    return LFMMI_OK;
} catch (...) {
    return fail_memory();
}

lfmmi_status lfmmi_verify_tokens_workspace(int32_t B, int32_t K, int32_t V, int64_t* bytes)
{
    if (!bytes) return fail(LFMMI_ERR_INVALID_ARG, "bytes is null");
    if (B < 0 || K < 0 || V < 1) return fail(LFMMI_ERR_INVALID_ARG, "B and K must be >= 0, V >= 1");
    if (V > (1 << 30)) return fail(LFMMI_ERR_UNSUPPORTED, "V exceeds 2^30");
    if (K > (1 << 29) || (int64_t)B * (2 * (int64_t)K + 1) > INT32_MAX)
        return fail(LFMMI_ERR_UNSUPPORTED, "B * (2 K + 1) exceeds 2^31 - 1");
    *bytes = B > 0 ? (int64_t)verify_workspace(B, K, V) : 0;
    return LFMMI_OK;
}

lfmmi_status lfmmi_verify_tokens(const void* logits, int32_t dtype, int32_t B, int32_t K, int32_t V,
                                 int64_t stride_b, int64_t stride_t, const void* draft_logits,
                                 int64_t draft_stride_b, int64_t draft_stride_t, const void* drafted,
                                 int32_t token_bytes, const int32_t* lengths, float scale, float draft_scale,
                                 const float* uniforms, int32_t* accepted, int32_t* tokens, int32_t* status,
                                 void* workspace, int64_t workspace_bytes, void* hip_stream)
try {
    if (!known(dtype)) return fail(LFMMI_ERR_INVALID_ARG, "unknown dtype");
    int64_t need = 0;
    lfmmi_status st = lfmmi_verify_tokens_workspace(B, K, V, &need);
    if (st == LFMMI_OK) st = check_strides(stride_b, stride_t, B, K + 1);
    if (st == LFMMI_OK && draft_logits) st = check_strides(draft_stride_b, draft_stride_t, B, K);
    if (st == LFMMI_OK) st = check_scale(scale);
    if (st == LFMMI_OK && draft_logits) st = check_scale(draft_scale);
    if (st == LFMMI_OK) st = check_lengths(lengths, B, K);
    if (st != LFMMI_OK) return st;
    if (K > 0 && token_bytes != 4 && token_bytes != 8) return fail(LFMMI_ERR_INVALID_ARG, "token_bytes must be 4 or 8");
    if (draft_logits && !uniforms) return fail(LFMMI_ERR_INVALID_ARG, "draft_logits without uniforms");
    if (B == 0) return LFMMI_OK;
    if (!logits || !accepted || !tokens || (K > 0 && !drafted))
        return fail(LFMMI_ERR_INVALID_ARG, "logits / drafted / accepted / tokens is null");
    const int64_t size = (int64_t)dtype_size(dtype), N = (int64_t)B * K;
    if (!aligned(logits, size) || !aligned(draft_logits, size) || (K > 0 && !aligned(drafted, token_bytes)) ||
        !aligned(uniforms, 4) || !aligned(accepted, 4) || !aligned(tokens, 4) || !aligned(status, 4))
        return fail_aligned();
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < need) return fail_workspace();
    Spans spans;
    spans.rows(logits, stride_b, stride_t, B, K + 1, V, size);
    if (K > 0) {
        if (draft_logits) spans.rows(draft_logits, draft_stride_b, draft_stride_t, B, K, V, size);
        spans.add(drafted, N * token_bytes, false);
    }
    spans.add(uniforms, (N + B) * 4, false);
    spans.add(accepted, (int64_t)B * 4, true);
    spans.add(tokens, (N + B) * 4, true);
    spans.add(status, (int64_t)B * 4, true);
    spans.add(workspace, need, true);
    if (spans.meet()) return fail_overlap();
    for (int32_t b = 0; b < B;) {
        SeqLengths lens;
        const int32_t n = fill_lengths(lengths, b, B, &lens);
        VerifyParams p{};
        p.x = at_bytes(logits, b * stride_b * size);
        p.stride_b = stride_b;
        p.stride_t = stride_t;
        if (K > 0) {
            p.draft = at_bytes(draft_logits, b * draft_stride_b * size);
            p.drafted = at_bytes(drafted, (int64_t)b * K * token_bytes);
        }
        p.draft_stride_b = draft_stride_b;
        p.draft_stride_t = draft_stride_t;
        p.token_bytes = token_bytes;
        p.B = n;
        p.K = K;
        p.V = V;
        p.scale = scale;
        p.draft_scale = draft_scale;
        p.uniforms = at(uniforms, (int64_t)b * (K + 1));
        p.accepted = accepted + b;
        p.tokens = tokens + (int64_t)b * (K + 1);
        p.status = at(status, b);
        p.parts = (V + kVerifyPart - 1) / kVerifyPart;
        p.workspace = workspace;
        const hipError_t e = launch_verify(p, lens, dtype, static_cast<hipStream_t>(hip_stream));
        if (e != hipSuccess) return fail_hip(e, "kernel launch");
        b += n;
    }
    return LFMMI_OK;
} catch (...) {
    return fail_memory();
}

}  // extern "C"
