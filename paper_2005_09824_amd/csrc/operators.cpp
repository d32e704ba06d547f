// C ABI of the operators on token log probabilities and on gradients: argument checks and
// launches. See include/lfmmi.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <string>
#include <vector>

#include "operators.h"
#include "status.h"

using namespace lfmmi;

static_assert(LFMMI_MAX_TOP == kMaxTop, "the header states the limit");
// partial sums, the factor in 16 bytes, and 28 bytes a tensor and 4
static_assert(LFMMI_GRAD_WORKSPACE_BYTES(0) >= 8 * kGradBlocks + 16 + 4, "the header states the size");

namespace {

constexpr int64_t kCacheBytes = (int64_t)256 << 20;  // behind the L2s

size_t dtype_size(int32_t dtype) { return dtype == LFMMI_F32 ? 4 : 2; }

bool known(int32_t dtype) { return dtype == LFMMI_F32 || dtype == LFMMI_BF16 || dtype == LFMMI_F16; }

bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// What the forward and the backward call check alike.
lfmmi_status check_rows(const void* logits, int32_t dtype, int32_t B, int32_t T, int32_t V,
                        int64_t stride_b, int64_t stride_t, const int32_t* lengths,
                        const void* targets, int32_t target_bytes, float scale)
{
    if (!known(dtype)) return fail(LFMMI_ERR_INVALID_ARG, "unknown dtype");
    if (B < 0 || T < 0) return fail(LFMMI_ERR_INVALID_ARG, "B and T must be >= 0");
    if (V < 1) return fail(LFMMI_ERR_INVALID_ARG, "V must be >= 1");
    if ((int64_t)B * T > INT32_MAX) return fail(LFMMI_ERR_UNSUPPORTED, "B * T exceeds 2^31 - 1");
    if (V > (1 << 30)) return fail(LFMMI_ERR_UNSUPPORTED, "V exceeds 2^30");
    if (stride_b < 0 || stride_t < 0) return fail(LFMMI_ERR_INVALID_ARG, "strides must be >= 0");
    // so that no offset passes 64 bits
    if (stride_b > ((int64_t)1 << 60) / std::max(B, 1) || stride_t > ((int64_t)1 << 60) / std::max(T, 1))
        return fail(LFMMI_ERR_UNSUPPORTED, "strides beyond 2^60 elements");
    if (!(scale >= 1e-6f && scale <= 1e6f))
        return fail(LFMMI_ERR_INVALID_ARG, "scale outside [1e-6, 1e6]");
    if (targets && target_bytes != 4 && target_bytes != 8)
        return fail(LFMMI_ERR_INVALID_ARG, "target_bytes must be 4 or 8");
    if (lengths)
        for (int32_t b = 0; b < B; ++b)
            if (lengths[b] < 0 || lengths[b] > T)
                return fail(LFMMI_ERR_INVALID_ARG, "lengths[" + std::to_string(b) + "] outside [0, T]");
    if (B == 0 || T == 0) return LFMMI_OK;
    if (!logits) return fail(LFMMI_ERR_INVALID_ARG, "logits is null");
    if (!aligned(logits, dtype_size(dtype)) || (targets && !aligned(targets, target_bytes)))
        return fail(LFMMI_ERR_INVALID_ARG, "an array is not aligned to its elements");
    return LFMMI_OK;
}

// Sequences that one launch takes, and their lengths.
int32_t fill_lengths(const int32_t* lengths, int32_t b, int32_t B, SeqLengths* out)
{
    if (!lengths) {
        out->n = 0;
        return B - b;
    }
    const int32_t n = std::min(B - b, kLengthsPerLaunch);
    out->n = n;
    std::copy(lengths + b, lengths + b + n, out->T);
    return n;
}

template <typename U>
U* at(U* p, int64_t i)
{
    return p ? p + i : nullptr;
}

const void* at_bytes(const void* p, int64_t i)
{
    return p ? static_cast<const char*>(p) + i : nullptr;
}

// What both calls write beside gradients.
struct Written {
    uintptr_t norm, workspace, workspace_end;
    bool meets(uintptr_t at, uintptr_t end) const
    {
        return (at < norm + sizeof(float) && norm < end) || (at < workspace_end && workspace < end);
    }
};

Written written_by(int32_t n, const float* norm, const void* workspace)
{
    const uintptr_t w = reinterpret_cast<uintptr_t>(workspace);
    return {reinterpret_cast<uintptr_t>(norm), w, w + (uintptr_t)LFMMI_GRAD_WORKSPACE_BYTES(n)};
}

lfmmi_status fail_written()
{
    return fail(LFMMI_ERR_INVALID_ARG, "norm or workspace overlaps another array");
}

lfmmi_status check_grads(int32_t n, const void* const* grads, const int64_t* counts,
                         const int32_t* dtypes, const float* norm, const void* workspace,
                         int64_t workspace_bytes)
{
    if (n < 0) return fail(LFMMI_ERR_INVALID_ARG, "n must be >= 0");
    if (!norm) return fail(LFMMI_ERR_INVALID_ARG, "norm is null");
    if (n > 0 && (!grads || !counts || !dtypes))
        return fail(LFMMI_ERR_INVALID_ARG, "grads / counts / dtypes is null");
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < LFMMI_GRAD_WORKSPACE_BYTES(n))
        return fail(LFMMI_ERR_INVALID_ARG, "workspace is null, too small or not aligned to 16 bytes");
    const Written written = written_by(n, norm, workspace);
    if (written.norm < written.workspace_end && written.workspace < written.norm + sizeof(float))
        return fail_written();
    for (int32_t i = 0; i < n; ++i) {
        if (!known(dtypes[i])) return fail(LFMMI_ERR_INVALID_ARG, "unknown dtype");
        if (counts[i] < 0) return fail(LFMMI_ERR_INVALID_ARG, "counts must be >= 0");
        if (counts[i] > ((int64_t)1 << 36)) return fail(LFMMI_ERR_UNSUPPORTED, "a count exceeds 2^36");
        if (counts[i] > 0 && !grads[i])
            return fail(LFMMI_ERR_INVALID_ARG, "grads[" + std::to_string(i) + "] is null");
        if (!aligned(grads[i], dtype_size(dtypes[i])))
            return fail(LFMMI_ERR_INVALID_ARG, "a gradient is not aligned to its elements");
        const uintptr_t at = reinterpret_cast<uintptr_t>(grads[i]);
        if (counts[i] > 0 && written.meets(at, at + (uintptr_t)counts[i] * dtype_size(dtypes[i])))
            return fail_written();
    }
    return LFMMI_OK;
}

struct Span {
    uintptr_t at, end;
    bool written;
};

// Whether an array that is written overlaps another array.
bool overlap(std::vector<Span>& spans)
{
    const auto before = [](const Span& a, const Span& b) { return a.at < b.at; };
    if (!std::is_sorted(spans.begin(), spans.end(), before))
        std::sort(spans.begin(), spans.end(), before);
    uintptr_t any = 0, written = 0;  // ends of what came before
    for (const Span& s : spans) {
        if (s.at < written || (s.written && s.at < any)) return true;
        any = std::max(any, s.end);
        if (s.written) written = std::max(written, s.end);
    }
    return false;
}

lfmmi_status check_outs(int32_t n, const void* const* grads, void* const* outs,
                        const int64_t* counts, const int32_t* dtypes, const Written& written)
{
    std::vector<Span> spans;
    spans.reserve(2 * (size_t)n);
    for (int32_t i = 0; i < n; ++i) {
        if (counts[i] == 0) continue;
        const size_t bytes = (size_t)counts[i] * dtype_size(dtypes[i]);
        const uintptr_t in = reinterpret_cast<uintptr_t>(grads[i]);
        uintptr_t out = in;
        if (outs) {
            if (!outs[i]) return fail(LFMMI_ERR_INVALID_ARG, "outs[" + std::to_string(i) + "] is null");
            if (!aligned(outs[i], dtype_size(dtypes[i])))
                return fail(LFMMI_ERR_INVALID_ARG, "an output is not aligned to its elements");
            out = reinterpret_cast<uintptr_t>(outs[i]);
            if (written.meets(out, out + bytes)) return fail_written();
        }
        spans.push_back({out, out + bytes, true});
        if (out != in) spans.push_back({in, in + bytes, false});
    }
    if (overlap(spans))
        return fail(LFMMI_ERR_INVALID_ARG,
                    "an array that is written overlaps another one, or is listed twice");
    return LFMMI_OK;
}

// Units of kGradUnit values of a tensor, from the address before it that kGradAlign divides.
int64_t units_of(const void* grad, int64_t count, int32_t dtype)
{
    const int64_t before = (int64_t)(reinterpret_cast<uintptr_t>(grad) % kGradAlign / dtype_size(dtype));
    return (before + count + kGradUnit - 1) / kGradUnit;
}

struct Grads {
    int32_t n;
    const void* const* in;
    void* const* out;  // or null: in place
    const int64_t* counts;
    const int32_t* dtypes;
};

void set(GradList* l, const Grads& g, int32_t i, int64_t)
{
    l->out[l->n] = g.out ? g.out[i] : const_cast<void*>(g.in[i]);
    l->count[l->n] = g.counts[i] << 2 | g.dtypes[i];
}

void set(GradPlaces* l, const Grads& g, int32_t i, int64_t units)
{
    const int64_t before = (int64_t)(reinterpret_cast<uintptr_t>(g.in[i]) % kGradAlign / dtype_size(g.dtypes[i]));
    l->rest[l->n] = (uint16_t)((units * kGradUnit - before - g.counts[i]) << 2 | g.dtypes[i]);
}

// Tensors from `from` on that a list takes, and the one behind them; `units` is counted on.
template <typename List>
int32_t fill_list(const Grads& g, int32_t from, int64_t* units, List* l)
{
    l->n = 0;
    int32_t i = from;
    for (; i < g.n && l->n < List::kTensors; ++i) {
        if (g.counts[i] == 0) continue;
        const int64_t of_it = units_of(g.in[i], g.counts[i], g.dtypes[i]);
        l->in[l->n] = g.in[i];
        l->first[l->n] = (int32_t)*units;
        set(l, g, i, of_it);
        *units += of_it;
        ++l->n;
    }
    l->first[l->n] = (int32_t)*units;
    return i;
}

// Launches for `tensors` tensors that are not empty.
template <typename List>
hipError_t launch_list(const Grads& g, int32_t tensors, const GradCall& c, hipStream_t stream)
{
    List l;
    int64_t units = 0;
    if (tensors <= List::kTensors) {
        fill_list(g, 0, &units, &l);
        return launch_grads(l, c, stream);
    }
    GradTable t;
    t.in = reinterpret_cast<const void**>(c.partials + kGradBlocks + 2);
    t.out = const_cast<void**>(t.in) + tensors;
    t.count = reinterpret_cast<int64_t*>(t.out + tensors);
    t.first = reinterpret_cast<int32_t*>(t.count + tensors);
    for (int32_t i = 0, at = 0; at < tensors; at += l.n) {
        i = fill_list(g, i, &units, &l);
        const hipError_t e = launch_grad_table(l, at, t, stream);
        if (e != hipSuccess) return e;
    }
    return launch_grads(t, c, stream);
}

// The norm, and with `scale` outs.
lfmmi_status run_grads(int32_t n, const void* const* grads, void* const* outs,
                       const int64_t* counts, const int32_t* dtypes, bool scale, float max_norm,
                       float* norm, void* workspace, hipStream_t stream)
{
    int64_t units = 0, bytes = 0;
    int32_t tensors = 0;
    bool in_place = true;
    for (int32_t i = 0; i < n; ++i) {
        if (counts[i] == 0) continue;
        ++tensors;
        units += units_of(grads[i], counts[i], dtypes[i]);
        bytes += counts[i] * (int64_t)dtype_size(dtypes[i]);
        in_place = in_place && (!outs || outs[i] == grads[i]);
    }
    if (units > INT32_MAX) return fail(LFMMI_ERR_UNSUPPORTED, "more than 2^44 values");
    GradCall c{};
    c.n = tensors;
    c.units = (int32_t)units;
    c.blocks = std::min(c.units, kGradBlocks);
    // what the second pass finds in the cache again; more than that goes past it
    const int64_t kept = scale ? kCacheBytes * 3 / 4 : 0;
    c.keep = bytes <= kCacheBytes ? 256 : (int32_t)(256 * kept / bytes);
    c.scale = scale;
    c.in_place = in_place;
    c.max_norm = max_norm;
    c.norm = norm;
    c.partials = static_cast<double*>(workspace);
    c.factor = reinterpret_cast<float*>(c.partials + kGradBlocks);
    const Grads g{n, grads, outs, counts, dtypes};
    // (replays of clipping in place 150 tensors of 30,000 fp32 values: 7.4 us by one list, 10.9 by a table that two
    // launches write; of 800,000: 80.7, 85.2)
    const hipError_t e = in_place ? launch_list<GradPlaces>(g, tensors, c, stream)
                                  : launch_list<GradList>(g, tensors, c, stream);
    return e == hipSuccess ? LFMMI_OK : fail_hip(e, "kernel launch");
}

}  // namespace

extern "C" {

lfmmi_status lfmmi_token_logprobs_workspace(int32_t dtype, int32_t B, int32_t T, int32_t V,
                                            int32_t top_k, int64_t* bytes)
{
    if (!bytes) return fail(LFMMI_ERR_INVALID_ARG, "bytes is null");
    if (!known(dtype) || B < 0 || T < 0 || V < 1 || top_k < 0 || top_k > kMaxTop || top_k > V)
        return fail(LFMMI_ERR_INVALID_ARG, "unknown dtype, or a size out of range");
    if (V > (1 << 30)) return fail(LFMMI_ERR_UNSUPPORTED, "V exceeds 2^30");
    if ((int64_t)B * T > INT32_MAX) return fail(LFMMI_ERR_UNSUPPORTED, "B * T exceeds 2^31 - 1");
    *bytes = B > 0 && T > 0 ? (int64_t)plan_tokens((int64_t)B * T, V, top_k).workspace : 0;
    return LFMMI_OK;
}

lfmmi_status lfmmi_token_logprobs(const void* logits, int32_t dtype, int32_t B, int32_t T,
                                  int32_t V, int64_t stride_b, int64_t stride_t,
                                  const int32_t* lengths, const void* targets,
                                  int32_t target_bytes, float scale, int32_t top_k, float* logp,
                                  float* entropy, float* stats, int32_t* top_id, float* top_logp,
                                  int32_t* status, void* workspace, int64_t workspace_bytes,
                                  void* hip_stream)
try {
    lfmmi_status st = check_rows(logits, dtype, B, T, V, stride_b, stride_t, lengths, targets,
                                 target_bytes, scale);
    if (st != LFMMI_OK) return st;
    if (top_k < 0 || top_k > V) return fail(LFMMI_ERR_INVALID_ARG, "top_k outside [0, V]");
    if (top_k > kMaxTop) return fail(LFMMI_ERR_UNSUPPORTED, "top_k exceeds LFMMI_MAX_TOP");
    if (logp && !targets) return fail(LFMMI_ERR_INVALID_ARG, "logp without targets");
    if (B == 0 || T == 0) return LFMMI_OK;
    const TokenPlan plan = plan_tokens((int64_t)B * T, V, top_k);
    if (plan.workspace > 0 &&
        (!workspace || !aligned(workspace, 16) || workspace_bytes < (int64_t)plan.workspace))
        return fail(LFMMI_ERR_INVALID_ARG, "workspace is null, too small or not aligned to 16 bytes");
    const int64_t size = (int64_t)dtype_size(dtype);
    for (int32_t b = 0; b < B;) {
        SeqLengths lens;
        const int32_t n = fill_lengths(lengths, b, B, &lens);
        const int64_t row = (int64_t)b * T;
        TokenParams p{};
        p.x = at_bytes(logits, b * stride_b * size);
        p.stride_b = stride_b;
        p.stride_t = stride_t;
        p.targets = at_bytes(targets, row * target_bytes);
        p.target_bytes = target_bytes;
        p.B = n;
        p.T = T;
        p.V = V;
        p.top_k = top_id || top_logp ? top_k : 0;
        p.scale = scale;
        p.logp = at(logp, row);
        p.entropy = at(entropy, row);
        p.stats = at(stats, 2 * row);
        p.top_id = at(top_id, row * top_k);
        p.top_logp = at(top_logp, row * top_k);
        p.status = at(status, row);
        p.once = (int64_t)B * T * V * size > kCacheBytes;
        p.parts = plan.parts;
        p.part_size = plan.part_size;
        p.workspace = workspace;
        const hipError_t e =
            launch_token_logprobs(p, lens, dtype, static_cast<hipStream_t>(hip_stream));
        if (e != hipSuccess) return fail_hip(e, "kernel launch");
        b += n;
    }
    return LFMMI_OK;
} catch (...) {
    return fail_memory();
}

lfmmi_status lfmmi_token_logprobs_backward(const void* logits, int32_t dtype, int32_t B, int32_t T,
                                           int32_t V, int64_t stride_b, int64_t stride_t,
                                           const int32_t* lengths, const void* targets,
                                           int32_t target_bytes, float scale, const float* stats,
                                           const float* entropy, const float* grad_logp,
                                           const float* grad_entropy, void* grad, void* hip_stream)
try {
    lfmmi_status st = check_rows(logits, dtype, B, T, V, stride_b, stride_t, lengths, targets,
                                 target_bytes, scale);
    if (st != LFMMI_OK) return st;
    if (grad_logp && !targets) return fail(LFMMI_ERR_INVALID_ARG, "grad_logp without targets");
    if (grad_entropy && !entropy) return fail(LFMMI_ERR_INVALID_ARG, "grad_entropy without entropy");
    if (B == 0 || T == 0) return LFMMI_OK;
    if (!stats || !grad) return fail(LFMMI_ERR_INVALID_ARG, "stats / grad is null");
    const int64_t size = (int64_t)dtype_size(dtype);
    if (!aligned(grad, size)) return fail(LFMMI_ERR_INVALID_ARG, "an array is not aligned to its elements");
    // in place means the very same elements
    const bool same = logits == grad && (T == 1 || stride_t == V) && (B == 1 || stride_b == (int64_t)T * V);
    if (!same) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(logits), g = reinterpret_cast<uintptr_t>(grad);
        const uintptr_t x_end = x + (uintptr_t)(((B - 1) * stride_b + (T - 1) * stride_t + V) * size);
        if (g < x_end && x < g + (uintptr_t)((int64_t)B * T * V * size))
            return fail(LFMMI_ERR_INVALID_ARG, "grad overlaps logits that are not contiguous");
    }
    for (int32_t b = 0; b < B;) {
        SeqLengths lens;
        const int32_t n = fill_lengths(lengths, b, B, &lens);
        const int64_t row = (int64_t)b * T;
        TokenGradParams p{};
        p.x = at_bytes(logits, b * stride_b * size);
        p.stride_b = stride_b;
        p.stride_t = stride_t;
        p.targets = at_bytes(targets, row * target_bytes);
        p.target_bytes = target_bytes;
        p.B = n;
        p.T = T;
        p.V = V;
        p.scale = scale;
        p.stats = stats + 2 * row;
        p.entropy = at(entropy, row);
        p.grad_logp = at(grad_logp, row);
        p.grad_entropy = at(grad_entropy, row);
        p.grad = static_cast<char*>(grad) + row * V * size;
        p.once = (int64_t)B * T * V * size > kCacheBytes;
        const hipError_t e = launch_token_grad(p, lens, dtype, static_cast<hipStream_t>(hip_stream));
        if (e != hipSuccess) return fail_hip(e, "kernel launch");
        b += n;
    }
    return LFMMI_OK;
} catch (...) {
    return fail_memory();
}

lfmmi_status lfmmi_grad_norm(int32_t n, const void* const* grads, const int64_t* counts,
                             const int32_t* dtypes, float* norm, void* workspace,
                             int64_t workspace_bytes, void* hip_stream)
try {
    const lfmmi_status st = check_grads(n, grads, counts, dtypes, norm, workspace, workspace_bytes);
    if (st != LFMMI_OK) return st;
    return run_grads(n, grads, nullptr, counts, dtypes, false, 0.f, norm, workspace,
                     static_cast<hipStream_t>(hip_stream));
} catch (...) {
    return fail_memory();
}

lfmmi_status lfmmi_clip_grads(int32_t n, const void* const* grads, void* const* outs,
                              const int64_t* counts, const int32_t* dtypes, float max_norm,
                              float* norm, void* workspace, int64_t workspace_bytes,
                              void* hip_stream)
try {
    lfmmi_status st = check_grads(n, grads, counts, dtypes, norm, workspace, workspace_bytes);
    if (st != LFMMI_OK) return st;
    if (!(max_norm >= 0.f)) return fail(LFMMI_ERR_INVALID_ARG, "max_norm must be >= 0");
    if ((st = check_outs(n, grads, outs, counts, dtypes, written_by(n, norm, workspace))) != LFMMI_OK)
        return st;
    return run_grads(n, grads, outs, counts, dtypes, true, max_norm, norm, workspace,
                     static_cast<hipStream_t>(hip_stream));
} catch (...) {
    return fail_memory();
}

}  // extern "C"
