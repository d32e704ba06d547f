// Plain-struct interface between the C ABI (operators.cpp) and the kernels on token log
// probabilities (tokens.hip) and on gradients (grads.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

namespace lfmmi {

constexpr int kMaxTop = 64;  // LFMMI_MAX_TOP

// Lengths travel as a kernel argument, this many sequences a launch (a call with more of
// them is cut into several); n == 0: every sequence has all T rows.
constexpr int kLengthsPerLaunch = 256;
struct SeqLengths {
    int32_t n;
    int32_t T[kLengthsPerLaunch];
};

struct TokenParams {
    const void* x;        // logits of sequence 0 of this launch; element (b, t, i) at
    int64_t stride_b;     // b * stride_b + t * stride_t + i
    int64_t stride_t;
    const void* targets;  // [B, T] or null
    int32_t target_bytes; // 4 or 8
    int32_t B, T, V;      // of this launch
    int32_t top_k;
    float scale;
    float* logp;          // [B, T] or null, and so on
    float* entropy;
    float* stats;         // [B, T, 2]
    int32_t* top_id;      // [B, T, top_k]
    float* top_logp;
    int32_t* status;
    bool once;  // the logits are too many for the caches
    int32_t parts, part_size;  // a row's logits are cut into `parts` parts of part_size
    void* workspace;
};

// How a call's rows are cut, and the bytes of workspace that takes.
constexpr int kMaxParts = 64, kMaxPartKeys = 256;  // alternatives of all parts of a row
struct TokenPlan {
    int32_t parts, part_size;
    size_t workspace;
};
TokenPlan plan_tokens(int64_t rows, int V, int top_k);

struct TokenGradParams {
    const void* x;
    int64_t stride_b, stride_t;
    const void* targets;
    int32_t target_bytes;
    int32_t B, T, V;
    float scale;
    const float* stats;
    const float* entropy;
    const float* grad_logp;     // or null
    const float* grad_entropy;  // or null
    void* grad;                 // [B, T, V] contiguous
    bool once;                  // the logits are too many for the caches
    int32_t pieces, piece;      // how a row is cut (set by the launch)
};

// dtype: lfmmi_dtype
hipError_t launch_token_logprobs(const TokenParams& p, const SeqLengths& lens, int dtype,
                                 hipStream_t stream);
hipError_t launch_token_grad(const TokenGradParams& p, const SeqLengths& lens, int dtype,
                             hipStream_t stream);

// Gradient tensors: values of tensor i are cut into units of kGradUnit, counted from the address before
// its first that kGradAlign divides; unit numbers run through the tensors and begin with first[i]; first[n]
// is how many there are.
constexpr int kGradUnit = 8192;
constexpr int kGradAlign = 128;    // bytes
constexpr int kGradBlocks = 2048;  // most workgroups of a launch: one partial sum each
constexpr int kGradAlone = 1024;   // units up to which a call that scales does without a launch for the norm
struct GradList {  // tensors that travel as a kernel argument, of 4 KB with a GradCall
    static constexpr int kTensors = 128;
    const void* in[kTensors];
    void* out[kTensors];
    int64_t count[kTensors];  // << 2 | lfmmi_dtype
    int32_t first[kTensors + 1];
    int32_t n;
};
struct GradPlaces {  // more of them, that are not written, or in place
    static constexpr int kTensors = 280;
    const void* in[kTensors];
    int32_t first[kTensors + 1];
    int32_t n;
    uint16_t rest[kTensors];  // what its last unit has behind the tensor, << 2 | lfmmi_dtype
};
struct GradTable {  // the same in the workspace, for any number
    const void** in;
    void** out;
    int64_t* count;
    int32_t* first;
};

struct GradCall {
    int32_t n, units, blocks;
    int32_t keep;      // 256ths of a workgroup's units, its last ones, that stay in the caches
    bool scale;        // the norm alone otherwise
    bool in_place;     // all tensors are
    float max_norm;
    float* norm;
    float* factor;     // [1] in the workspace
    double* partials;  // [blocks] there
};

static_assert(sizeof(GradList) + sizeof(GradCall) <= 4096 && sizeof(GradPlaces) + sizeof(GradCall) <= 4096, "");
static_assert(kGradUnit << 2 <= 1 << 16, "`rest` has 16 bits");

// Writes tensors from..from + l.n - 1 of a table, and the unit behind them.
hipError_t launch_grad_table(const GradList& l, int from, const GradTable& t, hipStream_t stream);
hipError_t launch_grad_table(const GradPlaces& l, int from, const GradTable& t, hipStream_t stream);
hipError_t launch_grads(const GradList& l, const GradCall& c, hipStream_t stream);
hipError_t launch_grads(const GradPlaces& l, const GradCall& c, hipStream_t stream);
hipError_t launch_grads(const GradTable& t, const GradCall& c, hipStream_t stream);

}  // namespace lfmmi
