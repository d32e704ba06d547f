// Plain-struct interface between the C ABI (layers.cpp) and the kernels around an output
// layer: embeddings (embed.hip), dropout and norms (norm.hip), drafted tokens (verify.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "operators.h"

namespace lfmmi {

// Random bits and what is done with them. threshold: in 65536ths, 0 where nothing is dropped.
struct Draw {
    uint64_t seed, offset;
    const int64_t* step;  // or null; added to offset
    int32_t threshold;
    float factor;  // of what is kept
};

struct DropoutParams {
    const void* x;
    void* y;
    int64_t stride_x, stride_y;
    int32_t R, D;
    Draw draw;
    bool once;  // what is written is too much for the caches
};
hipError_t launch_dropout(const DropoutParams& p, int dtype, hipStream_t stream);

struct NormParams {
    const void* x;         // of sequence 0 of this launch; row (b, t) at b * x_stride_b + t * x_stride_t
    const void* residual;  // or null
    int64_t x_stride_b, x_stride_t, r_stride_b, r_stride_t;
    int32_t B, T, D;       // of this launch
    int64_t row;           // of the call, that the launch begins with
    const void* weight;    // or null
    bool weight_f32;
    float eps;
    Draw draw;
    void* sum;             // [B, T, D] or null, and so on
    void* y;
    float* rstd;           // [B, T]
    uint8_t* q;
    float* q_scale;
    bool once;             // an output is too much for the caches
};
hipError_t launch_norm(const NormParams& p, const SeqLengths& lens, int dtype, hipStream_t stream);

int norm_blocks(int64_t rows, int D, int dtype);  // workgroups of a backward launch, each with a row of partial sums
struct NormGradParams {
    const void* h;
    int64_t stride_b, stride_t;
    int32_t B, T, D;
    int64_t row;
    const void* weight;
    bool weight_f32;
    Draw draw;
    const float* rstd;
    const void* grad_y;    // or null
    const void* grad_sum;  // or null
    void* grad_x;          // or null
    void* grad_residual;   // or null
    float* partials;       // [blocks, D] or null
    int32_t blocks;
    bool add;              // to the partial sums of an earlier launch
    bool once;
};
hipError_t launch_norm_grad(const NormGradParams& p, const SeqLengths& lens, int dtype, hipStream_t stream);
hipError_t launch_norm_weight(const float* partials, int blocks, int D, void* grad_weight, int dtype,
                              hipStream_t stream);

struct EmbedParams {
    const void* table;
    int64_t stride;
    const void* tokens;
    int32_t token_bytes;
    int32_t B, T, V, D;
    float scale;
    void* out;
    int32_t* status;  // or null
    bool once;
};
hipError_t launch_embed(const EmbedParams& p, const SeqLengths& lens, int dtype, hipStream_t stream);

// The gradient of a table: positions sorted by token, then every row of the table the sum of its positions' rows.
struct EmbedPlan {
    int32_t bits, passes;   // of a digit, and how many there are
    int32_t tile, tiles;    // positions that a workgroup sorts, and how many tiles there are
    int32_t pieces;         // whole pieces of the sorted positions
    size_t keys, order, hist, starts, partials, bytes;  // offsets in the workspace
};
constexpr int kEmbedPiece = 16;  // positions
EmbedPlan plan_embed(int64_t N, int V, int D);

struct EmbedGradParams {
    const void* g;  // row (b, t) at b * stride_b + t * stride_t
    int64_t stride_b, stride_t;
    const void* tokens;
    int32_t token_bytes;
    int32_t B, T, V, D;
    float scale;
    bool accumulate;
    void* grad;  // [V, D]
    void* workspace;
    EmbedPlan plan;
    bool once;
};
// The keys of sequences b..b + n - 1, where the lengths of all do not fit a launch (`lens` null then); all of the rest.
hipError_t launch_embed_keys(const EmbedGradParams& p, const SeqLengths& lens, int b, int n, hipStream_t stream);
hipError_t launch_embed_grad(const EmbedGradParams& p, const SeqLengths* lens, int dtype, hipStream_t stream);

struct VerifyParams {
    const void* x;  // [B, K + 1, V]
    const void* draft;  // [B, K, V] or null
    int64_t stride_b, stride_t, draft_stride_b, draft_stride_t;
    const void* drafted;  // [B, K]
    int32_t token_bytes;
    int32_t B, K, V;  // of this launch
    float scale, draft_scale;
    const float* uniforms;  // [B, K + 1], or null: greedy
    int32_t* accepted;
    int32_t* tokens;
    int32_t* status;
    int32_t parts;
    void* workspace;
};
constexpr int kVerifyPart = 2048;  // logits of a row that a wave takes
size_t verify_workspace(int64_t B, int K, int V);
hipError_t launch_verify(const VerifyParams& p, const SeqLengths& lens, int dtype, hipStream_t stream);

}  // namespace lfmmi
