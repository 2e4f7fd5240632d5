// Internal declarations of the operators that take no model: 4-bit products, draw of a word, distillation.
#pragma once

#include "rnnlm_internal.h"

namespace rnnlm {

struct Q4Args {
    int B, V, H, group;        // group: 32, 64 or 128
    const uint8_t *codes;      // [V][code_ld] bytes
    long long code_ld;
    const void *scale;         // [groups][V]
    const uint8_t *zero;       // [groups][V] or null: 8
    const float *bias;         // [V] or null
    const void *x;             // [B][x_ld]
    long long x_ld;
    void *y;                   // [B][y_ld]
    long long y_ld;
    bool scale_bf16, x_bf16, y_bf16;
};
hipError_t launch_q4(const Q4Args &a, hipStream_t stream);

struct SampleArgs {
    int N, V;
    bool bf16;
    const void *logits;
    long long ld;
    const float *temperature;  // nullable: 1
    const int32_t *top_k;      // nullable: all
    const float *top_p;        // nullable: 1
    const float *min_p;        // nullable: 0
    const float *u;
    int32_t *word;
    float *logprob;            // nullable
    void *ws;
};
size_t sample_workspace_bytes(int N, int V);
// Words that can be listed of a row in segments.  In bfloat16 a bin is one logit, and some hundredth of the words may have it.
__host__ __device__ constexpr int long_list(int V) { return V / 16 > 8192 ? V / 16 : 8192; }
// Does the launch that draws keep the list in LDS?  `listed` counts the words that there are, and may be more than the list's length.
constexpr int kLongHeld = 12288;
__host__ __device__ constexpr bool list_in_lds(int listed, int V) { return listed <= long_list(V) && listed <= kLongHeld; }
hipError_t launch_sample(const SampleArgs &a, hipStream_t stream);

struct DistillArgs {
    int N, V, K;
    bool bf16;
    const void *logits;
    long long ld;
    const int32_t *teacher_word;
    const float *teacher_logit;
    const int32_t *label;      // nullable
    float T, a;                // temperature, weight of the label's part
    const float *row_weight;   // nullable: 1
    float *loss;
    float *stats;              // [N][4]
    void *grad;                // nullable
    long long grad_ld;
    void *ws;
};
size_t distill_workspace_bytes(int N, int V);   // of this call
size_t distill_workspace_most(int N, int V);    // of any call of no more rows and words
// Segments of a row: how many, and their length (a multiple of a vector of E elements).
struct Cut { int segments, len; };
inline Cut cut_row(int V, int E, int segments) {
    const int vectors = (V + E - 1) / E, per = (vectors + segments - 1) / segments;
    return Cut{(vectors + per - 1) / per, per * E};
}
// Of the gradient alone: some 8192 words each, and more where a grid of fewer than 2^32 threads would not hold as many workgroups.
constexpr int kDistillThreads = 256;
constexpr long long kDistillGroups = 0xFFFFFFFFll / kDistillThreads;
inline Cut cut_for_backward(int N, int V, int E) {
    const int segments = (V + 8191) / 8192;
    return cut_row(V, E, segments * (long long)N <= kDistillGroups ? segments : (int)(kDistillGroups / N));
}
hipError_t launch_distill(const DistillArgs &a, hipStream_t stream);
hipError_t launch_distill_backward(const DistillArgs &a, hipStream_t stream);

}  // namespace rnnlm
