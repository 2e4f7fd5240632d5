// C ABI of the operators that take no model: argument checks in front of the launches, and the 4-bit quantiser (host code).
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "ops.h"

using namespace rnnlm;

namespace {

bool known_dtype(int dtype) { return dtype == RNNLM_F32 || dtype == RNNLM_BF16; }
size_t size_of(int dtype) { return dtype == RNNLM_BF16 ? 2 : 4; }
constexpr int kMaxWords = 1 << 30, kMaxUnits = 1 << 16, kMaxRows = 1 << 24;
constexpr int kMaxGroups = 1 << 21;                  // rows that take a workgroup each: a grid holds fewer than 2^32 threads
constexpr long long kMaxStride = 1ll << 40;
// Can `rows` rows of n elements of es bytes lie `ld` elements apart?  Their bytes have to be a number of 63 bits, which offsets and the search for
// shared bytes count on.
bool strides(long long rows, long long n, long long ld, size_t es) { return ld >= n && ld <= kMaxStride && (rows <= 1 || ld <= INT64_MAX / (long long)es / rows); }

// `rows` rows of `row` bytes, `stride` bytes apart.
struct Range {
    const void *p;
    size_t row, rows, stride;
    Range(const void *p, size_t bytes) : p(p), row(bytes), rows(1), stride(bytes) {}
    Range(const void *p, long long rows, long long n, long long ld, size_t es) : p(p), row((size_t)n * es), rows((size_t)rows), stride((size_t)ld * es) {}
    size_t bytes() const { return (rows - 1) * stride + row; }
    // Do they share a byte?  Of two that lie interleaved, rows of one in the gaps of the other, this is known where their strides are equal.
    bool meets(const Range &o) const {
        if (!p || !o.p || !row || !o.row || !rows || !o.rows) return false;
        const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(o.p);
        if (a >= b + o.bytes() || b >= a + bytes()) return false;
        if (stride != o.stride || rows == 1 || o.rows == 1) return true;
        const size_t d = a <= b ? (b - a) % stride : (stride - (a - b) % stride) % stride;   // of o's rows behind this one's
        return d < row || d + o.row > stride;
    }
};
// Does an output share a byte with an input or with another output?
template <size_t NI, size_t NO>
bool overlap(const Range (&ins)[NI], const Range (&outs)[NO]) {
    for (size_t o = 0; o < NO; ++o) {
        for (const Range &i : ins)
            if (outs[o].meets(i)) return true;
        for (size_t q = 0; q < o; ++q)
            if (outs[o].meets(outs[q])) return true;
    }
    return false;
}
bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int check_distill(int N, int V, int K, int dtype, const void *logits, long long ld, const int32_t *teacher_word, const float *teacher_logit,
                  const int32_t *label, float T, float a, const float *row_weight, const void *grad, long long grad_ld) {
    if (N < 0 || V <= 0 || K < 0 || !known_dtype(dtype)) return RNNLM_EINVAL;
    if (V > kMaxWords || N > kMaxGroups || K > RNNLM_DISTILL_MAX_K) return RNNLM_ERANGE;
    if (!strides(N, V, ld, size_of(dtype)) || (grad && !strides(N, V, grad_ld, size_of(dtype)))) return RNNLM_EINVAL;
    if (!(T > 0.f) || !std::isfinite(T) || !(a >= 0.f && a <= 1.f) || (!label && a != 0.f)) return RNNLM_EINVAL;
    if (N == 0) return RNNLM_OK;
    if (!logits || (K > 0 && (!teacher_word || !teacher_logit))) return RNNLM_EINVAL;
    if (!aligned(logits, size_of(dtype)) || !aligned(grad, size_of(dtype)) || !aligned(teacher_word, 4) || !aligned(teacher_logit, 4) ||
        !aligned(label, 4) || !aligned(row_weight, 4))
        return RNNLM_EINVAL;
    return RNNLM_OK;
}

}  // namespace

extern "C" {

int rnnlm_q4_matvec(int B, int V, int H, int group, const uint8_t *codes, long long code_ld, int scale_dtype, const void *scale,
                    const uint8_t *zero, const float *bias, int x_dtype, const void *x, long long x_ld, int y_dtype, void *y, long long y_ld,
                    void *hip_stream) {
    if (B < 0 || V <= 0 || H <= 0 || (group != 32 && group != 64 && group != 128)) return RNNLM_EINVAL;
    if (!known_dtype(scale_dtype) || !known_dtype(x_dtype) || !known_dtype(y_dtype)) return RNNLM_EINVAL;
    if (V > kMaxWords || H > kMaxUnits || B > kMaxRows) return RNNLM_ERANGE;
    const long long row = (H + 1) / 2, groups = (H + group - 1) / group;
    if (!strides(V, row, code_ld, 1) || !strides(B, H, x_ld, size_of(x_dtype)) || !strides(B, V, y_ld, size_of(y_dtype))) return RNNLM_EINVAL;
    if (B == 0) return RNNLM_OK;
    if (!codes || !scale || !x || !y) return RNNLM_EINVAL;
    if (!aligned(scale, size_of(scale_dtype)) || !aligned(x, size_of(x_dtype)) || !aligned(y, size_of(y_dtype)) || !aligned(bias, 4)) return RNNLM_EINVAL;
    const Range ins[] = {{codes, V, row, code_ld, 1}, {scale, (size_t)groups * V * size_of(scale_dtype)}, {zero, (size_t)groups * V},
                         {bias, (size_t)V * 4}, {x, B, H, x_ld, size_of(x_dtype)}};
    const Range outs[] = {{y, B, V, y_ld, size_of(y_dtype)}};
    if (overlap(ins, outs)) return RNNLM_EINVAL;
    const Q4Args a = {B, V, H, group, codes, code_ld, scale, zero, bias, x, x_ld, y, y_ld, scale_dtype == RNNLM_BF16, x_dtype == RNNLM_BF16,
                      y_dtype == RNNLM_BF16};
    return launch_q4(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? RNNLM_OK : RNNLM_EDEVICE;
}

int rnnlm_q4_quantize(int V, int H, int group, const float *w, uint8_t *codes, float *scale, uint8_t *zero) {
    if (V <= 0 || H <= 0 || (group != 32 && group != 64 && group != 128) || !w || !codes || !scale) return RNNLM_EINVAL;
    if (V > kMaxWords || H > kMaxUnits) return RNNLM_ERANGE;
    const size_t row = ((size_t)H + 1) / 2;
    std::fill(codes, codes + row * V, (uint8_t)0);
    for (int v = 0; v < V; ++v) {
        const float *wv = w + (size_t)v * H;
        for (int j0 = 0, g = 0; j0 < H; j0 += group, ++g) {
            const int j1 = std::min(H, j0 + group);
            float lo = 0.f, hi = 0.f;
            for (int j = j0; j < j1; ++j) {
                if (!std::isfinite(wv[j])) return RNNLM_EINVAL;
                lo = std::min(lo, wv[j]);
                hi = std::max(hi, wv[j]);
            }
            // the spread in double: of two large magnitudes it may pass the range of a float
            const double step = zero ? ((double)hi - (double)lo) / 15 : (double)std::max(hi, -lo) / 7;
            const float s = (float)step;
            const int z = !zero ? 8 : s > 0.f ? std::min(15, (int)nearbyint(-(double)lo / (double)s)) : 0;
            scale[(size_t)g * V + v] = s;
            if (zero) zero[(size_t)g * V + v] = (uint8_t)z;
            for (int j = j0; j < j1; ++j) {
                const int c = s > 0.f ? z + (int)nearbyint((double)wv[j] / (double)s) : z;
                const int q = std::min(15, std::max(zero ? 0 : 1, c));
                codes[(size_t)v * row + j / 2] |= (uint8_t)(q << (4 * (j & 1)));
            }
        }
    }
    return RNNLM_OK;
}

size_t rnnlm_sample_workspace_bytes(int N, int V) { return N <= 0 || V <= 0 ? 0 : sample_workspace_bytes(N, V); }

int rnnlm_sample(int N, int V, int dtype, const void *logits, long long ld, const float *temperature, const int32_t *top_k, const float *top_p,
                 const float *min_p, const float *u, int32_t *word, float *logprob, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (N < 0 || V <= 0 || !known_dtype(dtype)) return RNNLM_EINVAL;
    if (V > kMaxWords || N > kMaxGroups) return RNNLM_ERANGE;
    if (!strides(N, V, ld, size_of(dtype))) return RNNLM_EINVAL;
    if (N == 0) return RNNLM_OK;
    if (!logits || !u || !word) return RNNLM_EINVAL;
    if (!aligned(logits, size_of(dtype)) || !aligned(temperature, 4) || !aligned(top_k, 4) || !aligned(top_p, 4) || !aligned(min_p, 4) ||
        !aligned(u, 4) || !aligned(word, 4) || !aligned(logprob, 4))
        return RNNLM_EINVAL;
    const size_t need = sample_workspace_bytes(N, V), row = (size_t)N * 4;
    if (!workspace || workspace_bytes < need || !aligned(workspace, 16)) return RNNLM_EWORKSPACE;
    const Range ins[] = {{logits, N, V, ld, size_of(dtype)}, {temperature, row}, {top_k, row}, {top_p, row}, {min_p, row}, {u, row}};
    const Range outs[] = {{word, row}, {logprob, row}, {workspace, need}};
    if (overlap(ins, outs)) return RNNLM_EINVAL;
    const SampleArgs a = {N, V, dtype == RNNLM_BF16, logits, ld, temperature, top_k, top_p, min_p, u, word, logprob, workspace};
    return launch_sample(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? RNNLM_OK : RNNLM_EDEVICE;
}

size_t rnnlm_distill_workspace_bytes(int N, int V) { return N <= 0 || V <= 0 ? 0 : distill_workspace_most(N, V); }

int rnnlm_distill(int N, int V, int K, int dtype, const void *logits, long long ld, const int32_t *teacher_word, const float *teacher_logit,
                  const int32_t *label, float temperature, float label_weight, const float *row_weight, float *loss, float *stats, void *grad,
                  long long grad_ld, void *workspace, size_t workspace_bytes, void *hip_stream) {
    const int rc = check_distill(N, V, K, dtype, logits, ld, teacher_word, teacher_logit, label, temperature, label_weight, row_weight, grad, grad_ld);
    if (rc != RNNLM_OK || N == 0) return rc;
    if (!loss || !stats || !aligned(loss, 4) || !aligned(stats, 4)) return RNNLM_EINVAL;
    const size_t need = distill_workspace_bytes(N, V), es = size_of(dtype), nk = (size_t)N * K * 4;
    if (!workspace || workspace_bytes < need || !aligned(workspace, 16)) return RNNLM_EWORKSPACE;
    const bool in_place = grad == logits && grad_ld == ld;
    const Range ins[] = {{in_place ? nullptr : logits, N, V, ld, es}, {teacher_word, nk}, {teacher_logit, nk}, {label, (size_t)N * 4}, {row_weight, (size_t)N * 4}};
    const Range outs[] = {{loss, (size_t)N * 4}, {stats, (size_t)N * 16}, {grad, N, V, grad_ld, es}, {workspace, need}};
    if (overlap(ins, outs)) return RNNLM_EINVAL;
    if (in_place) {
        const Range z[] = {{logits, N, V, ld, es}}, others[] = {{loss, (size_t)N * 4}, {stats, (size_t)N * 16}, {workspace, need}};
        if (overlap(z, others)) return RNNLM_EINVAL;
    }
    const DistillArgs a = {N, V, K, dtype == RNNLM_BF16, logits, ld, teacher_word, teacher_logit, label, temperature, label_weight, row_weight,
                           loss, stats, grad, grad_ld, workspace};
    return launch_distill(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? RNNLM_OK : RNNLM_EDEVICE;
}

int rnnlm_distill_backward(int N, int V, int K, int dtype, const void *logits, long long ld, const int32_t *teacher_word,
                           const float *teacher_logit, const int32_t *label, float temperature, float label_weight, const float *row_weight,
                           const float *stats, void *grad, long long grad_ld, void *hip_stream) {
    const int rc = check_distill(N, V, K, dtype, logits, ld, teacher_word, teacher_logit, label, temperature, label_weight, row_weight, grad, grad_ld);
    if (rc != RNNLM_OK || N == 0) return rc;
    if (!grad || !stats || !aligned(stats, 4)) return RNNLM_EINVAL;
    const size_t es = size_of(dtype), nk = (size_t)N * K * 4;
    const bool in_place = grad == logits && grad_ld == ld;
    const Range ins[] = {{in_place ? nullptr : logits, N, V, ld, es}, {teacher_word, nk}, {teacher_logit, nk}, {label, (size_t)N * 4},
                         {row_weight, (size_t)N * 4}, {stats, (size_t)N * 16}};
    const Range outs[] = {{grad, N, V, grad_ld, es}};
    if (overlap(ins, outs)) return RNNLM_EINVAL;
    const DistillArgs a = {N, V, K, dtype == RNNLM_BF16, logits, ld, teacher_word, teacher_logit, label, temperature, label_weight, row_weight,
                           nullptr, const_cast<float *>(stats), grad, grad_ld, nullptr};
    return launch_distill_backward(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? RNNLM_OK : RNNLM_EDEVICE;
}

}  // extern "C"
