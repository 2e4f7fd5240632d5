// Loss of rows of logits against a teacher's top logits and labels, and its gradient.
#include "device_utils.h"
#include "ops.h"

namespace rnnlm {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

__device__ __forceinline__ float logit(const void *p, long long i, bool bf16) {
    return bf16 ? bf16_to_f32(static_cast<const uint16_t *>(p)[i]) : static_cast<const float *>(p)[i];
}
// e^(x / T), per = log2(e) / T in two floats: what rounding the exponent's argument loses goes into a first-order term, so that shares
// of any size are good to some 2^-22 of themselves.
struct Exponent {
    float per, rest;
    __device__ explicit Exponent(float T) {
        const double c = 1.4426950408889634 / (double)T;
        per = (float)c;
        rest = (float)(c - (double)per);
    }
    __device__ __forceinline__ float fine(float x) const {
        const float y = x * per;
        return y > -INFINITY ? fast_exp2(y) * (1.f + kLn2 * (__builtin_fmaf(x, per, -y) + x * rest)) : 0.f;
    }
};
__device__ __forceinline__ float block_sum(float v, float *part) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int w = 0; w < kWaves; ++w) v += part[w];
    return v;
}
__device__ __forceinline__ float block_max(float v, float *part) {
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = -INFINITY;
    for (int w = 0; w < kWaves; ++w) v = fmaxf(v, part[w]);
    return v;
}

// The plain form: a workgroup per row, three passes over it.
__global__ __launch_bounds__(kThreads) void distill_plain_kernel(DistillArgs a, bool forward) {
    __shared__ float part[kWaves];
    const int tid = threadIdx.x;
    for (int n = blockIdx.x; n < a.N; n += gridDim.x) {
        const long long base = n * a.ld;
        const int32_t *tw = a.teacher_word + (long long)n * a.K;
        const float *tl = a.teacher_logit + (long long)n * a.K;
        const Exponent exponent(a.T);
        const float per = exponent.per;
        const int label = a.label ? a.label[n] : -1;
        // teacher
        float t_top = -INFINITY;
        bool bad = label < -1 || label >= a.V;
        for (int k = tid; k < a.K; k += kThreads) {
            const float t = tl[k];
            if (tw[k] == -1) continue;
            bad |= tw[k] < -1 || tw[k] >= a.V || t != t || t == INFINITY;
            t_top = fmaxf(t_top, t);
        }
        t_top = block_max(t_top, part);
        bad = __syncthreads_or(bad);
        const bool soft = t_top > -INFINITY, hard = label >= 0;
        float t_sum = 0.f;
        if (soft)
            for (int k = tid; k < a.K; k += kThreads)
                if (tw[k] >= 0) t_sum += exponent.fine(tl[k] - t_top);
        t_sum = block_sum(t_sum, part);
        const float lq = logf(t_sum);
        float top, inv_T, inv_1;
        if (forward) {
            top = -INFINITY;
            bool nan = false;
            for (int i = tid; i < a.V; i += kThreads) {
                const float z = logit(a.logits, base + i, a.bf16);
                nan |= z != z;
                top = fmaxf(top, z);
            }
            top = block_max(top, part);
            if (__syncthreads_or(nan)) top = quiet_nan();
            float s_T = 0.f, s_1 = 0.f;
            for (int i = tid; i < a.V; i += kThreads) {
                const float d = logit(a.logits, base + i, a.bf16) - top;
                s_T += fast_exp2(d * per);
                s_1 += fast_exp2(d * kLog2e);
            }
            s_T = block_sum(s_T, part);
            s_1 = block_sum(s_1, part);
            const bool dead = !(s_T > 0.f) || top == INFINITY;               // NaN in it, or nothing finite
            inv_T = dead ? quiet_nan() : 1.f / s_T;
            inv_1 = dead ? quiet_nan() : 1.f / s_1;
            float l = 0.f;
            if (!bad && soft)
                for (int k = tid; k < a.K; k += kThreads)
                    if (tw[k] >= 0) {
                        const float log_q = (tl[k] - t_top) / a.T - lq, q = exponent.fine(tl[k] - t_top) / t_sum;
                        if (q > 0.f) l += q * (log_q - (logit(a.logits, base + tw[k], a.bf16) - top) / a.T + logf(s_T));
                    }
            l = soft && a.a < 1.f ? block_sum(l, part) * (1.f - a.a) * a.T * a.T : 0.f;
            const bool hard_part = hard && a.a > 0.f, soft_part = soft && a.a < 1.f;
            if (!bad && hard_part) l += a.a * (logf(s_1) - (logit(a.logits, base + label, a.bf16) - top));
            if (bad || ((soft_part || hard_part) && dead)) l = quiet_nan();
            if (tid == 0) {
                a.loss[n] = l;
                a.stats[4 * n] = top; a.stats[4 * n + 1] = inv_T; a.stats[4 * n + 2] = inv_1; a.stats[4 * n + 3] = 0.f;
            }
        } else {
            top = a.stats[4 * n]; inv_T = a.stats[4 * n + 1]; inv_1 = a.stats[4 * n + 2];
        }
        if (!a.grad) continue;
        const float g = a.row_weight ? a.row_weight[n] : 1.f;
        const float c_T = soft && a.a < 1.f ? g * (1.f - a.a) * a.T : 0.f, c_1 = hard && a.a > 0.f ? g * a.a : 0.f;
        for (int i = tid; i < a.V; i += kThreads) {
            const float d = logit(a.logits, base + i, a.bf16) - top;
            float r = bad || ((c_T != 0.f || c_1 != 0.f) && inv_T != inv_T) ? quiet_nan() : 0.f;
            if (c_T != 0.f) r += c_T * fast_exp2(d * per) * inv_T;
            if (c_1 != 0.f) r += c_1 * fast_exp2(d * kLog2e) * inv_1;
            if (c_T != 0.f)
                for (int k = 0; k < a.K; ++k)
                    if (tw[k] == i) r -= c_T * exponent.fine(tl[k] - t_top) / t_sum;
            if (i == label) r -= c_1;
            if (a.bf16) static_cast<uint16_t *>(a.grad)[n * a.grad_ld + i] = (uint16_t)pack_bf16x2(r, 0.f);
            else static_cast<float *>(a.grad)[n * a.grad_ld + i] = r;
        }
    }
}

}  // namespace

size_t distill_workspace_bytes(int N, int V) { return 256; }

hipError_t launch_distill(const DistillArgs &a, hipStream_t stream) {
    distill_plain_kernel<<<a.N < 65535 ? a.N : 65535, kThreads, 0, stream>>>(a, true);
    return hipGetLastError();
}
hipError_t launch_distill_backward(const DistillArgs &a, hipStream_t stream) {
    distill_plain_kernel<<<a.N < 65535 ? a.N : 65535, kThreads, 0, stream>>>(a, false);
    return hipGetLastError();
}

}  // namespace rnnlm
