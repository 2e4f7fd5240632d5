// Products with 4-bit weights: y[b][v] = bias[v] + sum_g scale[g][v] sum_{j in g} (code[v][j] - zero[g][v]) x[b][j].
#include "device_utils.h"
#include "ops.h"

namespace rnnlm {

namespace {

__device__ __forceinline__ float element(const void *p, long long i, bool bf16) {
    return bf16 ? bf16_to_f32(static_cast<const uint16_t *>(p)[i]) : static_cast<const float *>(p)[i];
}

// One wave per word and row: the plain form.
__global__ __launch_bounds__(256) void q4_plain_kernel(Q4Args a) {
    const int v = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (v >= a.V) return;
    for (int b = blockIdx.y; b < a.B; b += gridDim.y) {
        float sum = 0.f;
        for (int j = lane; j < a.H; j += 64) {
            const int g = j / a.group;
            const int c = (a.codes[v * a.code_ld + j / 2] >> (4 * (j & 1))) & 15, z = a.zero ? a.zero[(long long)g * a.V + v] : 8;
            sum += element(a.scale, (long long)g * a.V + v, a.scale_bf16) * (float)(c - z) * element(a.x, b * a.x_ld + j, a.x_bf16);
        }
        sum = wave_sum(sum) + (a.bias ? a.bias[v] : 0.f);
        if (lane == 0) {
            if (a.y_bf16) static_cast<uint16_t *>(a.y)[b * a.y_ld + v] = (uint16_t)pack_bf16x2(sum, 0.f);
            else static_cast<float *>(a.y)[b * a.y_ld + v] = sum;
        }
    }
}

}  // namespace

hipError_t launch_q4(const Q4Args &a, hipStream_t stream) {
    q4_plain_kernel<<<dim3((a.V + 3) / 4, a.B < 65535 ? a.B : 65535), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace rnnlm
