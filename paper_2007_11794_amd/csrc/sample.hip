// The next word of every row of logits by a given uniform number, with temperature, top-k, top-p and min-p.
//
// Words in the order of falling logits, equal ones by rising id, make every limit a prefix: top-k a count, top-p a weight, min-p a
// least weight.  A prefix is a key (the logit's order-preserving bits) and how many words of that very key belong to it.  Weights are
// integers, so that sums do not depend on their order.
#include "device_utils.h"
#include "ops.h"

namespace rnnlm {

namespace {

constexpr int kThreads = 1024;
typedef unsigned long long u64;

__device__ __forceinline__ float logit(const void *p, long long i, bool bf16) {
    const float z = bf16 ? bf16_to_f32(static_cast<const uint16_t *>(p)[i]) : static_cast<const float *>(p)[i];
    return z + 0.f;                                        // -0 is +0
}
// Rises with the number: negative numbers have all bits turned, others the sign.
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }

struct Weight {
    double top, per;       // the row's maximum; log2(e) / temperature
    double one;            // 2^fractional bits
    __device__ u64 operator()(float z) const {
        if (top == (double)INFINITY) return z == INFINITY ? (u64)one : 0;
        return (u64)rint(exp2(((double)z - top) * per) * one);
    }
};

__device__ __forceinline__ u64 wave_sum64(u64 v) {
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

// The plain form: a workgroup per row, every pass over the row in memory, eight bits of the key at a time.
__global__ __launch_bounds__(kThreads) void sample_plain_kernel(SampleArgs a, int bits) {
    __shared__ u64 hist_w[256], wave_w[16];
    __shared__ int hist_c[256];
    __shared__ float wave_f[16];
    __shared__ int wave_c[17];
    __shared__ u64 s_total, s_w;
    __shared__ long long s_c;
    __shared__ uint32_t s_prefix;
    __shared__ int s_word;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.V;
    for (int n = blockIdx.x; n < a.N; n += gridDim.x) {
        const long long base = n * a.ld;
        const float T = a.temperature ? a.temperature[n] : 1.f, p = a.top_p ? a.top_p[n] : 1.f, mp = a.min_p ? a.min_p[n] : 0.f, u = a.u[n];
        const int k = a.top_k ? a.top_k[n] : 0;
        float top = -INFINITY;
        bool nan = false;
        for (int i = tid; i < V; i += kThreads) {
            const float z = logit(a.logits, base + i, a.bf16);
            nan |= z != z;
            top = fmaxf(top, z);
        }
        top = wave_max(top);
        const bool bad_row = __syncthreads_or(nan);
        if (lane == 0) wave_f[wave] = top;
        __syncthreads();
        for (int w = 0; w < 16; ++w) top = fmaxf(top, wave_f[w]);
        const bool bad = bad_row || top == -INFINITY || !(T >= 0.f) || T == INFINITY || !(u >= 0.f && u < 1.f) || p != p || mp != mp;
        Weight weight{(double)top, T > 0.f ? 1.4426950408889634 / (double)T : 0.0, ldexp(1.0, bits)};
        // A prefix: words of a key above t, and the first m of key t (V: all of them).
        uint32_t t = 0;
        long long m = V;
        u64 total = 0;
        // The shortest prefix of the present one with `count` words (by_weight false) or a weight of `count` at least.
        auto cut = [&](bool by_weight, u64 want) {
            uint32_t prefix = 0;
            for (int shift = 24; shift >= 0; shift -= 8) {
                __syncthreads();
                if (tid < 256) { hist_w[tid] = 0; hist_c[tid] = 0; }
                __syncthreads();
                for (int i = tid; i < V; i += kThreads) {
                    const float z = logit(a.logits, base + i, a.bf16);
                    const uint32_t key = key_of(z);
                    if (shift < 24 && (key >> (shift + 8)) != prefix) continue;
                    if (key < t) continue;
                    atomicAdd(&hist_c[(key >> shift) & 255], 1);
                    if (by_weight) atomicAdd(&hist_w[(key >> shift) & 255], weight(z));
                }
                __syncthreads();
                if (tid == 0) {
                    int b = 255;
                    for (; b > 0; --b) {
                        const uint32_t lowest = ((prefix << 8 | (uint32_t)b) << shift);
                        u64 have = by_weight ? hist_w[b] : (u64)hist_c[b];
                        // the last key of the present prefix counts no more than m words
                        if (by_weight && shift == 0 && lowest == t && hist_c[b] > m) have = (u64)m * weight(of_key(t));
                        if (have >= want) break;
                        want -= have;
                    }
                    s_prefix = prefix << 8 | (uint32_t)b;
                    s_w = want;
                }
                __syncthreads();
                prefix = s_prefix;
                want = s_w;
            }
            const bool same = prefix == t;
            t = prefix;
            const u64 w = by_weight ? weight(of_key(t)) : 1;
            u64 many = w ? (want + w - 1) / w : (u64)V;
            if (many < 1) many = 1;
            if (same && (u64)m < many) many = (u64)m;
            m = (long long)many;
        };
        const u64 least = mp > 0.f ? (u64)ceil((double)fminf(mp, 1.f) * weight.one) : 0;
        // tie ranks: words of key t are numbered by id
        auto sum_kept = [&](bool find, u64 target, u64 floor_w) {
            __syncthreads();
            if (tid == 0) { s_total = 0; s_c = 0; s_word = -1; }
            __syncthreads();
            for (int i0 = 0; i0 < V; i0 += kThreads) {
                const int i = i0 + tid;
                const float z = i < V ? logit(a.logits, base + i, a.bf16) : -INFINITY;
                const uint32_t key = key_of(z);
                const bool tie = i < V && key == t;
                const u64 ties = __ballot(tie);
                if (lane == 0) wave_c[wave] = __popcll(ties);
                __syncthreads();
                long long rank = s_c + __popcll(ties & ((1ull << lane) - 1));
                int all = 0;
                for (int w = 0; w < 16; ++w) { if (w < wave) rank += wave_c[w]; all += wave_c[w]; }
                u64 w = 0;
                if (i < V && (key > t || (tie && rank < m))) { w = weight(z); if (w < floor_w) w = 0; }
                const u64 ws = wave_sum64(w);
                if (lane == 0) wave_w[wave] = ws;
                __syncthreads();
                u64 before = s_total, sum = 0;
                for (int q = 0; q < 16; ++q) { if (q < wave) before += wave_w[q]; sum += wave_w[q]; }
                if (find && before <= target && before + ws > target) {      // this wave has it
                    u64 upto = w;
#pragma unroll
                    for (int s = 1; s < 64; s <<= 1) { const u64 o = __shfl_up(upto, s); if (lane >= s) upto += o; }
                    const u64 hit = __ballot(before + upto > target);
                    if (lane == __ffsll((long long)hit) - 1) { s_word = i; s_w = w; }
                }
                __syncthreads();
                if (tid == 0) { s_total += sum; s_c += all; }
                __syncthreads();
                if (find && s_word >= 0) break;
            }
            total = s_total;
            __syncthreads();
        };
        if (bad) {
            if (tid == 0) { a.word[n] = -1; if (a.logprob) a.logprob[n] = quiet_nan(); }
            continue;
        }
        if (T == 0.f) {
            t = key_of(top); m = 1;
            weight.per = 0.0;
            weight.top = INFINITY;                        // every word kept weighs the same
            weight.one = 1.0;
            __syncthreads();
            if (tid == 0) s_word = 0x7FFFFFFF;
            __syncthreads();
            for (int i = tid; i < V; i += kThreads)
                if (logit(a.logits, base + i, a.bf16) == top) atomicMin(&s_word, i);
            __syncthreads();
            if (tid == 0) { a.word[n] = s_word; if (a.logprob) a.logprob[n] = 0.f; }
            __syncthreads();
            continue;
        }
        if (k > 0 && k < V) cut(false, (u64)k);
        if (p < 1.f) {
            sum_kept(false, 0, 0);
            const u64 want = p > 0.f ? (u64)ceil((double)p * (double)total) : 1;
            cut(true, want > 0 ? want : 1);
        }
        sum_kept(false, 0, least);
        const u64 whole = total;
        sum_kept(true, (u64)floor((double)u * (double)whole), least);
        if (tid == 0) {
            a.word[n] = s_word;
            if (a.logprob) a.logprob[n] = (float)log((double)s_w / (double)whole);
        }
        __syncthreads();
    }
}

}  // namespace

size_t sample_workspace_bytes(int N, int V) { return 256; }

hipError_t launch_sample(const SampleArgs &a, hipStream_t stream) {
    int bits = 62;
    for (long long v = 1; v < a.V; v <<= 1) --bits;
    sample_plain_kernel<<<a.N < 65535 ? a.N : 65535, kThreads, 0, stream>>>(a, bits);
    return hipGetLastError();
}

}  // namespace rnnlm
