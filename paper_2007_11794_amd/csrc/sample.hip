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

// 2^y for y <= 0 as a whole number of 2^-bits, to nearest (bits <= 50; anything below -200 is nothing).  2^f on [-1/2, 1/2] is 1 + f times a
// polynomial fitted for the least relative error, 1.5e-14; the product with 2^bits is rounded by adding 2^52, below which its last bit counts 1.
__device__ __forceinline__ u64 fixed_exp2(double y, int bits) {
    y = fmax(y, -200.0);
    const double n = rint(y), f = y - n;
    double q = 0x1.b3de2c7e1dde3p-24;
    q = fma(q, f, 0x1.63e69680bde3cp-20);
    q = fma(q, f, 0x1.ffce2fc63d69ep-17);
    q = fma(q, f, 0x1.430897f31267cp-13);
    q = fma(q, f, 0x1.5d87fd9386691p-10);
    q = fma(q, f, 0x1.3b2ab72412393p-7);
    q = fma(q, f, 0x1.c6b08d70c8822p-5);
    q = fma(q, f, 0x1.ebfbdff81be04p-3);
    q = fma(q, f, 0x1.62e42fefa37d1p-1);
    q = fma(q, f, 1.0);
    return (u64)__double_as_longlong(ldexp(q, (int)n + bits) + 0x1p52) - 0x4330000000000000ull;
}

struct Weight {
    double top, per;       // the row's maximum; log2(e) / temperature
    int bits;
    __device__ u64 operator()(float z) const {
        if (top == (double)INFINITY) return z == INFINITY ? 1ull << bits : 0;
        return fixed_exp2(((double)z - top) * per, bits);
    }
    __device__ u64 one() const { return 1ull << bits; }
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
        const Weight weight{(double)top, T > 0.f ? 1.4426950408889634 / (double)T : 0.0, bits};
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
        const u64 least = mp > 0.f ? (u64)ceil((double)fminf(mp, 1.f) * (double)weight.one()) : 0;
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


// ---- A row in the registers of one workgroup

constexpr int kBins = 2048;                  // of the distance to the row's maximum, kBins / 64 to a factor of two in weight
constexpr int kList = 2048;                  // words that can be sorted
constexpr float kBinsPerOctave = kBins / 64;

typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef uint32_t u32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x32 __attribute__((ext_vector_type(32)));
// R vectors of 16 bytes that a loop reads by a counter: code that runs once for a row and is written out for every one of its vectors is not
// executed but fetched (a third of a megabyte of it took 345 us where this takes a tenth).
template <int R> struct Vectors;
template <> struct Vectors<4> {
    u32x16 x;
    __device__ __forceinline__ u32x4 get(int r) const { return u32x4{x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]}; }
    __device__ __forceinline__ void set(int r, u32x4 v) {
#pragma unroll
        for (int q = 0; q < 4; ++q) x[4 * r + q] = v[q];
    }
    // f(r, vector) for r below `used`
    template <typename F> __device__ __forceinline__ void each(int used, F f) const {
#pragma unroll 1
        for (int r = 0; r < 4 && r < used; ++r) f(r, get(r));
    }
};
template <> struct Vectors<16> {
    u32x32 x, y;
    __device__ __forceinline__ void set(int r, u32x4 v) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (r < 8) x[4 * r + q] = v[q];
            else y[4 * (r - 8) + q] = v[q];
        }
    }
    template <typename F> __device__ __forceinline__ void each(int used, F f) const {
#pragma unroll 1
        for (int r = 0; r < 8 && r < used; ++r) f(r, u32x4{x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]});
#pragma unroll 1
        for (int r = 8; r < 16 && r < used; ++r) f(r, u32x4{y[4 * r - 32], y[4 * r - 31], y[4 * r - 30], y[4 * r - 29]});
    }
};

template <typename Z> struct RowOf;
template <> struct RowOf<float> {
    static constexpr int E = 4;
    static constexpr uint32_t kNothing = 0xFF800000u;
    static __device__ __forceinline__ float get(u32x4 v, int i) { return __uint_as_float(v[i]); }
    static __device__ __forceinline__ float one(const float *p) { return *p; }
    static __device__ __forceinline__ uint32_t pack(const float (&z)[4], int i) { return __float_as_uint(z[i]); }
};
template <> struct RowOf<uint16_t> {
    static constexpr int E = 8;
    static constexpr uint32_t kNothing = 0xFF80FF80u;
    static __device__ __forceinline__ float get(u32x4 v, int i) { return __uint_as_float(i & 1 ? v[i >> 1] & 0xFFFF0000u : v[i >> 1] << 16); }
    static __device__ __forceinline__ float one(const uint16_t *p) { return bf16_to_f32(*p); }
    static __device__ __forceinline__ uint32_t pack(const float (&z)[8], int i) { return __float_as_uint(z[2 * i]) >> 16 | (__float_as_uint(z[2 * i + 1]) & 0xFFFF0000u); }   // (bfloat16 values)
};

__device__ __forceinline__ u64 wave_scan64(u64 v, int lane) {                // inclusive
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) { const u64 o = __shfl_up(v, s); if (lane >= s) v += o; }
    return v;
}
// Order of the words: larger logits first, equal ones by rising id.
__device__ __forceinline__ u64 place(float z, uint32_t id) { return (u64)key_of(z + 0.f) << 32 | (uint32_t)~id; }
__device__ __forceinline__ float logit_of(u64 place) { return of_key((uint32_t)(place >> 32)); }

struct Shared {
    u64 weight[kBins];                       // histogram; weights of the listed words
    u64 list[kList];
    int count[kBins];
    u64 wave64[16];
    float wavef[16];
    u64 want, total, found_w, border;
    int bin, n, word, m;
};

template <int THREADS>
__device__ __forceinline__ u64 block_scan64(u64 v, Shared &sh, u64 &total) {  // inclusive over the threads
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v = wave_scan64(v, lane);
    __syncthreads();
    if (lane == 63) sh.wave64[wave] = v;
    __syncthreads();
    u64 before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const u64 x = sh.wave64[w];
        if (w < wave) before += x;
        all += x;
    }
    total = all;
    return v + before;
}

// list[0 .. n) in falling (or rising) order, padded to a power of two with what comes last.  Exchanges over up to 64 places stay in one
// wave's 128 and need no barrier.
template <int THREADS, bool FALLING>
__device__ __forceinline__ void sort_list(u64 *list, int n) {
    int P = 2;
    while (P < n) P <<= 1;
    for (int i = n + threadIdx.x; i < P; i += THREADS) list[i] = FALLING ? 0 : ~0ull;
    __syncthreads();
    for (int size = 2; size <= P; size <<= 1)
        for (int stride = size >> 1; stride; stride >>= 1) {
            for (int i = threadIdx.x; i < P / 2; i += THREADS) {
                const int a = 2 * i - (i & (stride - 1)), b = a + stride;
                const u64 x = list[a], y = list[b];
                const bool falls = ((a & size) == 0) == FALLING;
                if (falls ? x < y : x > y) { list[a] = y; list[b] = x; }
            }
            if (stride > 64 || (stride == 1 && size >= 128)) __syncthreads();
            else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        }
    __syncthreads();
}

// The limits and the draw on n listed words, among them all that can be kept: top_k of them (all: n), then top-p, min-p, and the draw in the
// order of the ids.
template <int THREADS>
__device__ __forceinline__ void draw_from_list(Shared &sh, int n, int top_k, float p, u64 least, float u, const Weight &weight) {
    constexpr int M = kList / THREADS;
    const int tid = threadIdx.x;
    if (top_k > n) top_k = n;
    sort_list<THREADS, true>(sh.list, n);
    u64 w[M], sum = 0, total;
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const int at = tid * M + i;
        w[i] = at < top_k ? weight(logit_of(sh.list[at])) : 0;
        sum += w[i];
    }
    if (tid == 0) { sh.m = top_k; sh.n = top_k; }
    u64 upto = block_scan64<THREADS>(sum, sh, total) - sum;
    u64 want = p > 0.f ? (u64)ceil((double)p * (double)total) : 1;
    if (want < 1) want = 1;
    u64 keep[M];
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const int at = tid * M + i;
        const u64 before = upto;
        upto += w[i];
        if (at < top_k) {
            if (p < 1.f && before < want && upto >= want) sh.m = at + 1;
            if (w[i] < least) atomicMin(&sh.n, at);
            sh.weight[at] = w[i];
        }
        keep[i] = at < top_k ? (u64)(uint32_t)~(uint32_t)sh.list[at] << 32 | (uint32_t)at : 0;
    }
    __syncthreads();
    const int m = min(sh.m, sh.n);
#pragma unroll
    for (int i = 0; i < M; ++i)
        if (tid * M + i < m) sh.list[tid * M + i] = keep[i];
    __syncthreads();
    sort_list<THREADS, false>(sh.list, m);
    sum = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const int at = tid * M + i;
        w[i] = at < m ? sh.weight[(uint32_t)sh.list[at]] : 0;
        sum += w[i];
    }
    upto = block_scan64<THREADS>(sum, sh, total) - sum;
    const u64 target = (u64)floor((double)u * (double)total);
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const u64 before = upto;
        upto += w[i];
        if (before <= target && target < upto) { sh.word = (int)(sh.list[tid * M + i] >> 32); sh.found_w = w[i]; sh.total = total; }
    }
    __syncthreads();
}

template <typename Z, int THREADS, int R>
__global__ __launch_bounds__(THREADS, 4) void sample_row_kernel(SampleArgs a, int bits) {
    typedef RowOf<Z> O;
    constexpr int E = O::E, WAVES = THREADS / 64, kPerThread = kBins / THREADS;
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = blockIdx.x, V = a.V;
    const Z *row = static_cast<const Z *>(a.logits) + n * a.ld;
    const float T = a.temperature ? a.temperature[n] : 1.f, p = a.top_p ? a.top_p[n] : 1.f, mp = a.min_p ? a.min_p[n] : 0.f, u = a.u[n];
    const int k = a.top_k ? a.top_k[n] : 0;
    // a wave's vectors lie behind each other: vector (wave * used + r) * 64 + lane, so that words rise with wave, r, lane, element
    const int vectors = (V + E - 1) / E, used = (vectors + 64 * WAVES - 1) / (64 * WAVES), first = wave * used * 64 + lane;
    u32x4 loaded[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        loaded[r] = u32x4{O::kNothing, O::kNothing, O::kNothing, O::kNothing};
        const int i = first + r * 64;
        if (r < used && (i + 1) * E <= V) loaded[r] = *reinterpret_cast<const u32x4_any *>(reinterpret_cast<const char *>(row) + (uint32_t)i * 16u);
    }
    if (V % E) {                                              // the last vector, element by element
        const int r_last = (vectors - 1 - first) / 64;
        if (vectors - 1 == first + r_last * 64 && r_last < used && vectors - 1 >= first) {
            float z[E];
#pragma unroll
            for (int j = 0; j < E; ++j) z[j] = (vectors - 1) * E + j < V ? O::one(row + (vectors - 1) * E + j) : -INFINITY;
            u32x4 x;
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = O::pack(z, q);
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r == r_last) loaded[r] = x;
        }
    }
    Vectors<R> v;
#pragma unroll
    for (int r = 0; r < R; ++r) v.set(r, loaded[r]);
    bool alike = false;                                       // +infinity is 0 from here on, all else -infinity
    auto each_vector = [&](auto f) {                          // f(r, vector)
        v.each(used, [&](int r, u32x4 x) {
            if (alike) {
                float z[E];
#pragma unroll
                for (int j = 0; j < E; ++j) z[j] = O::get(x, j) == INFINITY ? 0.f : -INFINITY;
#pragma unroll
                for (int q = 0; q < 4; ++q) x[q] = O::pack(z, q);
            }
            f(r, x);
        });
    };
    auto each = [&](auto f) {                                 // f(logit, id), ids of a thread rising
        each_vector([&](int r, u32x4 x) {
#pragma unroll
            for (int j = 0; j < E; ++j) f(O::get(x, j), (uint32_t)((first + r * 64) * E + j));
        });
    };
    for (int i = tid; i < kBins; i += THREADS) { sh.count[i] = 0; sh.weight[i] = 0; }
    if (tid == 0) sh.n = 0;
    float mine = -INFINITY;
    bool nan = false;
    each([&](float z, uint32_t) { mine = fmaxf(mine, z); nan |= z != z; });
    float top = wave_max(mine);
    if (lane == 0) sh.wavef[wave] = top;
    const bool bad = __syncthreads_or(nan || !(T >= 0.f) || T == INFINITY || !(u >= 0.f && u < 1.f) || p != p || mp != mp);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, sh.wavef[w]);
    if (bad || top == -INFINITY) {
        if (tid == 0) { a.word[n] = -1; if (a.logprob) a.logprob[n] = quiet_nan(); }
        return;
    }
    if (T == 0.f) {
        if (tid == 0) sh.word = 0x7FFFFFFF;
        __syncthreads();
        uint32_t at = 0x7FFFFFFF;
        if (mine == top) each([&](float z, uint32_t id) { if (z == top && id < at) at = id; });
        if (at != 0x7FFFFFFF) atomicMin(&sh.word, (int)at);
        __syncthreads();
        if (tid == 0) { a.word[n] = sh.word; if (a.logprob) a.logprob[n] = 0.f; }
        return;
    }
    if (top == INFINITY) {                                    // those words alone, alike
        alike = true;
        mine = mine == INFINITY ? 0.f : -INFINITY;
        top = 0.f;
    }
    const Weight weight{(double)top, 1.4426950408889634 / (double)T, bits};
    const float bin_scale = fminf((float)(weight.per * kBinsPerOctave), 3.4e38f);
    auto bin_of = [&](float z) {                              // rises as z falls; what is in the last one weighs nothing
        const float x = (top - z) * bin_scale;
        return x < (float)(kBins - 1) ? (int)x : kBins - 1;
    };
    const u64 least = mp > 0.f ? (u64)ceil((double)fminf(mp, 1.f) * (double)weight.one()) : 0;
    // Appends words to the list; beyond kList they are only counted.
    auto append = [&](bool take, float z, uint32_t id) {
        const u64 who = __ballot(take);
        if (who == 0) return;
        int at = 0;
        if (lane == 0) at = atomicAdd(&sh.n, __popcll(who));
        at = __builtin_amdgcn_readfirstlane(at) + __popcll(who & ((1ull << lane) - 1));
        if (take && at < kList) sh.list[at] = place(z, id);
    };
    // The bin where `want` of the histogram (counts, or weights) is reached from the front, and what is still wanted of that bin.
    auto find_bin = [&](bool by_weight, u64 want) {
        u64 h[kPerThread], sum = 0, total;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            h[i] = by_weight ? sh.weight[tid * kPerThread + i] : (u64)sh.count[tid * kPerThread + i];
            sum += h[i];
        }
        if (tid == 0) sh.bin = kBins - 1;
        u64 upto = block_scan64<THREADS>(sum, sh, total) - sum;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            if (upto < want && upto + h[i] >= want) { sh.bin = tid * kPerThread + i; sh.want = want - upto; }
            upto += h[i];
        }
        __syncthreads();
    };
    auto finish = [&](int word, u64 w, u64 total) {
        if (tid == 0) { a.word[n] = word; if (a.logprob) a.logprob[n] = (float)log((double)w / (double)total); }
    };

    const bool few = k > 0 && k < V;
    // Few words, or few of them kept: all that can be kept fit the list.  The top_k-th largest of the threads' own maxima is no more than the
    // top_k-th largest logit, so whatever lies in its bin or in front of it is enough.
    if (V <= kList || (few && k <= THREADS / 2)) {
        int edge = kBins - 1;
        if (V > kList) {
            if (mine > -INFINITY) atomicAdd(&sh.count[bin_of(mine)], 1);
            __syncthreads();
            find_bin(false, (u64)k);
            edge = sh.bin;
        }
        if (V <= kList || edge < kBins - 1) {
            if (V <= kList) each([&](float z, uint32_t id) { append(z > -INFINITY, z, id); });
            else {
                // floats in front of the bin's far edge; the edge itself is checked by the bin
                each([&](float z, uint32_t id) { append((top - z) * bin_scale < (float)(edge + 1), z, id); });
            }
            __syncthreads();
            const int listed = sh.n;
            if (listed <= kList) {
                __syncthreads();
                draw_from_list<THREADS>(sh, listed, few ? k : listed, p, least, u, weight);
                finish(sh.word, sh.found_w, sh.total);
                return;
            }
        }
        __syncthreads();
        for (int i = tid; i < kBins; i += THREADS) sh.count[i] = 0;
        __syncthreads();
    }

    // All words: limits as the place of the last word kept.
    u64 border = 0;
    auto kept = [&](float z, uint32_t id) { return place(z, id) >= border; };
    // The shortest prefix that reaches `want` words or weight (of the histogram that is there, by distance): the new border.
    auto cut = [&](bool by_weight, u64 want) {
        find_bin(by_weight, want);
        const int bin = sh.bin;
        if (bin == kBins - 1) return;                         // beyond it nothing has a weight
        want = sh.want;
        uint32_t low = 0, high = 0xFFFFFFFFu, id_low = 0, id_high = 0xFFFFFFFFu;      // of the keys, and of the ids where only one key is left
        auto inside = [&](float z, uint32_t id) {
            const uint32_t key = key_of(z + 0.f);
            return bin_of(z) == bin && key >= low && key <= high && id >= id_low && id <= id_high && kept(z, id);
        };
        while (true) {
            __syncthreads();
            if (tid == 0) sh.n = 0;
            __syncthreads();
            each([&](float z, uint32_t id) { append(inside(z, id), z, id); });
            __syncthreads();
            const int listed = sh.n;
            if (listed <= kList) {
                __syncthreads();
                sort_list<THREADS, true>(sh.list, listed);
                constexpr int M = kList / THREADS;
                u64 w[M], sum = 0, total;
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    const int at = tid * M + i;
                    w[i] = at < listed ? by_weight ? weight(logit_of(sh.list[at])) : 1 : 0;
                    sum += w[i];
                }
                if (tid == 0) sh.border = listed ? sh.list[listed - 1] : border;
                u64 upto = block_scan64<THREADS>(sum, sh, total) - sum;
#pragma unroll
                for (int i = 0; i < M; ++i) {
                    if (upto < want && upto + w[i] >= want) sh.border = sh.list[tid * M + i];
                    upto += w[i];
                }
                __syncthreads();
                border = sh.border;
                return;
            }
            // More words than can be sorted, most of them alike: a histogram over what tells them apart, keys first, then ids.
            for (int i = tid; i < kBins; i += THREADS) { sh.count[i] = 0; sh.weight[i] = 0; }
            __syncthreads();
            const bool by_key = low < high;
            const uint32_t span = by_key ? high - low : min(id_high, (uint32_t)vectors * E - 1) - id_low;
            int shift = 0;
            while (span >> shift >= (uint32_t)kBins) ++shift;
            each([&](float z, uint32_t id) {
                if (!inside(z, id)) return;
                const int at = by_key ? (int)((high - key_of(z + 0.f)) >> shift) : (int)((id - id_low) >> shift);
                if (by_weight) atomicAdd(&sh.weight[at], weight(z));
                else atomicAdd(&sh.count[at], 1);
            });
            __syncthreads();
            find_bin(by_weight, want);
            const uint32_t at = (uint32_t)sh.bin << shift, more = (1u << shift) - 1;
            want = sh.want;
            if (by_key) {
                high -= at;
                low = high - low > more ? high - more : low;
            } else {
                id_low += at;
                id_high = min(id_high, id_low + more);
            }
        }
    };
    if (few) {
        each([&](float z, uint32_t id) { if (z > -INFINITY) atomicAdd(&sh.count[bin_of(z)], 1); });
        __syncthreads();
        cut(false, (u64)k);
        __syncthreads();
        for (int i = tid; i < kBins; i += THREADS) sh.weight[i] = 0;
        __syncthreads();
    }
    if (p < 1.f) {
        u64 sum = 0, total;
        each([&](float z, uint32_t id) {
            if (!kept(z, id)) return;
            const u64 w = weight(z);
            if (w == 0) return;
            sum += w;
            atomicAdd(&sh.weight[bin_of(z)], w);
        });
        block_scan64<THREADS>(sum, sh, total);
        const u64 want = p > 0.f ? (u64)ceil((double)p * (double)total) : 1;
        cut(true, want > 0 ? want : 1);
    }
    // The draw: sums of waves, of its vectors for the wave that has it, of its lanes, of the lane's words.
    u64 sum = 0, total;
    each([&](float z, uint32_t id) {
        if (!kept(z, id)) return;
        const u64 w = weight(z);
        sum += w >= least ? w : 0;
    });
    const u64 upto_thread = block_scan64<THREADS>(sum, sh, total);
    const u64 upto_wave = __shfl(upto_thread, 63), in_wave = wave_sum64(sum);
    const u64 target = (u64)floor((double)u * (double)total);
    u64 before = upto_wave - in_wave;
    if (before <= target && target < upto_wave) {
        bool done = false;
        each_vector([&](int r, u32x4 x) {
            if (done) return;
            u64 w[E], s = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float z = O::get(x, j);
                w[j] = kept(z, (uint32_t)((first + r * 64) * E + j)) ? weight(z) : 0;
                if (w[j] < least) w[j] = 0;
                s += w[j];
            }
            const u64 upto = before + wave_scan64(s, lane), all = __shfl(upto, 63);
            if (all > target) {
                u64 at = upto - s;
                if (at <= target && target < upto) {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        if (at <= target && target < at + w[j]) { sh.word = (first + r * 64) * E + j; sh.found_w = w[j]; }
                        at += w[j];
                    }
                }
                done = true;
            }
            before = all;
        });
    }
    __syncthreads();
    finish(sh.word, sh.found_w, total);
}

}  // namespace

size_t sample_workspace_bytes(int N, int V) { return 256; }

namespace {
template <typename Z>
hipError_t launch_rows(const SampleArgs &a, int bits, hipStream_t stream) {
    const int vectors = (a.V + RowOf<Z>::E - 1) / RowOf<Z>::E;
    if (vectors <= 256 * 4) sample_row_kernel<Z, 256, 4><<<a.N, 256, 0, stream>>>(a, bits);
    else if (vectors <= 1024 * 4) sample_row_kernel<Z, 1024, 4><<<a.N, 1024, 0, stream>>>(a, bits);
    else if (vectors <= 1024 * 16) sample_row_kernel<Z, 1024, 16><<<a.N, 1024, 0, stream>>>(a, bits);
    else sample_plain_kernel<<<a.N < 65535 ? a.N : 65535, kThreads, 0, stream>>>(a, bits);
    return hipGetLastError();
}
}  // namespace

hipError_t launch_sample(const SampleArgs &a, hipStream_t stream) {
    int bits = 62;                                            // sums of V weights stay below 2^62
    for (long long v = 1; v < a.V; v <<= 1) --bits;
    if (bits > 50) bits = 50;
    return a.bf16 ? launch_rows<uint16_t>(a, bits, stream) : launch_rows<float>(a, bits, stream);
}

}  // namespace rnnlm
