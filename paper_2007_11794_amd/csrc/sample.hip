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

// Values that all lanes share, in scalar registers.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ __forceinline__ float uniform(float x) { return __uint_as_float(uniform(__float_as_uint(x))); }
__device__ __forceinline__ u64 uniform(u64 x) { return (u64)uniform((uint32_t)(x >> 32)) << 32 | uniform((uint32_t)x); }
__device__ __forceinline__ double uniform(double x) { return __longlong_as_double((long long)uniform((u64)__double_as_longlong(x))); }

// a * b + c with c in scalar registers (the compiler copies it into a vector register in front of every use)
__device__ __forceinline__ double fma_with(double a, double b, double c) {
    double r;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "s"(c));
    return r;
}

// 2^y for y <= 0 as a whole number of 2^-bits, to nearest (bits <= 50; anything below -200 is nothing).  2^f on [-1/2, 1/2] is 1 + f times a
// polynomial fitted for the least relative error, 1.5e-14; the product with 2^bits is rounded by adding 2^52, below which its last bit counts 1.
__device__ __forceinline__ u64 fixed_exp2(double y, int bits) {
    y = fmax(y, -200.0);
    const double n = rint(y), f = y - n;
    double q = fma_with(0x1.b3de2c7e1dde3p-24, f, 0x1.63e69680bde3cp-20);
    q = fma_with(q, f, 0x1.ffce2fc63d69ep-17);
    q = fma_with(q, f, 0x1.430897f31267cp-13);
    q = fma_with(q, f, 0x1.5d87fd9386691p-10);
    q = fma_with(q, f, 0x1.3b2ab72412393p-7);
    q = fma_with(q, f, 0x1.c6b08d70c8822p-5);
    q = fma_with(q, f, 0x1.ebfbdff81be04p-3);
    q = fma_with(q, f, 0x1.62e42fefa37d1p-1);
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

// Bins of the distance to the row's maximum, over the kOctaves factors of two in which a weight is not nothing; words that can be listed;
// words that are put in order by comparing each with each.
constexpr int kOctaves = 52, kSmall = 256;
constexpr int bins_of(int threads) { return threads > 256 ? 4096 : 1024; }
constexpr int list_of(int threads) { return threads > 256 ? 2048 : 512; }

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

// Inclusive prefix sums over the wave in registers, as wave_inclusive_scan.
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 moved(u64 v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xF, false);
    return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 wave_scan64(u64 v) {
    v += moved<0x111, 0xF>(v);
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);
    return v + moved<0x143, 0xC>(v);
}
__device__ __forceinline__ u64 last_lane(u64 v) {
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63);
}
// Order of the words: larger logits first, equal ones by rising id.
__device__ __forceinline__ u64 place(float z, uint32_t id) { return (u64)key_of(z + 0.f) << 32 | (uint32_t)~id; }
__device__ __forceinline__ float logit_of(u64 place) { return of_key((uint32_t)(place >> 32)); }

template <int THREADS>
struct Shared {
    union {                                  // histogram
        u64 weight[bins_of(THREADS)];
        int count[bins_of(THREADS)];
    };
    u64 list[list_of(THREADS)];
    u64 small[kSmall], small_w[kSmall];
    u64 wave64[16], low64[16], high64[16];
    float wavef[16];
    u64 want, found_w, border;
    int bin, n, word;
};

// Inclusive over the threads.
template <int THREADS>
__device__ __forceinline__ u64 block_scan64(u64 v, Shared<THREADS> &sh, u64 &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    v = wave_scan64(v);
    __syncthreads();
    if (lane == 63) sh.wave64[wave] = v;
    __syncthreads();
    const u64 all = wave_scan64(lane < THREADS / 64 ? sh.wave64[lane] : 0);
    total = last_lane(all);
    const int before = __builtin_amdgcn_readfirstlane(wave) - 1;
    const uint32_t lo = before < 0 ? 0 : (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)all, before);
    const uint32_t hi = before < 0 ? 0 : (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(all >> 32), before);
    return v + ((u64)hi << 32 | lo);
}

template <typename Z, int THREADS, int R>
__global__ __launch_bounds__(THREADS, 4) void sample_row_kernel(SampleArgs a, int bits) {
    typedef RowOf<Z> O;
    constexpr int E = O::E, WAVES = THREADS / 64, kBins = bins_of(THREADS), kList = list_of(THREADS), kPerThread = kBins / THREADS;
    constexpr float kBinsPerOctave = (float)kBins / kOctaves;
    __shared__ Shared<THREADS> sh;
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
    for (int i = tid; i < kBins; i += THREADS) sh.count[i] = 0;
    if (tid == 0) sh.n = 0;
    float mine = -INFINITY;
    bool nan = false;
    each([&](float z, uint32_t) { mine = fmaxf(mine, z); nan |= z != z; });
    float top = wave_max(mine);
    if (lane == 0) sh.wavef[wave] = top;
    const bool bad = __syncthreads_or(nan || !(T >= 0.f) || T == INFINITY || !(u >= 0.f && u < 1.f) || p != p || mp != mp);
    top = uniform(wave_max(lane < WAVES ? sh.wavef[lane] : -INFINITY));
    if (bad || top == -INFINITY) {
        if (tid == 0) { a.word[n] = -1; if (a.logprob) a.logprob[n] = quiet_nan(); }
        return;
    }
    if (T == 0.f) {
        if (tid == 0) sh.word = 0x7FFFFFFF;
        __syncthreads();
        uint32_t at = 0x7FFFFFFF;
        if (__any(mine == top)) each([&](float z, uint32_t id) { at = z == top && id < at ? id : at; });
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
    const Weight weight{uniform((double)top), uniform(1.4426950408889634 / (double)T), bits};
    const float bin_scale = uniform(fminf((float)(weight.per * kBinsPerOctave), 3.4e38f));
    auto bin_of = [&](float z) {                              // rises as z falls; what is in the last one weighs nothing
        const float x = (top - z) * bin_scale;
        return x < (float)(kBins - 1) ? (int)x : kBins - 1;
    };
    const u64 least = mp > 0.f ? uniform((u64)ceil((double)fminf(mp, 1.f) * (double)weight.one())) : 0;
    // Appends words to a list, `to` of at most `most`; beyond that they are only counted.  M words of a thread at once.
    auto append = [&](auto take, auto put, int most) {
        int at = 0;
        constexpr int M = sizeof(take) / sizeof(bool);
        u64 who[M];
        int all = 0;
#pragma unroll
        for (int i = 0; i < M; ++i) { who[i] = __ballot(take.is[i]); all += __popcll(who[i]); }
        if (all == 0) return;
        if (lane == 0) at = atomicAdd(&sh.n, all);
        at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const int mine_at = at + __popcll(who[i] & ((1ull << lane) - 1));
            if (take.is[i] && mine_at < most) put(i, mine_at);
            at += __popcll(who[i]);
        }
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
        if (upto < want && upto + sum >= want) {
#pragma unroll
            for (int i = 0; i < kPerThread; ++i) {
                if (upto < want && upto + h[i] >= want) { sh.bin = tid * kPerThread + i; sh.want = want - upto; }
                upto += h[i];
            }
        }
        __syncthreads();
    };

    // Few words kept: they are listed.  The top_k-th largest of the threads' own maxima is no more than the top_k-th largest logit, so whatever
    // lies in its bin or in front of it is enough.
    const bool few = k > 0 && k < V;
    bool in_list = false;
    int listed = 0;
    if (few && k <= THREADS / 2) {
        if (mine > -INFINITY) atomicAdd(&sh.count[bin_of(mine)], 1);
        __syncthreads();
        find_bin(false, (u64)k);
        const int edge = sh.bin;
        if (edge < kBins - 1) {
            each_vector([&](int r, u32x4 x) {
                struct { bool is[E]; } take;
#pragma unroll
                for (int j = 0; j < E; ++j) take.is[j] = (top - O::get(x, j)) * bin_scale < (float)(edge + 1);
                append(take, [&](int j, int to) { sh.list[to] = place(O::get(x, j), (uint32_t)((first + r * 64) * E + j)); }, kList);
            });
            __syncthreads();
            listed = sh.n;
            in_list = listed <= kList;
        }
    }
    auto over = [&](auto f) {                                 // the listed words, or all
        if (in_list)
            for (int i = tid; i - tid < listed; i += THREADS) {
                const u64 w = i < listed ? sh.list[i] : 0;
                f(i < listed, logit_of(w), (uint32_t)~(uint32_t)w);
            }
        else each([&](float z, uint32_t id) { f(id < (uint32_t)V, z, id); });
    };

    // Limits as the place of the last word kept: top_k, top_p, and of listed words the draw as well, which is the same search in the order of
    // the ids.  Each by a histogram, the bin in which what is wanted is reached, and that bin's words.
    u64 border = 0, total = 0;
    int id_shift = 0;
    while (V >> id_shift >= kBins) ++id_shift;
#pragma unroll 1
    for (int stage = 0; stage < 3; ++stage) {
        if (stage == 0 ? !few : stage == 1 ? !(p < 1.f) : !in_list) continue;
        const bool by_weight = stage > 0, by_id = stage == 2;
        auto weigh = [&](float z) {
            const u64 w = by_weight ? weight(z) : 1;
            return by_id && w < least ? 0 : w;
        };
        auto bin_at = [&](float z, uint32_t id) { return by_id ? (int)(id >> id_shift) : bin_of(z); };
        auto order = [&](float z, uint32_t id) { return by_id ? ~(u64)id : place(z, id); };          // falls from word to word
        auto is_kept = [&](float z, uint32_t id) { return z > -INFINITY && place(z, id) >= border; };
        __syncthreads();
        for (int i = tid; i < kBins; i += THREADS) sh.weight[i] = 0;
        __syncthreads();
        u64 sum = 0;
        if (by_weight) over([&](bool is, float z, uint32_t id) {
            u64 w = weight(z);
            w = is && is_kept(z, id) && !(by_id && w < least) ? w : 0;
            sum += w;
            if (w) atomicAdd(&sh.weight[bin_at(z, id)], w);
        });
        else over([&](bool is, float z, uint32_t id) {
            if (is && is_kept(z, id)) atomicAdd(&sh.count[bin_at(z, id)], 1);
        });
        block_scan64<THREADS>(sum, sh, total);
        u64 want = (u64)k;
        if (stage == 1) { want = p > 0.f ? (u64)ceil((double)p * (double)total) : 1; if (want < 1) want = 1; }
        if (stage == 2) want = (u64)floor((double)u * (double)total) + 1;
        find_bin(by_weight, want);
        const int bin = sh.bin;
        if (bin == kBins - 1 && !by_id) continue;             // beyond it nothing has a weight
        want = sh.want;
        u64 low = 0, high = ~0ull;                            // of the orders
        // (most vectors have no word of one bin)
        auto inside = [&](bool is, float z, uint32_t id) {
            bool yes = is && bin_at(z, id) == bin;
            if (!__any(yes)) return false;
            const u64 o = order(z, id);
            return yes && is_kept(z, id) && o >= low && o <= high;
        };
        while (true) {
            __syncthreads();
            if (tid == 0) sh.n = 0;
            __syncthreads();
            u64 least_o = ~0ull, most_o = 0;
            over([&](bool is, float z, uint32_t id) {
                struct { bool is[1]; } take = {{inside(is, z, id)}};
                if (!__any(take.is[0])) return;
                const u64 o = order(z, id);
                if (take.is[0]) { least_o = o < least_o ? o : least_o; most_o = o > most_o ? o : most_o; }
                append(take, [&](int, int to) { sh.small[to] = o; sh.small_w[to] = weigh(z); }, kSmall);
            });
            __syncthreads();
            const int some = sh.n;
            if (some <= kSmall) {
                if (tid == 0) sh.border = border;
                __syncthreads();
                if (tid < some) {
                    const u64 o = sh.small[tid], w = sh.small_w[tid];
                    u64 before = 0;
                    for (int j = 0; j < some; ++j) before += sh.small[j] > o ? sh.small_w[j] : 0;
                    if (before < want && before + w >= want) { sh.border = o; sh.found_w = w; sh.word = (int)(uint32_t)~o; }
                }
                __syncthreads();
                if (!by_id) border = uniform(sh.border);
                break;
            }
            // More words than are compared one by one: a histogram over the orders that there are.
            for (int i = tid; i < kBins; i += THREADS) sh.weight[i] = 0;
            for (int m = 1; m < 64; m <<= 1) {
                const u64 l = __shfl_xor(least_o, m), h = __shfl_xor(most_o, m);
                least_o = l < least_o ? l : least_o;
                most_o = h > most_o ? h : most_o;
            }
            if (lane == 0) { sh.low64[wave] = least_o; sh.high64[wave] = most_o; }
            __syncthreads();
            low = ~0ull;
            high = 0;
            for (int w = 0; w < WAVES; ++w) {
                low = sh.low64[w] < low ? sh.low64[w] : low;
                high = sh.high64[w] > high ? sh.high64[w] : high;
            }
            low = uniform(low);
            high = uniform(high);
            int shift = 0;
            while ((high - low) >> shift >= (u64)kBins) ++shift;
            over([&](bool is, float z, uint32_t id) {
                if (!inside(is, z, id)) return;
                const int at = (int)((high - order(z, id)) >> shift);
                if (by_weight) atomicAdd(&sh.weight[at], weigh(z));
                else atomicAdd(&sh.count[at], 1);
            });
            __syncthreads();
            find_bin(by_weight, want);
            want = sh.want;
            high -= (u64)sh.bin << shift;
            const u64 more = (1ull << shift) - 1;
            if (high - low > more) low = high - more;
        }
    }
    if (!in_list) {
        // The draw among all words: sums of threads, of the vectors of the wave that has it, of its lanes, of the lane's words.
        // (of words of a weight of `least` at least; a hundredth of a factor of two is left for the rounding of logarithm and bound)
        float floor_z = border ? logit_of(border) : -INFINITY;
        if (least) floor_z = fmaxf(floor_z, (float)(weight.top + ((double)log2f(fminf(mp, 1.f)) - 0.01) / weight.per) - 1e-6f * fabsf(top));
        floor_z = uniform(floor_z);
        auto weigh = [&](u32x4 x, int r, u64 (&w)[E]) {
            u64 s = 0;
            float high = O::get(x, 0);
#pragma unroll
            for (int j = 1; j < E; ++j) high = fmaxf(high, O::get(x, j));
#pragma unroll
            for (int j = 0; j < E; ++j) w[j] = 0;
            if (!__any(high >= floor_z && high > -INFINITY)) return s;
#pragma unroll
            for (int j = 0; j < E; ++j) w[j] = weight(O::get(x, j));
            if (border)
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (place(O::get(x, j), (uint32_t)((first + r * 64) * E + j)) < border) w[j] = 0;
            if (least)
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (w[j] < least) w[j] = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) s += w[j];
            return s;
        };
        u64 sum = 0, w[E];
        each_vector([&](int r, u32x4 x) { sum += weigh(x, r, w); });
        const u64 upto_thread = block_scan64<THREADS>(sum, sh, total), upto_wave = last_lane(upto_thread), in_wave = last_lane(wave_scan64(sum));
        const u64 target = uniform((u64)floor((double)u * (double)total));
        u64 before = upto_wave - in_wave;
        if (before <= target && target < upto_wave) {
            bool done = false;
            each_vector([&](int r, u32x4 x) {
                if (done) return;
                const u64 s = weigh(x, r, w), upto = before + wave_scan64(s), all = last_lane(upto);
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
    }
    if (tid == 0) {
        a.word[n] = sh.word;
        if (a.logprob) a.logprob[n] = (float)log((double)sh.found_w / (double)total);
    }
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
