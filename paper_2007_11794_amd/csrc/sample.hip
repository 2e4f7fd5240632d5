// The next word of every row of logits by a given uniform number, with temperature, top-k, top-p and min-p.
//
// Words in the order of falling logits, equal ones by rising id, make every limit a prefix: top-k a count, top-p a weight, min-p a
// least weight; the draw is a prefix too, in the order of the ids.  Weights are whole numbers (fixed point), so that sums depend neither on
// their order nor on how a row is cut.  A prefix is found by a histogram over bins that follow the order, the bin in which what is
// wanted is reached, and the words of that bin, some tens, each compared with each.
//
// A row that fits the registers of one workgroup is read once.  Longer ones are cut into segments of that size for four small workgroups each,
// and take four launches: maxima, histograms, the words of the deciding bin, the draw.
//
// What bounds it: weights in 64 bits, 17 double-precision additions, products and multiply-adds of some five clocks of a SIMD with four waves, a maximum of nine
// and ten other instructions a word, 12 us for one pass over the 65536 words of a compute unit, where a limit or the draw needs all of them; rows of small
// top_k need the weights of some hundred.  256 rows of 65536, us: top_k and top_p 40, min_p 28, no limit 39, top_p alone 78 (two such passes, 14 of it the
// kept words' weights for the draw, and an LDS atomic a word), of which memory takes 14.  The kernel of these rows is at the end of its registers: ten vector ones
// and some seventy scalar ones are kept elsewhere, 44 bytes of scratch memory a lane.
// Single precision would not do: a border between two of a million words moves by what the sum in front of it is off, and the word has to be the
// definition's.
#include "device_utils.h"
#include "ops.h"

namespace rnnlm {

namespace {

typedef unsigned long long u64;
typedef u32x4 u32x4_any __attribute__((aligned(2)));          // rows may start at any element
typedef uint32_t u32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x32 __attribute__((ext_vector_type(32)));

// ---- order and weight of a word

// Rises with the number: negative numbers have all bits turned, others the sign.  -0 is +0.
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
// Falls from word to word: larger logits first, equal ones by rising id.
__device__ __forceinline__ u64 place(float z, uint32_t id) { return (u64)key_of(z) << 32 | (uint32_t)~id; }
__device__ __forceinline__ float logit_of(u64 place) { return of_key((uint32_t)(place >> 32)); }
__device__ __forceinline__ uint32_t id_of(u64 place) { return ~(uint32_t)place; }

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

// 2^y for y <= 0 as a whole number of 2^-bits, to nearest (bits <= 50; anything below -200 is nothing).  2^f on [-1/2, 1/2] is 1 + f times a polynomial fitted for the
// least relative error: with the rounding of its steps 3.3e-16 = 2^-51.4, so that a weight is off by less than one unit of 2^-50, whatever f.  (A degree less is good to
// 1.5e-14, 17 of those units, two to 8.1e-13, and a border between two words moves by that share of the sum.)  Sums and products alone, at full rate: the nearest whole number
// n comes of adding 1.5 * 2^52 and taking it off, its power of two goes into the exponent, and the result is rounded by adding 2^52, below which the last
// bit counts 1 (with the instructions for rounding, conversion and scaling 256 rows of 65536 take 40.4 us for 38.4 without limits, 82.0 for 78.2 with top_p).
__device__ __forceinline__ u64 fixed_exp2(double y, int bits) {
    y = fmax(y, -200.0);
    const double t = y + 0x1.8p52, f = y - (t - 0x1.8p52);
    double q = fma_with(0x1.e3a9369210e0ap-28, f, 0x1.b671b4e00fe0ap-24);
    q = fma_with(q, f, 0x1.62c1478e7a2f7p-20);
    q = fma_with(q, f, 0x1.ffcb58c80dfbap-17);
    q = fma_with(q, f, 0x1.4309126c04a5fp-13);
    q = fma_with(q, f, 0x1.5d87fe9b8fd28p-10);
    q = fma_with(q, f, 0x1.3b2ab6fbd6d25p-7);
    q = fma_with(q, f, 0x1.c6b08d703e172p-5);
    q = fma_with(q, f, 0x1.ebfbdff82c431p-3);
    q = fma_with(q, f, 0x1.62e42fefa3a12p-1);
    q = fma(q, f, 1.0);
    const uint32_t n = (uint32_t)__double_as_longlong(t) + (uint32_t)bits;
    const u64 x = (u64)__double_as_longlong(q) + ((u64)(n << 20) << 32);
    return (u64)__double_as_longlong(__longlong_as_double((long long)x) + 0x1p52) - 0x4330000000000000ull;
}

// ---- sums over a wave and a workgroup

template <int CTRL, int ROWS>
__device__ __forceinline__ u64 moved(u64 v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xF, false);
    return (u64)hi << 32 | lo;
}
// Inclusive prefix sums in registers, as wave_inclusive_scan.
__device__ __forceinline__ u64 wave_scan64(u64 v) {
    v += moved<0x111, 0xF>(v);
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);
    return v + moved<0x143, 0xC>(v);
}
__device__ __forceinline__ u64 of_lane(u64 v, int lane) {
    return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}

// Bins of the distance to the row's maximum, over the kOctaves factors of two in which a weight is not nothing; words that can be listed;
// words that are put in order by comparing each with each.
constexpr int kOctaves = 52, kSmall = 256;
// (16384 bins leave the deciding one of 65536 words some 30 of them; of 4096 it had over kSmall in flat rows, and took three passes more.)
constexpr int bins_of(int words) { return words > 16384 ? 16384 : words > 4096 ? 4096 : 1024; }
constexpr int list_of(int words) { return words > 4096 ? 2048 : 512; }
// Where bin b is: a thread's bins lie behind each other, and the threads of a wave read theirs from different banks.
__device__ __forceinline__ int slot(int b) { return b ^ (b >> 4 & 15); }

template <int BINS, int LIST>
struct Shared {
    union {                                                   // histogram
        u64 weight[BINS];
        int count[BINS];
    };
    u64 list[LIST];
    u64 small[kSmall], small_w[kSmall];
    u64 wave64[16], low64[16], high64[16];
    float wavef[16];
    u64 want, found_w, border;
    int bin, n, word;
};

// Inclusive over the threads.
template <int THREADS, typename S>
__device__ __forceinline__ u64 block_scan64(u64 v, S &sh, u64 &total) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    v = wave_scan64(v);
    __syncthreads();
    if (lane == 63) sh.wave64[wave] = v;
    __syncthreads();
    const u64 all = wave_scan64(lane < THREADS / 64 ? sh.wave64[lane] : 0);
    total = of_lane(all, 63);
    return v + (wave > 0 ? of_lane(all, wave - 1) : 0);
}
template <int THREADS, typename S>
__device__ __forceinline__ float block_max(float v, S &sh) {
    const int lane = threadIdx.x & 63;
    v = wave_max(v);
    __syncthreads();
    if (lane == 0) sh.wavef[threadIdx.x >> 6] = v;
    __syncthreads();
    return uniform(wave_max(lane < THREADS / 64 ? sh.wavef[lane] : -INFINITY));
}

// ---- a row

struct Limits {
    float T, p, mp, u;
    int k;
    __device__ Limits(const SampleArgs &a, int n)
        : T(a.temperature ? a.temperature[n] : 1.f), p(a.top_p ? a.top_p[n] : 1.f), mp(a.min_p ? a.min_p[n] : 0.f), u(a.u[n]), k(a.top_k ? a.top_k[n] : 0) {}
    __device__ bool bad() const { return !(T >= 0.f) || T == INFINITY || !(u >= 0.f && u < 1.f) || p != p || mp != mp; }
    __device__ bool few(int V) const { return k > 0 && k < V; }
    __device__ bool part() const { return p < 1.f; }
    __device__ u64 want_p(u64 total) const {
        const u64 w = p > 0.f ? (u64)ceil((double)p * (double)total) : 1;
        return w > 0 ? w : 1;
    }
    __device__ u64 target(u64 total) const { return uniform((u64)floor((double)u * (double)total)); }
};

// Weights and bins of a row whose maximum is known.
struct Scale {
    double high, per;                                         // the maximum; log2(e) / temperature
    float top, half_top, bin_scale;                           // bin_scale: bins for half the distance (the whole of it may pass the range of a float)
    int bits, last_bin;
    bool alike;                                               // a maximum of +infinity: those words are 0 here, all others -infinity
    u64 least;                                                // min_p's weight
    __device__ Scale(const Limits &l, float maximum, int bits, int bins) : bits(bits), last_bin(bins - 1) {
        alike = maximum == INFINITY;
        top = alike ? 0.f : maximum;
        half_top = 0.5f * top;
        high = uniform((double)top);
        per = uniform(1.4426950408889634 / (double)l.T);
        bin_scale = uniform(fminf((float)(per * (2.0 * bins / kOctaves)), 3.4e38f));
        least = l.mp > 0.f ? uniform((u64)ceil((double)fminf(l.mp, 1.f) * (double)(1ull << bits))) : 0;
    }
    __device__ __forceinline__ float seen(float z) const { return !alike ? z : z == INFINITY ? 0.f : -INFINITY; }
    __device__ __forceinline__ u64 weight(float z) const { return fixed_exp2(((double)z - high) * per, bits); }
    // Bounds of the logits in a bin and, for the lower one, in those in front of it, with room for the rounding of bin_of.
    __device__ __forceinline__ float lowest(int bin) const {
        return fmaxf(uniform(__builtin_fmaf(-2.f, (float)(bin + 1) * (1.f + 0x1p-20f) / bin_scale, top) - 0x1p-20f * fabsf(top)), -__FLT_MAX__);
    }
    __device__ __forceinline__ float highest(int bin) const {
        return uniform(__builtin_fmaf(-2.f, (float)bin * (1.f - 0x1p-20f) / bin_scale, top) + 0x1p-20f * fabsf(top));
    }
    // rises as z falls; what is in the last one weighs nothing
    __device__ __forceinline__ int bin_of(float z) const {
        const float x = __builtin_fmaf(-0.5f, z, half_top) * bin_scale;
        return x < (float)last_bin ? (int)x : last_bin;
    }
};

template <typename Z> struct Row;
template <> struct Row<float> {
    static constexpr int E = 4;
    static constexpr uint32_t kNothing = 0xFF800000u;
    static __device__ __forceinline__ float get(u32x4 v, int i) { return __uint_as_float(v[i]); }
    static __device__ __forceinline__ float one(const float *p) { return *p; }
    static __device__ __forceinline__ uint32_t pack(const float (&z)[4], int i) { return __float_as_uint(z[i]); }
};
template <> struct Row<uint16_t> {
    static constexpr int E = 8;
    static constexpr uint32_t kNothing = 0xFF80FF80u;
    static __device__ __forceinline__ float get(u32x4 v, int i) { return __uint_as_float(i & 1 ? v[i >> 1] & 0xFFFF0000u : v[i >> 1] << 16); }
    static __device__ __forceinline__ float one(const uint16_t *p) { return bf16_to_f32(*p); }
    static __device__ __forceinline__ uint32_t pack(const float (&z)[8], int i) { return __float_as_uint(z[2 * i]) >> 16 | (__float_as_uint(z[2 * i + 1]) & 0xFFFF0000u); }   // (bfloat16 values)
};

// R vectors of 16 bytes that a loop reads by a counter: code that runs once for a row and is written out for every one of its vectors is not
// executed but fetched (256 rows of 65536: 314 KB of code 345 us, 50 KB 119).
template <int R> struct Vectors;
template <> struct Vectors<4> {
    u32x16 x;
    __device__ __forceinline__ void set(int r, u32x4 v) {
#pragma unroll
        for (int q = 0; q < 4; ++q) x[4 * r + q] = v[q];
    }
    // f(r, vector) for r below `used`
    template <typename F> __device__ __forceinline__ void each(int used, F f) const {
#pragma unroll 1
        for (int r = 0; r < 4 && r < used; ++r) f(r, u32x4{x[4 * r], x[4 * r + 1], x[4 * r + 2], x[4 * r + 3]});
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

// M words of a thread; a logit of -infinity is no word.
template <int N>
struct Some {
    static constexpr int M = N;
    float z[N];
    uint32_t id[N];
};

// n words from `row` on in the registers of a workgroup; elements behind them are -infinity.  A wave's vectors lie behind each other, so
// that ids rise with wave, vector, lane, element.
template <typename Z, int THREADS, int R>
struct Words {
    typedef Z Type;
    static constexpr int E = Row<Z>::E;
    Vectors<R> v;
    int used, first;                                          // vectors of a thread; index of its first
    __device__ __forceinline__ Words(const Z *row, int n) {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), vectors = (n + E - 1) / E;
        used = (vectors + THREADS - 1) / THREADS;
        first = wave * used * 64 + lane;
        u32x4 loaded[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            loaded[r] = u32x4{Row<Z>::kNothing, Row<Z>::kNothing, Row<Z>::kNothing, Row<Z>::kNothing};
            const int i = first + r * 64;
            if (r < used && (i + 1) * E <= n) loaded[r] = *reinterpret_cast<const u32x4_any *>(reinterpret_cast<const char *>(row) + (uint32_t)i * 16u);
        }
        if (n % E) {                                          // the last vector, element by element
            const int last = vectors - 1, r_last = (last - first) / 64;
            if (last >= first && last == first + r_last * 64 && r_last < used) {
                float z[E];
#pragma unroll
                for (int j = 0; j < E; ++j) z[j] = last * E + j < n ? Row<Z>::one(row + last * E + j) : -INFINITY;
                u32x4 x;
#pragma unroll
                for (int q = 0; q < 4; ++q) x[q] = Row<Z>::pack(z, q);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (r == r_last) loaded[r] = x;
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) v.set(r, loaded[r]);
    }
    // f(index of the first, a vector's logits as the scale sees them), rising with vector, lane, element
    template <typename F> __device__ __forceinline__ void vectors(bool alike, F f) const {
        v.each(used, [&](int r, u32x4 x) {
            float z[E];
#pragma unroll
            for (int j = 0; j < E; ++j) {
                z[j] = Row<Z>::get(x, j);
                if (alike) z[j] = z[j] == INFINITY ? 0.f : -INFINITY;
            }
            f((first + r * 64) * E, z);
        });
    }
    // f(index of the first, four logits as the scale sees them), indices of a thread rising
    template <typename F> __device__ __forceinline__ void fours(bool alike, F f) const {
        v.each(used, [&](int r, u32x4 x) {
#pragma unroll 1
            for (int h = 0; h < E; h += 4) {
                float z[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) z[j] = E == 4 ? Row<Z>::get(x, j) : h ? Row<Z>::get(x, E - 4 + j) : Row<Z>::get(x, j);
                if (alike)
#pragma unroll
                    for (int j = 0; j < 4; ++j) z[j] = z[j] == INFINITY ? 0.f : -INFINITY;
                f((first + r * 64) * E + h, z);
            }
        });
    }
    // f(words), ids from `from` on
    template <typename F> __device__ __forceinline__ void each(bool alike, int from, F f) const {
        fours(alike, [&](int i, const float (&z)[4]) { f(Some<4>{{z[0], z[1], z[2], z[3]}, {(uint32_t)(from + i), (uint32_t)(from + i + 1), (uint32_t)(from + i + 2), (uint32_t)(from + i + 3)}}); });
    }
    // The places of all words from `low` to `high` into a list of at most `most`, `n` of them counted; a thread's behind each other.
    __device__ __forceinline__ void list(const Scale &scale, float low, float high, int from, u64 *to, int *n, int most) const {
        int mine = 0;
        fours(scale.alike, [&](int, const float (&z)[4]) {
            if (!__any(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])) >= low)) return;
#pragma unroll
            for (int j = 0; j < 4; ++j) mine += z[j] >= low && z[j] <= high;
        });
        const int upto = wave_inclusive_scan(mine), all = __builtin_amdgcn_readlane(upto, 63);
        if (all == 0) return;
        int at = 0;
        if ((threadIdx.x & 63) == 63) at = atomicAdd(n, all);
        at = __builtin_amdgcn_readlane(at, 63) + upto - mine;
        fours(scale.alike, [&](int i, const float (&z)[4]) {
            if (!__any(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])) >= low)) return;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (z[j] >= low && z[j] <= high) {
                    if (at < most) to[at] = place(z[j], (uint32_t)(from + i + j));
                    ++at;
                }
        });
    }
    // This thread's largest logit; NaN where there is one.
    __device__ __forceinline__ float largest() const {
        float high = -INFINITY;
        bool nan = false;
        v.each(used, [&](int, u32x4 x) {
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float z = Row<Z>::get(x, j);
                high = fmaxf(high, z);
                nan |= z != z;
            }
        });
        return nan ? quiet_nan() : high;
    }
};

// ---- the search for a prefix

enum Kind { kCount, kWeight, kDraw };        // top_k: words, by place.  top_p: weight, by place.  The draw: weight of at least `least`, by id.

// `over(f)` calls f(words) for the words of a source (registers, a list, memory), the same number of times in all lanes of a wave.
template <int THREADS, int BINS, int LIST>
struct Search {
    static constexpr int WAVES = THREADS / 64;
    Shared<BINS, LIST> &sh;
    const Scale &scale;
    u64 border;                              // place of the last word kept (0: all)
    uint32_t id_from;                        // ids go to bins from here on
    int id_shift, coarse;                    // 2^coarse of the scale's bins are one here: a list needs few, and they are cleared and added up for every limit
    __device__ Search(Shared<BINS, LIST> &sh, const Scale &scale, uint32_t from, int n) : sh(sh), scale(scale), border(0), id_from(from), id_shift(0), coarse(0) {
        while ((n - 1) >> id_shift >= BINS) ++id_shift;
    }
    __device__ __forceinline__ void coarsen(int to) { coarse = to; id_shift += to; }
    __device__ __forceinline__ int last_bin() const { return (BINS >> coarse) - 1; }
    __device__ __forceinline__ bool kept(float z, uint32_t id) const { return z > -INFINITY && place(z, id) >= border; }
    __device__ __forceinline__ u64 weigh(Kind kind, float z) const {
        const u64 w = kind == kCount ? 1 : scale.weight(z);
        return kind == kDraw && w < scale.least ? 0 : w;
    }
    __device__ __forceinline__ int bin_at(Kind kind, float z, uint32_t id) const { return kind == kDraw ? (int)((id - id_from) >> id_shift) : scale.bin_of(z) >> coarse; }
    __device__ __forceinline__ u64 order(Kind kind, float z, uint32_t id) const { return kind == kDraw ? ~(u64)id : place(z, id); }
    // Histogram of the words kept.  (Whoever read the last one did so in front of a barrier.)
    template <typename O>
    __device__ __forceinline__ void histogram(Kind kind, O over) {
        for (int i = threadIdx.x; i < BINS >> coarse; i += THREADS) sh.weight[i] = 0;
        __syncthreads();
        if (kind != kCount) over([&](auto some) {
#pragma unroll
            for (int j = 0; j < some.M; ++j) {
                u64 w = scale.weight(some.z[j]);
                w = kept(some.z[j], some.id[j]) && !(kind == kDraw && w < scale.least) ? w : 0;
                if (w) atomicAdd(&sh.weight[slot(bin_at(kind, some.z[j], some.id[j]))], w);
            }
        });
        else over([&](auto some) {
#pragma unroll
            for (int j = 0; j < some.M; ++j)
                if (kept(some.z[j], some.id[j])) atomicAdd(&sh.count[slot(bin_at(kCount, some.z[j], some.id[j]))], 1);
        });
        __syncthreads();
    }
    // The bin where want_of(all of the histogram) is reached from the front (the last one if it is not), and what is still wanted of that bin.
    template <typename F>
    __device__ __forceinline__ int find_bin(bool counts, u64 &want, u64 &total, F want_of) {
        const int tid = threadIdx.x, bins = BINS >> coarse, per_thread = (bins + THREADS - 1) / THREADS;
        auto in_bin = [&](int i) { return counts ? (u64)sh.count[slot(tid * per_thread + i)] : sh.weight[slot(tid * per_thread + i)]; };
        u64 sum = 0;
#pragma unroll 4
        for (int i = 0; i < per_thread; ++i) sum += in_bin(i);
        u64 upto = block_scan64<THREADS>(sum, sh, total) - sum;
        want = want_of(total);
        if (tid == 0) {
            sh.n = 0;                                         // of the bin's words, for resolve()
            sh.border = border;
            if (total < want) { sh.bin = bins - 1; sh.want = want; }
        }
        if (upto < want && upto + sum >= want) {
            int i = 0;
            for (u64 h = in_bin(0); upto + h < want; h = in_bin(++i)) upto += h;
            sh.bin = tid * per_thread + i;
            sh.want = want - upto;
        }
        __syncthreads();
        want = uniform(sh.want);
        return __builtin_amdgcn_readfirstlane(sh.bin);
    }
    // Of the words of `bin` the one at which `want` is reached: the new border, or the word drawn (sh.word, sh.found_w).  Behind find_bin().
    template <typename O>
    __device__ __forceinline__ void resolve(Kind kind, int bin, u64 want, O over) {
        const int tid = threadIdx.x, lane = tid & 63;
        u64 low = 0, high = ~0ull;                            // of the orders
        const float low_z = kind == kDraw ? -INFINITY : scale.lowest(((bin + 1) << coarse) - 1), high_z = kind == kDraw ? INFINITY : scale.highest(bin << coarse);
        auto inside = [&](float z, uint32_t id) {
            const u64 o = order(kind, z, id);
            return bin_at(kind, z, id) == bin && kept(z, id) && o >= low && o <= high;
        };
        // f(which are inside, words), where there are any
        auto insiders = [&](auto f) {
            over([&](auto some) {
                constexpr int M = decltype(some)::M;
                // most batches have no word of one bin, and of those most none as large
                float largest = some.z[0];
#pragma unroll
                for (int j = 1; j < M; ++j) largest = fmaxf(largest, some.z[j]);
                if (!__any(largest >= low_z)) return;
                bool any = false;
#pragma unroll
                for (int j = 0; j < M; ++j) any |= kind == kDraw ? bin_at(kind, some.z[j], some.id[j]) == bin : some.z[j] >= low_z && some.z[j] <= high_z;
                if (!__any(any)) return;
#pragma unroll
                for (int j = 0; j < M; ++j) f(inside(some.z[j], some.id[j]), some.z[j], some.id[j]);
            });
        };
        while (true) {
            u64 least_o = ~0ull, most_o = 0;
            insiders([&](bool is, float z, uint32_t id) {
                const u64 who = __ballot(is);
                if (who == 0) return;
                int at = 0;
                if (lane == 0) at = atomicAdd(&sh.n, __popcll(who));
                const u64 o = order(kind, z, id);
                at = __builtin_amdgcn_readfirstlane(at) + __popcll(who & ((1ull << lane) - 1));
                if (is) {
                    least_o = o < least_o ? o : least_o;
                    most_o = o > most_o ? o : most_o;
                    if (at < kSmall) { sh.small[at] = o; sh.small_w[at] = weigh(kind, z); }
                }
            });
            __syncthreads();
            const int some = __builtin_amdgcn_readfirstlane(sh.n);
            if (some <= kSmall) {
                if (tid < some) {
                    const u64 o = sh.small[tid], w = sh.small_w[tid];
                    u64 before = 0;
                    for (int j0 = 0; j0 < some; j0 += 8)      // (eight from LDS at a time; kSmall is a multiple)
#pragma unroll
                        for (int j = j0; j < j0 + 8; ++j) before += j < some && sh.small[j] > o ? sh.small_w[j] : 0;
                    if (before < want && before + w >= want) { sh.border = o; sh.found_w = w; sh.word = (int)id_of(o); }
                }
                __syncthreads();
                if (kind != kDraw) border = uniform(sh.border);
                return;
            }
            // More words than are compared one by one: a histogram over the orders that there are.
            for (int m = 1; m < 64; m <<= 1) {
                const u64 l = __shfl_xor(least_o, m), h = __shfl_xor(most_o, m);
                least_o = l < least_o ? l : least_o;
                most_o = h > most_o ? h : most_o;
            }
            if (lane == 0) { sh.low64[tid >> 6] = least_o; sh.high64[tid >> 6] = most_o; }
            for (int i = tid; i < BINS >> coarse; i += THREADS) sh.weight[i] = 0;
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
            while ((high - low) >> shift >= (u64)(BINS >> coarse)) ++shift;
            insiders([&](bool is, float z, uint32_t id) {
                if (!is) return;
                const int at = (int)((high - order(kind, z, id)) >> shift);
                if (kind == kCount) atomicAdd(&sh.count[slot(at)], 1);
                else atomicAdd(&sh.weight[slot(at)], weigh(kind, z));
            });
            __syncthreads();
            u64 total;
            const u64 still = want;
            high -= (u64)find_bin(kind == kCount, want, total, [&](u64) { return still; }) << shift;
            const u64 more = (1ull << shift) - 1;
            if (high - low > more) low = high - more;
        }
    }
    // One limit, or the draw: the weight of all words it was made of (0 where nothing had to be searched).
    template <typename O>
    __device__ __forceinline__ u64 step(Kind kind, const Limits &l, O over) {
        histogram(kind, over);
        u64 want, total;
        const int bin = find_bin(kind == kCount, want, total, [&](u64 all) { return kind == kCount ? (u64)l.k : kind == kWeight ? l.want_p(all) : l.target(all) + 1; });
        if (bin < last_bin() || kind == kDraw) resolve(kind, bin, want, over);      // in the last bin nothing has a weight
        return total;
    }
    // All limits and the draw.
    template <typename O>
    __device__ __forceinline__ u64 all_steps(const Limits &l, int V, O over) {
        u64 total = 0;
#pragma unroll 1
        for (int kind = kCount; kind <= kDraw; ++kind)
            if (kind == kCount ? l.few(V) : kind == kWeight ? l.part() : true) total = step((Kind)kind, l, over);
        return total;
    }
};

__device__ __forceinline__ void answer(const SampleArgs &a, int n, int word, float logprob) {
    if (threadIdx.x == 0) {
        a.word[n] = word;
        if (a.logprob) a.logprob[n] = logprob;
    }
}
__device__ __forceinline__ float log_share(u64 w, u64 total) { return (float)log((double)w / (double)total); }

// The draw among words in registers, ids from `from` on, that `border` keeps, in the order of the ids: sums of threads, of the vectors of the wave
// that has it, of its lanes, of the lane's words.  target_of(their weight) is what the sum has to pass.
template <int THREADS, typename W, typename S, typename F>
__device__ __forceinline__ u64 draw_from_registers(const W &words, S &sh, const Scale &scale, const Limits &l, u64 border, int from, F target_of) {
    // No word below it is kept.  (By min_p: of a number of `least` at least, which half a unit less is rounded to, with a hundredth of a factor of
    // two for what logarithm and bound are off.)
    float floor_z = border ? logit_of(border) : -INFINITY;
    if (scale.least) floor_z = fmaxf(floor_z, (float)(scale.high + ((double)log2f((float)scale.least - 0.5f) - scale.bits - 0.01) / scale.per) - 1e-6f * fabsf(scale.top));
    floor_z = uniform(floor_z);
    auto weigh = [&](int i, const float (&z)[4], u64 (&w)[4]) {
        u64 s = 0;
        const float high = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = 0;
        if (!__any(high >= floor_z && high > -INFINITY)) return s;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = scale.weight(z[j]);
        if (border)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (place(z[j], (uint32_t)(from + i + j)) < border) w[j] = 0;
        if (scale.least)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (w[j] < scale.least) w[j] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) s += w[j];
        return s;
    };
    u64 sum = 0, total;
    words.fours(scale.alike, [&](int i, const float (&z)[4]) {
        u64 w[4];
        sum += weigh(i, z, w);
    });
    const u64 upto_wave = of_lane(block_scan64<THREADS>(sum, sh, total), 63), target = target_of(total);
    u64 before = upto_wave - of_lane(wave_scan64(sum), 63);
    if (before <= target && target < upto_wave) {
        bool done = false;
        words.vectors(scale.alike, [&](int i, const float (&z)[W::E]) {
            if (done) return;
            u64 w[W::E / 4][4], s = 0;
#pragma unroll
            for (int h = 0; h < W::E / 4; ++h) {
                const float four[4] = {z[4 * h], z[4 * h + 1], z[4 * h + 2], z[4 * h + 3]};
                s += weigh(i + 4 * h, four, w[h]);
            }
            const u64 upto = before + wave_scan64(s), all = of_lane(upto, 63);
            if (all > target) {
                u64 at = upto - s;
                if (at <= target && target < upto) {
#pragma unroll
                    for (int j = 0; j < W::E; ++j) {
                        const u64 x = w[j / 4][j % 4];
                        if (at <= target && target < at + x) { sh.word = from + i + j; sh.found_w = x; }
                        at += x;
                    }
                }
                done = true;
            }
            before = all;
        });
    }
    __syncthreads();
    return total;
}

template <typename Z, int THREADS, int R>
constexpr int row_bins() { return bins_of(THREADS * R * Row<Z>::E); }
// A row in the registers of one workgroup.
template <typename Z, int THREADS, int R>
__global__ __launch_bounds__(THREADS, 4) void sample_row_kernel(SampleArgs a, int bits) {
    constexpr int BINS = row_bins<Z, THREADS, R>(), LIST = list_of(THREADS * R * Row<Z>::E);
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Shared<BINS, LIST> &sh = *reinterpret_cast<Shared<BINS, LIST> *>(lds);
    const int tid = threadIdx.x, n = blockIdx.x, V = a.V;
    const Limits l(a, n);
    const Words<Z, THREADS, R> words(static_cast<const Z *>(a.logits) + n * a.ld, V);
    for (int i = tid; i < BINS; i += THREADS) sh.count[i] = 0;
    if (tid == 0) { sh.n = 0; sh.word = 0x7FFFFFFF; }
    float mine = words.largest();
    const bool nan = __syncthreads_or(mine != mine);
    const float maximum = block_max<THREADS>(mine, sh);
    if (nan || l.bad() || maximum == -INFINITY) { answer(a, n, -1, quiet_nan()); return; }
    if (l.T == 0.f) {
        uint32_t at = 0x7FFFFFFF;
        if (__any(mine == maximum)) words.each(false, 0, [&](auto some) {
#pragma unroll
            for (int j = 0; j < some.M; ++j) at = some.z[j] == maximum && some.id[j] < at ? some.id[j] : at;
        });
        if (at != 0x7FFFFFFF) atomicMin(&sh.word, (int)at);
        __syncthreads();
        answer(a, n, sh.word, 0.f);
        return;
    }
    const Scale scale(l, maximum, bits, BINS);
    mine = scale.seen(mine);
    Search<THREADS, BINS, LIST> search(sh, scale, 0, V);
    // Few words kept: they are listed.  The top_k-th largest of the threads' own maxima is no more than the top_k-th largest logit, so whatever
    // lies in its bin or in front of it is enough.
    bool in_list = false;
    int listed = 0;
    if (l.few(V) && l.k <= THREADS / 2) {
        if (mine > -INFINITY) atomicAdd(&sh.count[slot(scale.bin_of(mine))], 1);
        __syncthreads();
        u64 want, all;
        const int edge = search.find_bin(true, want, all, [&](u64) { return (u64)l.k; });
        if (edge < BINS - 1) {
            words.list(scale, scale.lowest(edge), INFINITY, 0, sh.list, &sh.n, LIST);
            __syncthreads();
            listed = __builtin_amdgcn_readfirstlane(sh.n);
            in_list = listed <= LIST;
            if (in_list) search.coarsen(BINS > THREADS ? __builtin_ctz(BINS / THREADS) : 0);
        }
    }
    auto over = [&](auto f) {
        if (in_list)
            for (int i = tid; i - tid < listed; i += THREADS) {
                const u64 w = i < listed ? sh.list[i] : 0;
                f(Some<1>{{i < listed ? logit_of(w) : -INFINITY}, {id_of(w)}});
            }
        else words.each(scale.alike, 0, f);
    };
    u64 total = 0;
#pragma unroll 1
    for (int kind = kCount; kind <= kDraw; ++kind)
        if (kind == kCount ? l.few(V) : kind == kWeight ? l.part() : in_list) total = search.step((Kind)kind, l, over);
    if (!in_list) total = draw_from_registers<THREADS>(words, sh, scale, l, search.border, 0, [&](u64 all) { return l.target(all); });
    answer(a, n, sh.word, log_share(sh.found_w, total));
}

// ---- rows in segments

constexpr int kSegThreads = 256, kSegWaves = kSegThreads / 64, kSegVectors = 16, kLongBins = 4096, kPickThreads = 1024;
template <typename Z> __host__ __device__ constexpr int segment_words() { return kSegThreads * kSegVectors * Row<Z>::E; }
// Words of a wave's part of the segment that word `from` begins, as Words lays them out.
template <typename Z> __device__ __forceinline__ int part_words(int V, int from) {
    const int len = min(V - from, segment_words<Z>());
    return ((len + Row<Z>::E - 1) / Row<Z>::E + kSegThreads - 1) / kSegThreads * 64 * Row<Z>::E;
}

// Of one row in the workspace, behind its histogram of kLongBins weights (or counts): the deciding bin and what is wanted of it, the words listed,
// how many there are, of every segment its maximum, and of every wave's quarter of one the weight of its words that are kept for certain.
struct LongRow {
    u64 *hist, *list, *sums;
    u64 *want;
    int *bin, *listed;
    float *tops;
    static __host__ __device__ size_t bytes(int V, int segments) { return (size_t)(kLongBins + long_list(V) + segments * kSegWaves) * 8 + 16 + ((size_t)segments * 4 + 15) / 16 * 16; }
    __device__ LongRow(void *ws, int n, int V, int segments) {
        char *p = static_cast<char *>(ws) + n * bytes(V, segments);
        hist = reinterpret_cast<u64 *>(p);
        list = hist + kLongBins;
        sums = list + long_list(V);
        want = sums + segments * kSegWaves;
        bin = reinterpret_cast<int *>(want + 1);
        listed = bin + 1;
        tops = reinterpret_cast<float *>(listed + 1);
    }
    // Segment s: the sum over this wave of `sum`.
    __device__ __forceinline__ void put_sum(int s, u64 sum) const {
        sum = wave_scan64(sum);
        if ((threadIdx.x & 63) == 63) sums[s * kSegWaves + (threadIdx.x >> 6)] = sum;
    }
    // The row's maximum; NaN where there is one.
    template <int THREADS, typename S>
    __device__ __forceinline__ float maximum(int segments, S &sh) const {
        float m = -INFINITY;
        bool nan = false;
        for (int i = threadIdx.x; i < segments; i += THREADS) {
            const float t = tops[i];
            nan |= t != t;
            m = fmaxf(m, t);
        }
        nan = __syncthreads_or(nan);
        m = block_max<THREADS>(m, sh);
        return nan ? quiet_nan() : m;
    }
};
// Of a row with top_k all words that can be kept are listed, and the last launch does the rest, unless they are too many; then, and with top_p alone,
// the words of the deciding bin.  (Too many with top_p as well: the last launch reads the row itself.)
__device__ __forceinline__ bool lists_all(const Limits &l, int V) { return l.few(V) && l.k <= long_list(V) / 2; }
__device__ __forceinline__ bool lists_bin(const Limits &l, int V) { return l.few(V) ? !lists_all(l, V) && !l.part() : l.part(); }

template <typename Z>
__global__ __launch_bounds__(kSegThreads) void sample_tops_kernel(SampleArgs a, int segments) {
    __shared__ Shared<16, 1> sh;
    const int n = blockIdx.x / segments, s = blockIdx.x % segments, from = s * segment_words<Z>(), len = min(a.V - from, segment_words<Z>());
    const LongRow r(a.ws, n, a.V, segments);
    const Words<Z, kSegThreads, kSegVectors> words(static_cast<const Z *>(a.logits) + n * a.ld + from, len);
    for (int i = s * kSegThreads + threadIdx.x; i < kLongBins; i += segments * kSegThreads) r.hist[i] = 0;
    if (s == 0 && threadIdx.x == 0) *r.listed = 0;
    const float mine = words.largest();
    const bool nan = __syncthreads_or(mine != mine);
    const float top = block_max<kSegThreads>(mine, sh);
    if (threadIdx.x == 0) r.tops[s] = nan ? quiet_nan() : top;
}

template <typename Z>
__global__ __launch_bounds__(kSegThreads) void sample_weigh_kernel(SampleArgs a, int segments, int bits) {
    __shared__ Shared<kLongBins, 1> sh;
    const int n = blockIdx.x / segments, s = blockIdx.x % segments, from = s * segment_words<Z>(), len = min(a.V - from, segment_words<Z>());
    const Limits l(a, n);
    const LongRow r(a.ws, n, a.V, segments);
    const Words<Z, kSegThreads, kSegVectors> words(static_cast<const Z *>(a.logits) + n * a.ld + from, len);
    const float maximum = r.maximum<kSegThreads>(segments, sh);
    if (l.bad() || !(maximum > -INFINITY) || l.T == 0.f) return;
    const Scale scale(l, maximum, bits, kLongBins);
    Search<kSegThreads, kLongBins, 1> search(sh, scale, 0, a.V);
    auto over = [&](auto f) { words.each(scale.alike, from, f); };
    if (!l.few(a.V) && !l.part()) {
        u64 sum = 0;
        over([&](auto some) {
#pragma unroll
            for (int j = 0; j < some.M; ++j) {
                const u64 w = search.weigh(kDraw, some.z[j]);
                sum += some.z[j] > -INFINITY ? w : 0;
            }
        });
        r.put_sum(s, sum);
        return;
    }
    const bool counts = l.few(a.V);
    search.histogram(counts ? kCount : kWeight, over);
    for (int i = threadIdx.x; i < kLongBins; i += kSegThreads) {
        const u64 h = counts ? (u64)sh.count[i] : sh.weight[i];
        if (h) atomicAdd(&r.hist[i], h);
    }
}

template <typename Z>
__global__ __launch_bounds__(kSegThreads) void sample_gather_kernel(SampleArgs a, int segments, int bits) {
    __shared__ Shared<kLongBins, 1> sh;
    const int tid = threadIdx.x, n = blockIdx.x / segments, s = blockIdx.x % segments, from = s * segment_words<Z>(), len = min(a.V - from, segment_words<Z>());
    const Limits l(a, n);
    const bool all = lists_all(l, a.V);
    if (!all && !lists_bin(l, a.V)) return;
    const LongRow r(a.ws, n, a.V, segments);
    const Words<Z, kSegThreads, kSegVectors> words(static_cast<const Z *>(a.logits) + n * a.ld + from, len);
    const float maximum = r.maximum<kSegThreads>(segments, sh);
    if (l.bad() || !(maximum > -INFINITY) || l.T == 0.f) return;
    const Scale scale(l, maximum, bits, kLongBins);
    Search<kSegThreads, kLongBins, 1> search(sh, scale, 0, a.V);
    u64 h[kLongBins / kSegThreads], want, total;               // (all on their way at once)
#pragma unroll
    for (int i = 0; i < kLongBins / kSegThreads; ++i) h[i] = r.hist[i * kSegThreads + tid];
#pragma unroll
    for (int i = 0; i < kLongBins / kSegThreads; ++i) sh.weight[i * kSegThreads + tid] = h[i];
    __syncthreads();
    const int bin = search.find_bin(false, want, total, [&](u64 all_of_it) { return l.few(a.V) ? (u64)l.k : l.want_p(all_of_it); });
    if (s == 0 && tid == 0) { *r.bin = bin; *r.want = want; }
    // The words of the bin (a few more do no harm), or all up to it, and the weight of those in front of it.
    const float low = scale.lowest(bin);
    if (all || bin < kLongBins - 1) words.list(scale, low, all ? INFINITY : scale.highest(bin), from, r.list, r.listed, long_list(a.V));
    if (all) return;
    u64 sum = 0;
    words.each(scale.alike, from, [&](auto some) {
        bool any = false;
#pragma unroll
        for (int j = 0; j < some.M; ++j) any |= some.z[j] >= low;
        if (!__any(any)) return;
#pragma unroll
        for (int j = 0; j < some.M; ++j) {
            const u64 w = search.weigh(kDraw, some.z[j]);
            sum += some.z[j] > -INFINITY && scale.bin_of(some.z[j]) < bin ? w : 0;
        }
    });
    r.put_sum(s, sum);
}

template <typename Z>
__global__ __launch_bounds__(kPickThreads, 4) void sample_pick_kernel(SampleArgs a, int segments, int bits) {
    constexpr int BINS = kLongBins;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    Shared<BINS, 1> &sh = *reinterpret_cast<Shared<BINS, 1> *>(lds);
    u64 *const held = reinterpret_cast<u64 *>(lds + sizeof(Shared<BINS, 1>));
    const int tid = threadIdx.x, n = blockIdx.x, V = a.V;
    const Limits l(a, n);
    const LongRow r(a.ws, n, a.V, segments);
    const Z *row = static_cast<const Z *>(a.logits) + n * a.ld;
    const float maximum = r.maximum<kPickThreads>(segments, sh);
    if (l.bad() || !(maximum > -INFINITY)) { answer(a, n, -1, quiet_nan()); return; }
    if (tid == 0) sh.word = 0x7FFFFFFF;
    __syncthreads();
    if (l.T == 0.f) {
        for (int s = tid; s < segments; s += kPickThreads)
            if (r.tops[s] == maximum) atomicMin(&sh.word, s);
        __syncthreads();
        const int from = sh.word * segment_words<Z>(), to = min(V, from + segment_words<Z>());
        __syncthreads();
        if (tid == 0) sh.word = 0x7FFFFFFF;
        __syncthreads();
        for (int i = from + tid; i < to; i += kPickThreads)
            if (Row<Z>::one(row + i) == maximum) { atomicMin(&sh.word, i); break; }
        __syncthreads();
        answer(a, n, sh.word, 0.f);
        return;
    }
    const Scale scale(l, maximum, bits, BINS);
    Search<kPickThreads, BINS, 1> search(sh, scale, 0, V);
    // Words in memory, eight of a thread on their way at once.
    auto over_row = [&](auto f) {
        for (int i0 = 0; i0 < V; i0 += 8 * kPickThreads) {
            float z[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int i = i0 + q * kPickThreads + tid;
                z[q] = i < V ? scale.seen(Row<Z>::one(row + i)) : -INFINITY;
            }
#pragma unroll 1
            for (int q = 0; q < 8; ++q) {
                float x = z[0];
#pragma unroll
                for (int p = 1; p < 8; ++p) x = q == p ? z[p] : x;
                const int i = i0 + q * kPickThreads + tid;
                f(Some<1>{{x}, {(uint32_t)i}});
            }
        }
    };
    const bool all = lists_all(l, V), of_bin = lists_bin(l, V);
    const int listed = all || of_bin ? *r.listed : 0;
    const bool fits = listed <= long_list(V);                 // (too many are counted on, but not listed)
    // (several passes go over the list: it stays in LDS where it fits)
    const u64 *list = r.list;
    if (list_in_lds(listed, V)) {
        for (int i = tid; i < listed; i += kPickThreads) held[i] = r.list[i];
        list = held;
        __syncthreads();
    }
    auto over_list = [&](auto f) {
        for (int i0 = 0; i0 < listed; i0 += 8 * kPickThreads) {
            u64 w[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int i = i0 + q * kPickThreads + tid;
                w[q] = i < listed ? list[i] : 0;
            }
#pragma unroll 1
            for (int q = 0; q < 8 && i0 + q * kPickThreads < listed; ++q) {
                u64 x = w[0];
#pragma unroll
                for (int p = 1; p < 8; ++p) x = q == p ? w[p] : x;
                f(Some<1>{{i0 + q * kPickThreads + tid < listed ? logit_of(x) : -INFINITY}, {id_of(x)}});
            }
        }
    };
    u64 total;
    if (!fits || (all || of_bin ? false : l.few(V))) {
        total = search.all_steps(l, V, over_row);
    } else if (all) {
        total = search.all_steps(l, V, over_list);
    } else {
        const int parts = segments * kSegWaves;
        const bool in_lds = parts <= BINS;                    // what the bin's words add to the parts' sums
        for (int i = tid; i < BINS; i += kPickThreads) sh.weight[i] = 0;
        if (of_bin && listed) {
            const int bin = *r.bin;
            if (tid == 0) { sh.n = 0; sh.border = 0; }
            __syncthreads();
            search.resolve(l.few(V) ? kCount : kWeight, bin, *r.want, over_list);
            for (int i = tid; i < BINS; i += kPickThreads) sh.weight[i] = 0;
            __syncthreads();
            over_list([&](auto some) {
                if (!search.kept(some.z[0], some.id[0]) || scale.bin_of(some.z[0]) != bin) return;
                const u64 w = search.weigh(kDraw, some.z[0]);
                const int seg = some.id[0] / segment_words<Z>(), from = seg * segment_words<Z>(), s = seg * kSegWaves + ((int)some.id[0] - from) / part_words<Z>(V, from);
                if (in_lds) atomicAdd(&sh.weight[s], w);
                else __hip_atomic_fetch_add(&r.sums[s], w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            });
            seen_by_all();
        }
        __syncthreads();
        auto sum_of = [&](int s) { return s < parts ? __hip_atomic_load(&r.sums[s], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + (in_lds ? sh.weight[s] : 0) : 0ull; };
        u64 sum = 0, in_turn;
        for (int s = tid; s < parts; s += kPickThreads) sum += sum_of(s);
        block_scan64<kPickThreads>(sum, sh, total);
        const u64 target = l.target(total);
        if (tid == 0) sh.bin = 0;
        u64 before = 0;
        for (int s0 = 0; s0 < parts; s0 += kPickThreads) {            // the part that has it, and what lies in front of it
            const u64 mine = sum_of(s0 + tid), upto = before + block_scan64<kPickThreads>(mine, sh, in_turn);
            if (upto - mine <= target && target < upto) { sh.bin = s0 + tid; sh.want = target - (upto - mine) + 1; }
            before += in_turn;
        }
        __syncthreads();
        const int s = __builtin_amdgcn_readfirstlane(sh.bin), segment = s / kSegWaves * segment_words<Z>(), part_of = part_words<Z>(V, segment);
        const int from = segment + s % kSegWaves * part_of, to = min(V, from + part_of);
        const u64 wanted = uniform(sh.want);
        const Words<Z, kPickThreads, 4> words(row + from, to - from);
        draw_from_registers<kPickThreads>(words, sh, scale, l, search.border, from, [&](u64) { return wanted - 1; });
    }
    answer(a, n, sh.word, log_share(sh.found_w, total));
}

template <typename Z>
int segments_of(int V) { return (V + segment_words<Z>() - 1) / segment_words<Z>(); }

template <typename Z, int THREADS, int R>
hipError_t launch_row(const SampleArgs &a, int bits, hipStream_t stream) {
    static LdsLimit limit;
    constexpr size_t bytes = sizeof(Shared<row_bins<Z, THREADS, R>(), list_of(THREADS * R * Row<Z>::E)>);
    const auto kernel = sample_row_kernel<Z, THREADS, R>;
    const hipError_t e = limit.ensure(reinterpret_cast<const void *>(kernel), bytes);
    if (e != hipSuccess) return e;
    kernel<<<a.N, THREADS, bytes, stream>>>(a, bits);
    return hipGetLastError();
}
template <typename Z>
hipError_t launch(const SampleArgs &a, int bits, hipStream_t stream) {
    const int vectors = (a.V + Row<Z>::E - 1) / Row<Z>::E;
    // Four waves a row for short rows, and for any that fit them where there are more rows than compute units.  Us, 256 threads / 1024: a row of 1000
    // words 11.3 / 13.8; rows of 2853: 141 take 19.2 / 15.2, 600 take 21.7 / 32.5; 256 rows of 4000, top_p, 19.4 / 13.3.
    if (vectors <= 256 * 4 && (a.V < 2048 || a.N > kChipGroups)) return launch_row<Z, 256, 4>(a, bits, stream);
    if (vectors <= 1024 * 4) return launch_row<Z, 1024, 4>(a, bits, stream);
    if (vectors <= 1024 * 16) return launch_row<Z, 1024, 16>(a, bits, stream);
    const int segments = segments_of<Z>(a.V);
    if ((long long)a.N * segments > 0x7FFFFFFF / kSegThreads) return hipErrorInvalidValue;     // (more than 2^37 logits)
    const int groups = a.N * segments;
    static LdsLimit limit;
    constexpr size_t pick_bytes = sizeof(Shared<kLongBins, 1>) + (size_t)kLongHeld * 8;
    const hipError_t e = limit.ensure(reinterpret_cast<const void *>(sample_pick_kernel<Z>), pick_bytes);
    if (e != hipSuccess) return e;
    sample_tops_kernel<Z><<<groups, kSegThreads, 0, stream>>>(a, segments);
    sample_weigh_kernel<Z><<<groups, kSegThreads, 0, stream>>>(a, segments, bits);
    sample_gather_kernel<Z><<<groups, kSegThreads, 0, stream>>>(a, segments, bits);
    sample_pick_kernel<Z><<<a.N, kPickThreads, pick_bytes, stream>>>(a, segments, bits);
    return hipGetLastError();
}

}  // namespace

size_t sample_workspace_bytes(int N, int V) {                 // (of either type)
    return V > 1024 * 16 * Row<float>::E ? (size_t)N * LongRow::bytes(V, segments_of<float>(V)) : 16;
}

hipError_t launch_sample(const SampleArgs &a, hipStream_t stream) {
    int bits = 62;                                            // sums of V weights stay below 2^62
    for (long long v = 1; v < a.V; v <<= 1) --bits;
    if (bits > 50) bits = 50;
    return a.bf16 ? launch<uint16_t>(a, bits, stream) : launch<float>(a, bits, stream);
}

}  // namespace rnnlm
