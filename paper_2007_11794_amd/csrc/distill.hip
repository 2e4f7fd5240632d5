// Loss of rows of logits against a teacher's top logits and labels, and its gradient.
//
// A row is read once: it stays in the registers of its workgroup from its maximum over its sums to its gradient (of longer rows a part stays in
// LDS, and what is left is read again).  The teacher's words are some tens among tens of thousands: the gradient is
// written as if there were none, and their own places once more behind it, from the logits gathered before.  Where rows are too few
// to fill the chip they are cut into segments: one launch for a segment's maximum and sums, one that joins them and goes on.
//
// What bounds it is memory: 1024 rows of 65536 in bfloat16 with labels, loss and gradient, 68 us = 3.9 TB/s of a copy's 4.8 (up to four exponentials a
// logit are 27 us of every SIMD's time, beside it); 509 rows of 20011, gradient alone, 15.4 us = 5.3 TB/s; 256 rows of 200000 in fp32 110 us, of which
// 45 % of a row's bytes are read twice.
#include <algorithm>

#include "device_utils.h"
#include "ops.h"

namespace rnnlm {

namespace {

// Logits count by half their distance from the largest one: the whole of it may pass the range of a float, at temperatures where it still counts.  (One
// instruction, as a difference, with the same rounding.)
__device__ __forceinline__ float half_distance(float z, float half_top) { return __builtin_fmaf(0.5f, z, -half_top); }
constexpr float kPer1 = 2.f * kLog2e;                        // 2 log2(e) / T at T = 1

// e^(2 x / T) of half a distance x, per = 2 log2(e) / T in two floats: what rounding the exponent's argument loses goes into a first-order term, so that
// shares of any size are good to some 2^-22 of themselves.  (Below T = 2^-126 per would be infinite, and 0 times it NaN.)
struct Exponent {
    float per, rest;
    __device__ explicit Exponent(float T) {
        const double c = 2 * 1.4426950408889634 / fmax((double)T, 0x1p-126);
        per = (float)c;
        rest = (float)(c - (double)per);
    }
    __device__ __forceinline__ float fine(float x) const {
        const float y = x * per;
        return y > -INFINITY ? fast_exp2(y) * (1.f + kLn2 * (__builtin_fmaf(x, per, -y) + x * rest)) : 0.f;
    }
};

typedef u32x4 u32x4_any __attribute__((aligned(2)));         // rows may start at any element
typedef f32x4 f32x4_any __attribute__((aligned(4)));

// Vectors of 16 bytes of a row.
template <typename Z> struct Row;
template <> struct Row<float> {
    static constexpr int E = 4;
    static __device__ __forceinline__ float get(u32x4 v, int i) { return __uint_as_float(v[i]); }
    static __device__ __forceinline__ u32x4 make(const float (&x)[4]) { return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])}; }
    static __device__ __forceinline__ float one(const float *p) { return *p; }
    static __device__ __forceinline__ void put(float *p, float x) { *p = x; }
    static __device__ __forceinline__ u32x4 nothing() { return u32x4{0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u}; }
};
template <> struct Row<uint16_t> {
    static constexpr int E = 8;
    static __device__ __forceinline__ float get(u32x4 v, int i) { return __uint_as_float(i & 1 ? v[i >> 1] & 0xFFFF0000u : v[i >> 1] << 16); }
    static __device__ __forceinline__ u32x4 make(const float (&x)[8]) { return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])}; }
    static __device__ __forceinline__ float one(const uint16_t *p) { return bf16_to_f32(*p); }
    static __device__ __forceinline__ void put(uint16_t *p, float x) { *p = (uint16_t)pack_bf16x2(x, 0.f); }
    static __device__ __forceinline__ u32x4 nothing() { return u32x4{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u}; }
};

// The compiler takes this for another value: what it computed from the old one is not kept in registers for later (a row's differences
// from its maximum, twice the registers of a row in bfloat16, went to scratch memory).
__device__ __forceinline__ void forget(u32x4 &v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ int forget(int v) { asm volatile("" : "+v"(v)); return v; }

// Vector `i` of a row, or of a segment: p is the same in all lanes and i * 16 fits 32 bits (a row has at most 2^30 elements of 4 bytes),
// so that the address is one register.  Elements behind the last whole vector, fewer than E, are one for each of the first threads.
template <typename Z>
__device__ __forceinline__ u32x4 load_vector(const Z *p, int i) {
    return *reinterpret_cast<const u32x4_any *>(reinterpret_cast<const char *>(p) + (uint32_t)i * 16u);
}
template <typename Z>
__device__ __forceinline__ void store_vector(Z *p, int i, const float (&x)[Row<Z>::E]) {
    *reinterpret_cast<u32x4_any *>(reinterpret_cast<char *>(p) + (uint32_t)i * 16u) = Row<Z>::make(x);
}
template <typename Z>
__device__ __forceinline__ float load_tail(const Z *p, int n) {
    const int at = n / Row<Z>::E * Row<Z>::E + (int)threadIdx.x;
    return threadIdx.x < (unsigned)Row<Z>::E && at < n ? Row<Z>::one(p + at) : -INFINITY;
}
template <typename Z>
__device__ __forceinline__ void store_tail(Z *p, int n, float x) {
    const int at = n / Row<Z>::E * Row<Z>::E + (int)threadIdx.x;
    if (threadIdx.x < (unsigned)Row<Z>::E && at < n) Row<Z>::put(p + at, x);
}

// Sums (or maxima) of M values over the workgroup, in a fixed order; `part` is LDS scratch of M * waves floats, free again on return.
template <int M, bool MAX, int WAVES>
__device__ __forceinline__ void block_reduce(float (&v)[M], float *part) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < M; ++i) v[i] = MAX ? wave_max(v[i]) : wave_sum(v[i]);
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < M; ++i) part[i * WAVES + wave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < M; ++i) {
        float r = lane < WAVES ? part[i * WAVES + lane] : MAX ? -INFINITY : 0.f;
        v[i] = MAX ? wave_max(r) : wave_sum(r);
    }
    __syncthreads();
}

// The teacher's list of one row, in LDS.
struct List {
    int K;
    int *word;           // [K], -1: none
    float *q, *z;        // [K] the teacher's logit, then its share; the student's logit
    int *hash;           // [hash_mask + 1]
    int hash_mask;
    __device__ List(char *lds, int K, int hash_size) : K(K), hash_mask(hash_size - 1) {
        word = reinterpret_cast<int *>(lds);
        q = reinterpret_cast<float *>(word + K);
        z = q + K;
        hash = reinterpret_cast<int *>(z + K);
    }
    // Words and logits from memory; returns this thread's largest logit, +infinity where something is wrong with an entry.
    template <int THREADS>
    __device__ __forceinline__ float read(const DistillArgs &a, int n) {
        const int32_t *tw = a.teacher_word + (long long)n * K;
        const float *tl = a.teacher_logit + (long long)n * K;
        float top = -INFINITY;
        for (int i = threadIdx.x; i <= hash_mask; i += THREADS) hash[i] = -1;
        for (int k = threadIdx.x; k < K; k += THREADS) {
            const int w = tw[k];
            const float t = tl[k];
            word[k] = w;
            q[k] = t;
            if (w != -1) top = fmaxf(top, w < -1 || w >= a.V || t != t ? INFINITY : t);
        }
        return top;
    }
    // Puts this thread's words into the table; true where one is there already.
    template <int THREADS>
    __device__ __forceinline__ bool repeated() {
        bool again = false;
        for (int k = threadIdx.x; k < K; k += THREADS) {
            const int w = word[k];
            if (w < 0) continue;
            for (uint32_t at = ((uint32_t)w * 0x9E3779B1u >> 7) & hash_mask;; at = (at + 1) & hash_mask) {     // (half of it stays free)
                const int was = atomicCAS(&hash[at], -1, w);
                if (was == -1) break;
                if (was == w) { again = true; break; }
            }
        }
        return again;
    }
    // What the teacher gives to the word of entry k: its share, or where words repeat the sum of theirs, in the order of the list, at the
    // first of them; nothing (-1) at the others.
    __device__ __forceinline__ float share_of(int k, bool repeats) const {
        if (!repeats) return q[k];
        float sum = 0.f;
        for (int j = 0; j < K; ++j)
            if (word[j] == word[k]) {
                if (j < k) return -1.f;
                sum += q[j];
            }
        return sum;
    }
};

// What a share at the temperature weighs in the gradient: row weight times (1 - a), k, times T.  (The product of the weights alone may pass the range of
// a float.)
__device__ __forceinline__ float soft_weight(const DistillArgs &a, float k, float share) { return (float)((double)k * (double)a.T * (double)share); }

// The gradient of a row but for the teacher's words and the label.  TWO: shares at both temperatures, else those at one (`per`).
template <bool TWO>
struct RowGrad {
    float half_top, per, c, c_1;   // weights times 1 / sums
    bool dead, nothing;
    __device__ RowGrad(const DistillArgs &a, float per_T, float top, float inv_T, float inv_1, float k, float k_1, bool bad) : half_top(0.5f * top), per(per_T) {
        dead = bad || ((k != 0.f || k_1 != 0.f) && inv_T != inv_T);
        nothing = !dead && k == 0.f && k_1 == 0.f;
        c = dead ? quiet_nan() : k != 0.f ? soft_weight(a, k, inv_T) : 0.f;
        c_1 = !dead && k_1 != 0.f ? k_1 * inv_1 : 0.f;
        if (!TWO && k_1 != 0.f) { c += c_1; per = kPer1; }    // (both only at T = 1)
    }
    __device__ __forceinline__ float operator()(float z) const {
        const float d = half_distance(z, half_top);
        const float r = c * fast_exp2(d * per);
        return TWO ? __builtin_fmaf(c_1, fast_exp2(d * kPer1), r) : r;
    }
};

// The places of the teacher's words and of the label within [from, from + len) of the row, written over what is there.  `in_list`: the label
// is one of the words.  Called behind a barrier that awaited the stores.
template <typename Z, int THREADS, typename Grad>
__device__ __forceinline__ void write_listed(const DistillArgs &a, const List &list, const Grad &grad, Z *out, int from, int len, float k, float k_1, bool repeats,
                                             int label, float z_label) {
    bool mine = false;
    for (int i = threadIdx.x; k != 0.f && i < list.K; i += THREADS) {
        const int w = list.word[i];
        if (w < from || w >= from + len) continue;
        mine |= w == label;
        const float q = list.share_of(i, repeats);
        if (q >= 0.f) Row<Z>::put(out + w, grad(list.z[i]) - soft_weight(a, k, q) - (w == label ? k_1 : 0.f));
    }
    const bool in_list = __syncthreads_or(mine);
    if (threadIdx.x == 0 && !in_list && label >= from && label < from + len && k_1 != 0.f) Row<Z>::put(out + label, grad(z_label) - k_1);
}

// The soft part of a row's loss, (1 - a) T^2 sum q (log q - log p), is held in units of T^2, below T = 1 of 2 T: the sum grows as 1 / T, and T^2 passes
// the range of a float far in front of what their product is.
struct SoftUnits {
    float distance, log;           // of half a distance, and of a logarithm
    __device__ explicit SoftUnits(const DistillArgs &a)
        : distance(a.T < 1.f ? 1.f - a.a : 2.f * (1.f - a.a) / a.T), log(a.T < 1.f ? 0.5f * a.T * (1.f - a.a) : 1.f - a.a) {}
};
// Loss of a row: `soft` in those units; the label's -log p is log_sum less twice z_label, half its distance.
__device__ __forceinline__ float row_loss(const DistillArgs &a, bool bad, bool soft_part, bool hard_part, bool dead, float soft, float log_sum, float z_label) {
    if (bad || ((soft_part || hard_part) && dead)) return quiet_nan();
    float l = 0.f;
    if (soft_part) l = a.T < 1.f ? (2.f * a.T) * soft : a.T * (a.T * soft);
    if (hard_part) l += a.a * log_sum - 2.f * a.a * z_label;
    return l;
}

// Which exponentials a row takes.
enum Form {
    kOne,          // T = 1: the same for both parts
    kTwoSums,      // T != 1: sums at both temperatures for the statistics, a gradient at one (label_weight 0 or 1)
    kTwo           // T != 1, both parts
};

// One workgroup per row.
template <typename Z, int THREADS, int R, int STASH, bool GRAD, Form FORM>
__global__ __launch_bounds__(THREADS, 4) void distill_row_kernel(DistillArgs a, int hash_size) {
    constexpr int E = Row<Z>::E, WAVES = THREADS / 64;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float part[3 * WAVES];
    const int tid = threadIdx.x, n = blockIdx.x, V = a.V, vectors = V / E;
    const Z *row = static_cast<const Z *>(a.logits) + n * a.ld;
    const Exponent exponent(a.T);
    const float per = exponent.per;
    u32x4 *const stash = reinterpret_cast<u32x4 *>(lds);
    List list(lds + STASH * THREADS * 16, a.K, hash_size);
    const int label = a.label ? a.label[n] : -1;
    const float t_mine = list.read<THREADS>(a, n);
    // what stays in registers: vectors tid, tid + THREADS, ...
    u32x4 v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        v[r] = Row<Z>::nothing();
        if (r * THREADS + tid < vectors) v[r] = load_vector(row, r * THREADS + tid);
    }
    const float z_tail = load_tail(row, V);
    // This thread's maximum and its sums relative to it, so that exponentials are taken while other waves' vectors are on their way and
    // not behind the whole row's maximum.
    float mine = z_tail;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < E; ++j) mine = fmaxf(mine, Row<Z>::get(v[r], j));
    float from = mine == -INFINITY ? 0.f : 0.5f * mine;
    float at_T[E] = {}, at_1[E] = {};
    auto add = [&](u32x4 x) {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float d = half_distance(Row<Z>::get(x, j), from);
            at_T[j] += fast_exp2(d * per);
            if (FORM != kOne) at_1[j] += fast_exp2(d * kPer1);
        }
    };
#pragma unroll
    for (int r = 0; r < R; ++r) {
        forget(v[r]);
        add(v[r]);
    }
    at_T[0] += fast_exp2(half_distance(z_tail, from) * per);
    if (FORM != kOne) at_1[0] += fast_exp2(half_distance(z_tail, from) * kPer1);
    // What does not stay in registers, four vectors on their way at a time.  The first STASH of a thread stay in LDS.
    for (int f = 0; R * THREADS + f * THREADS < vectors; f += 4) {
        u32x4 x[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = (R + f + q) * THREADS + tid;
            x[q] = Row<Z>::nothing();
            if (i < vectors) x[q] = load_vector(row, i);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (GRAD && f + q < STASH) stash[(f + q) * THREADS + tid] = x[q];
            float high = mine;
#pragma unroll
            for (int j = 0; j < E; ++j) high = fmaxf(high, Row<Z>::get(x[q], j));
            if (high > mine) {
                const float d = half_distance(mine, 0.5f * high), by_T = fast_exp2(d * per), by_1 = fast_exp2(d * kPer1);
#pragma unroll
                for (int j = 0; j < E; ++j) { at_T[j] *= by_T; at_1[j] *= by_1; }
                mine = high;
                from = 0.5f * high;
            }
            add(x[q]);
        }
    }
    float m[2] = {t_mine, mine};
    block_reduce<2, true, WAVES>(m, part);                  // (also: the list is there)
    const float t_top = m[0], half_t_top = 0.5f * t_top, top = m[1], half_top = 0.5f * top;
    const bool bad = t_top == INFINITY || label < -1 || label >= V;
    const bool soft_part = t_top > -INFINITY && a.a < 1.f, hard_part = label >= 0 && a.a > 0.f;
    for (int k = tid; k < a.K; k += THREADS) {
        const int w = list.word[k];
        if (w >= 0 && !bad) list.z[k] = Row<Z>::one(row + w);
    }
    const float z_label = !bad && label >= 0 ? Row<Z>::one(row + label) : 0.f;
#pragma unroll
    for (int j = E / 2; j; j /= 2)
#pragma unroll
        for (int i = 0; i < j; ++i) { at_T[i] += at_T[i + j]; at_1[i] += at_1[i + j]; }
    // (a thread without a finite logit has sums of 0, or of NaN; the row's own maximum is infinite or there is nothing where `top` is)
    const float down = mine > -INFINITY ? half_distance(mine, half_top) : 0.f;
    float s[3] = {at_T[0] * fast_exp2(down * per), at_1[0] * fast_exp2(down * kPer1), 0.f};
    for (int k = tid; k < a.K; k += THREADS)
        if (list.word[k] >= 0) s[2] += exponent.fine(half_distance(list.q[k], half_t_top));
    block_reduce<3, false, WAVES>(s, part);
    const float s_T = s[0], s_1 = FORM == kOne ? s[0] : s[1], t_sum = s[2];
    const bool dead = !(s_T > 0.f);                         // a NaN, +infinity, or nothing finite
    const float inv_T = dead ? quiet_nan() : 1.f / s_T, inv_1 = dead ? quiet_nan() : 1.f / s_1;
    float l[1] = {0.f};
    if (soft_part && !bad) {
        const SoftUnits units(a);
        const float log_sum = logf(s_T), log_t = logf(t_sum);
        for (int k = tid; k < a.K; k += THREADS) {
            if (list.word[k] < 0) continue;
            const float d = half_distance(list.q[k], half_t_top), q = exponent.fine(d) / t_sum;
            if (q > 0.f) l[0] += q * ((d - half_distance(list.z[k], half_top)) * units.distance + (log_sum - log_t) * units.log);
            list.q[k] = q;
        }
    }
    block_reduce<1, false, WAVES>(l, part);
    if (tid == 0) {
        a.loss[n] = row_loss(a, bad, soft_part, hard_part, dead, l[0], logf(s_1), half_distance(z_label, half_top));
        *reinterpret_cast<f32x4_any *>(a.stats + 4ll * n) = f32x4{top, inv_T, inv_1, 0.f};
    }
    if (!GRAD) return;
    const float g = a.row_weight ? a.row_weight[n] : 1.f;
    const float k = soft_part ? g * (1.f - a.a) : 0.f, k_1 = hard_part ? g * a.a : 0.f;
    const RowGrad<FORM == kTwo> grad(a, per, top, inv_T, inv_1, k, k_1, bad);
    Z *out = static_cast<Z *>(a.grad) + n * a.grad_ld;
    const int at = forget(tid);
    if (grad.nothing) {                                   // nothing is learned from the row, whatever it holds
        const float zeros[E] = {};
        for (int i = tid; i < vectors; i += THREADS) store_vector(out, i, zeros);
        store_tail(out, V, 0.f);
        return;
    }
    // what is read again first, the last of it in front: that is still in the L2
    const int far_last = vectors > R * THREADS ? (vectors - R * THREADS - 1) / THREADS & ~3 : -1;
    for (int f = far_last; f >= 0; f -= 4) {
        u32x4 y[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = (R + f + q) * THREADS + tid;
            if (f + q < STASH) y[q] = stash[(f + q) * THREADS + tid];
            else if (i < vectors) y[q] = load_vector(row, i);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int i = (R + f + q) * THREADS + tid;
            float x[E];
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = grad(Row<Z>::get(y[q], j));
            if (i < vectors) store_vector(out, i, x);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        forget(v[r]);
        float x[E];
#pragma unroll
        for (int j = 0; j < E; ++j) x[j] = grad(Row<Z>::get(v[r], j));
        if (r * THREADS + at < vectors) store_vector(out, r * THREADS + at, x);
    }
    store_tail(out, V, grad(z_tail));
    if (grad.dead) return;
    const bool again = list.repeated<THREADS>();
    seen_by_all();
    const bool repeats = __syncthreads_or(again);
    write_listed<Z, THREADS>(a, list, grad, out, 0, V, k, k_1, repeats, label, z_label);
}

// ---- rows in segments
constexpr int kSegThreads = kDistillThreads, kSegWaves = kSegThreads / 64, kMaxSegments = 64;
// Of one segment: maximum m, sums relative to it at both temperatures, sum of q (z - m) / 2 and of q over the teacher's words in it, the label's
// (z - m) / 2.
struct Part { float m, s_T, s_1, qz, q, label, pad[2]; };

template <typename Z>
__global__ __launch_bounds__(kSegThreads) void distill_part_kernel(DistillArgs a, int segments, int seg_len, int hash_size) {
    constexpr int E = Row<Z>::E, WAVES = kSegWaves;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float part[5 * WAVES];
    const int tid = threadIdx.x, n = blockIdx.x / segments, from = blockIdx.x % segments * seg_len, len = min(seg_len, a.V - from);
    const Z *row = static_cast<const Z *>(a.logits) + n * a.ld;
    const Exponent exponent(a.T);
    const float per = exponent.per;
    List list(lds, a.K, hash_size);
    const int label = a.label ? a.label[n] : -1;
    float m[2] = {list.read<kSegThreads>(a, n), -INFINITY};
    const int vectors = len / E;
    const float z_tail = load_tail(row + from, len);
    m[1] = z_tail;
    for (int i = tid; i < vectors; i += kSegThreads) {
        const u32x4 x = load_vector(row + from, i);
#pragma unroll
        for (int j = 0; j < E; ++j) m[1] = fmaxf(m[1], Row<Z>::get(x, j));
    }
    block_reduce<2, true, WAVES>(m, part);
    const float t_top = m[0], half_t_top = 0.5f * t_top, top = m[1], half_top = 0.5f * top;
    const bool listed = t_top > -INFINITY && t_top < INFINITY;
    float at_T[E] = {}, at_1[E] = {};
    for (int i = tid; i < vectors; i += kSegThreads) {
        const u32x4 x = load_vector(row + from, i);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const float z = Row<Z>::get(x, j), d = z == -INFINITY ? -INFINITY : half_distance(z, half_top);     // (half_top may be -infinity itself here)
            at_T[j] += fast_exp2(d * per);
            at_1[j] += fast_exp2(d * kPer1);
        }
    }
#pragma unroll
    for (int j = E / 2; j; j /= 2)
#pragma unroll
        for (int i = 0; i < j; ++i) { at_T[i] += at_T[i + j]; at_1[i] += at_1[i + j]; }
    const float d_tail = z_tail == -INFINITY ? -INFINITY : half_distance(z_tail, half_top);
    float s[5] = {at_T[0] + fast_exp2(d_tail * per), at_1[0] + fast_exp2(d_tail * kPer1), 0.f, 0.f, 0.f};
    if (listed)
        for (int k = tid; k < a.K; k += kSegThreads)
            if (list.word[k] >= 0) s[2] += exponent.fine(half_distance(list.q[k], half_t_top));
    block_reduce<5, false, WAVES>(s, part);
    const float t_sum = s[2];
    float d[2] = {0.f, 0.f};
    if (listed)
        for (int k = tid; k < a.K; k += kSegThreads) {
            const int w = list.word[k];
            if (w < from || w >= from + len) continue;
            const float q = exponent.fine(half_distance(list.q[k], half_t_top)) / t_sum, z = Row<Z>::one(row + w);
            if (q > 0.f) { d[0] += q * (z == -INFINITY ? -INFINITY : half_distance(z, half_top)); d[1] += q; }
        }
    block_reduce<2, false, WAVES>(d, part);
    if (tid == 0) {
        Part p = {top, s[0], s[1], d[0], d[1], 0.f, {0.f, 0.f}};
        if (label >= from && label < from + len) { const float z = Row<Z>::one(row + label); p.label = z == -INFINITY ? -INFINITY : half_distance(z, half_top); }
        static_cast<Part *>(a.ws)[blockIdx.x] = p;
    }
}

// BACKWARD: statistics from memory, else from the segments' parts (then the row's first segment writes loss and statistics).
template <typename Z, bool BACKWARD, bool TWO>
__global__ __launch_bounds__(kSegThreads) void distill_segment_kernel(DistillArgs a, int parts, int part_len, int segments, int seg_len, int hash_size) {
    constexpr int E = Row<Z>::E, WAVES = kSegWaves, R = 4;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float part[2 * WAVES];
    const int tid = threadIdx.x, lane = tid & 63, n = blockIdx.x / segments, seg = blockIdx.x % segments, from = seg * seg_len, V = a.V;
    const int len = a.grad ? min(seg_len, V - from) : 0, vectors = len / E;
    const Z *row = static_cast<const Z *>(a.logits) + n * a.ld;
    const Exponent exponent(a.T);
    const float per = exponent.per;
    List list(lds, a.K, hash_size);
    const int label = a.label ? a.label[n] : -1;
    float m[1] = {list.read<kSegThreads>(a, n)};
    u32x4 first[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        first[r] = Row<Z>::nothing();
        if (r * kSegThreads + tid < vectors) first[r] = load_vector(row + from, r * kSegThreads + tid);
    }
    const float z_tail = load_tail(row + from, len);
    block_reduce<1, true, WAVES>(m, part);
    const float t_top = m[0];
    const bool bad = t_top == INFINITY || label < -1 || label >= V;
    const bool soft_part = t_top > -INFINITY && a.a < 1.f, hard_part = label >= 0 && a.a > 0.f;
    float s[1] = {0.f};
    for (int k = tid; k < a.K; k += kSegThreads) {
        const int w = list.word[k];
        if (w < 0 || bad) continue;
        s[0] += exponent.fine(half_distance(list.q[k], 0.5f * t_top));
        if (w >= from && w < from + len) list.z[k] = Row<Z>::one(row + w);
    }
    const float z_label = !bad && label >= from && label < from + len ? Row<Z>::one(row + label) : 0.f;
    block_reduce<1, false, WAVES>(s, part);
    const float t_sum = s[0];
    const SoftUnits units(a);
    float entropy[1] = {0.f};
    if (soft_part && !bad) {
        const float log_t = logf(t_sum);
        for (int k = tid; k < a.K; k += kSegThreads) {
            if (list.word[k] < 0) continue;
            const float d = half_distance(list.q[k], 0.5f * t_top), q = exponent.fine(d) / t_sum;
            if (q > 0.f) entropy[0] += q * (d * units.distance - log_t * units.log);
            list.q[k] = q;
        }
    }
    float top, inv_T, inv_1;
    if (BACKWARD) {
        top = a.stats[4ll * n];
        inv_T = a.stats[4ll * n + 1];
        inv_1 = a.stats[4ll * n + 2];
    } else {
        Part p = {-INFINITY, 0.f, 0.f, 0.f, 0.f, 0.f, {0.f, 0.f}};          // every wave joins them for itself
        if (lane < parts) p = static_cast<const Part *>(a.ws)[(long long)n * parts + lane];
        top = wave_max(p.m);
        const bool some = p.m > -INFINITY;
        const float d = half_distance(p.m, 0.5f * top);
        const float s_T = wave_sum(some ? p.s_T * fast_exp2(d * per) : p.s_T), s_1 = wave_sum(some ? p.s_1 * fast_exp2(d * kPer1) : p.s_1);
        const bool dead = !(s_T > 0.f) || top == INFINITY;
        inv_T = dead ? quiet_nan() : 1.f / s_T;
        inv_1 = dead ? quiet_nan() : 1.f / s_1;
        if (seg == 0) {
            block_reduce<1, false, WAVES>(entropy, part);
            const float qz = wave_sum(p.q > 0.f ? p.qz + p.q * d : 0.f), q = wave_sum(p.q);
            const float z_half = wave_sum(hard_part && !bad && label / part_len == lane ? p.label + (some ? d : 0.f) : 0.f);
            if (tid == 0) {
                a.loss[n] = row_loss(a, bad, soft_part, hard_part, dead, entropy[0] - qz * units.distance + q * (logf(s_T) * units.log), logf(s_1), z_half);
                *reinterpret_cast<f32x4_any *>(a.stats + 4ll * n) = f32x4{top, inv_T, inv_1, 0.f};
            }
        }
    }
    if (len == 0) return;
    const float g = a.row_weight ? a.row_weight[n] : 1.f;
    const float k = soft_part ? g * (1.f - a.a) : 0.f, k_1 = hard_part ? g * a.a : 0.f;
    const RowGrad<TWO> grad(a, per, top, inv_T, inv_1, k, k_1, bad);
    Z *out = static_cast<Z *>(a.grad) + n * a.grad_ld + from;
    if (grad.nothing) {
        const float zeros[E] = {};
        for (int i = tid; i < vectors; i += kSegThreads) store_vector(out, i, zeros);
        store_tail(out, len, 0.f);
        return;
    }
    __syncthreads();                                        // every place of the list that is in this segment has been read
    auto put = [&](int i, u32x4 y) {
        float x[E];
#pragma unroll
        for (int j = 0; j < E; ++j) x[j] = grad(Row<Z>::get(y, j));
        store_vector(out, i, x);
    };
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (r * kSegThreads + tid < vectors) put(r * kSegThreads + tid, first[r]);
    for (int i = R * kSegThreads + tid; i < vectors; i += kSegThreads) put(i, load_vector(row + from, i));
    store_tail(out, len, grad(z_tail));
    if (grad.dead) return;
    const bool again = list.repeated<kSegThreads>();
    seen_by_all();
    const bool repeats = __syncthreads_or(again);
    write_listed<Z, kSegThreads>(a, list, grad, out - from, from, len, k, k_1, repeats, label, z_label);
}

int hash_size_of(int K) {
    int h = 16;
    while (h < 2 * K) h <<= 1;
    return h;
}
size_t list_bytes(int K) { return (size_t)K * 12 + (size_t)hash_size_of(K) * 4; }

Form form_of(const DistillArgs &a) { return a.T == 1.f ? kOne : a.a > 0.f && a.a < 1.f ? kTwo : kTwoSums; }

template <typename Z, int THREADS, int R, int STASH, bool GRAD, Form FORM>
hipError_t launch_row_kernel(const DistillArgs &a, hipStream_t stream) {
    static LdsLimit limit;
    const size_t bytes = list_bytes(a.K) + (size_t)STASH * THREADS * 16;
    const auto kernel = distill_row_kernel<Z, THREADS, R, STASH, GRAD, FORM>;
    const hipError_t e = limit.ensure(reinterpret_cast<const void *>(kernel), bytes);
    if (e != hipSuccess) return e;
    kernel<<<a.N, THREADS, bytes, stream>>>(a, hash_size_of(a.K));
    return hipGetLastError();
}
template <typename Z, int THREADS, int R, int STASH>
hipError_t launch_steps(const DistillArgs &a, hipStream_t stream) {           // (loss and gradient)
    const Form form = form_of(a);
    if (form == kOne) return launch_row_kernel<Z, THREADS, R, STASH, true, kOne>(a, stream);
    return form == kTwo ? launch_row_kernel<Z, THREADS, R, STASH, true, kTwo>(a, stream) : launch_row_kernel<Z, THREADS, R, STASH, true, kTwoSums>(a, stream);
}
template <typename Z, int THREADS, int R>
hipError_t launch_rows(const DistillArgs &a, hipStream_t stream) {
    if (a.grad) return launch_steps<Z, THREADS, R, 0>(a, stream);
    return form_of(a) == kOne ? launch_row_kernel<Z, THREADS, R, 0, false, kOne>(a, stream) : launch_row_kernel<Z, THREADS, R, 0, false, kTwoSums>(a, stream);
}
template <typename Z, bool BACKWARD, bool TWO>
hipError_t launch_segments(const DistillArgs &a, int parts, int part_len, int segments, int seg_len, hipStream_t stream) {
    static LdsLimit limit;
    const size_t bytes = list_bytes(a.K);
    const auto kernel = distill_segment_kernel<Z, BACKWARD, TWO>;
    const hipError_t e = limit.ensure(reinterpret_cast<const void *>(kernel), bytes);
    if (e != hipSuccess) return e;
    kernel<<<(unsigned)a.N * segments, kSegThreads, bytes, stream>>>(a, parts, part_len, segments, seg_len, hash_size_of(a.K));
    return hipGetLastError();
}

// Rows too few to fill the chip by one workgroup each, and so long that one compute unit's way to memory (some 80 GB/s) takes longer than a
// second launch.  Steps, us, a workgroup a row / segments: fp32, V = 65536: 1 row 14.7 / 13.2, 16 rows 15.3 / 13.1, 64 rows 18.0 / 18.5, 100 rows
// 19.1 / 25.3; V = 200000: 100 rows 55.7 / 75.4; V = 20000: 8 rows 10.1 / 13.1, the loss alone 9.1 / 12.2.
constexpr int kFewRows = 48;
int segments_of(int N, int V, bool bf16) {
    if (N > kFewRows || (long long)V * (bf16 ? 2 : 4) < 192 * 1024) return 1;
    int s = 2 * kChipGroups / N;
    if (s > V / 4096) s = V / 4096;
    return s < 2 ? 1 : s > kMaxSegments ? kMaxSegments : s;
}

template <typename Z>
hipError_t forward(const DistillArgs &a, hipStream_t stream) {
    constexpr int E = Row<Z>::E;
    const int s = segments_of(a.N, a.V, a.bf16);
    if (s > 1) {
        static LdsLimit limit;
        const size_t bytes = list_bytes(a.K);
        const Cut cut = cut_row(a.V, E, s);
        const hipError_t e = limit.ensure(reinterpret_cast<const void *>(distill_part_kernel<Z>), bytes);
        if (e != hipSuccess) return e;
        distill_part_kernel<Z><<<a.N * cut.segments, kSegThreads, bytes, stream>>>(a, cut.segments, cut.len, hash_size_of(a.K));
        const int to_write = a.grad ? cut.segments : 1;
        return form_of(a) == kTwo ? launch_segments<Z, false, true>(a, cut.segments, cut.len, to_write, cut.len, stream)
                                  : launch_segments<Z, false, false>(a, cut.segments, cut.len, to_write, cut.len, stream);
    }
    const int vectors = (a.V + E - 1) / E;
    // The fewest waves that hold a row, for as many rows at once as the chip takes.  Us, this size / the next: 2000 rows of 1500 14.8 / 25.8, 2000 of 4000 18.1 /
    // 27.5, 200 of 4000 10.0 / 10.1; 500 of 16000 16.0 / 17.8, 2000 of 10000 40.2 / 50.7; 500 of 32000 29.2 / 37.2, 60 of 32000 11.6 / 13.8.
    if (vectors <= 256 * 4) return launch_rows<Z, 256, 4>(a, stream);
    if (vectors <= 512 * 8) return launch_rows<Z, 512, 8>(a, stream);
    if (vectors <= 512 * 16) return launch_rows<Z, 512, 16>(a, stream);
    if (vectors <= 1024 * 16 || !a.grad || list_bytes(a.K) > 28 * 1024) return launch_rows<Z, 1024, 16>(a, stream);
    return launch_steps<Z, 1024, E == 4 ? 20 : 16, 8>(a, stream);
}

template <typename Z>
hipError_t backward(const DistillArgs &a, hipStream_t stream) {
    const Cut cut = cut_for_backward(a.N, a.V, Row<Z>::E);
    return form_of(a) == kTwo ? launch_segments<Z, true, true>(a, 0, 1, cut.segments, cut.len, stream) : launch_segments<Z, true, false>(a, 0, 1, cut.segments, cut.len, stream);
}

}  // namespace

size_t distill_workspace_bytes(int N, int V) {
    const int s = segments_of(N, V, false);                 // (bfloat16 has no more)
    return s > 1 ? (size_t)N * s * sizeof(Part) : 16;
}
size_t distill_workspace_most(int N, int V) {               // (segments_of() does not fall with V)
    size_t most = 16;
    for (int n = 1; n <= N && n <= kFewRows; ++n) most = std::max(most, distill_workspace_bytes(n, V));
    return most;
}

hipError_t launch_distill(const DistillArgs &a, hipStream_t stream) { return a.bf16 ? forward<uint16_t>(a, stream) : forward<float>(a, stream); }
hipError_t launch_distill_backward(const DistillArgs &a, hipStream_t stream) { return a.bf16 ? backward<uint16_t>(a, stream) : backward<float>(a, stream); }

}  // namespace rnnlm
