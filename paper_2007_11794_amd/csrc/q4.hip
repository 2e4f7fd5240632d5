// Products with 4-bit weights: y[b][v] = bias[v] + sum_g scale[g][v] sum_{j in g} (code[v][j] - zero[g][v]) x[b][j].
//
// Few rows: the codes are read once, half a byte for every weight, and everything else has to keep out of their way.  A code less
// its zero is a small whole number, exact in fp16, so the matrix cores take it as it is, and the scale goes onto the fp32 sum of its
// group: no weight is ever rounded.  An fp32 x is two fp16 terms relative to its row's largest magnitude (two products instead of one), the second times
// 2^11, so that a unit next to one 2^28 times as large still has its 23 bits (relative to that one it is good to 2^-50; as the first term's last bits, 2^-39);
// a bf16 x is one.
//
// One wave takes 16 words by 16 * MT rows.  Its B operand (16x16x32: lane = word, 8 units) comes straight from memory: a
// lane loads 16 bytes, 32 consecutive codes of its word, the four lanes of a word 64 consecutive bytes; a transpose of 4 x 4 dwords over
// those four lanes (four register swaps) turns "32 units of one group per lane" into "the same group in all four lanes", so that a matrix
// instruction never mixes two groups, whatever their size.  The A operand, the rows, lies in LDS in operand order, staged once per workgroup.
//
// What bounds it: V = 1048576, H = 1024, 1 row in bf16 in 117 us is 4.8 TB/s, what a copy reaches; in fp32, whose rows take twice the LDS and leave a compute
// unit two workgroups of three, 158 us.  Shorter launches (V = 200000, H = 1024, 16 rows in bf16, zero points 37 us, 3.2 TB/s; V = 65536, H = 512, 1 row
// 9.2 us) are the way to the first products (launch, rows to LDS and their magnitudes, 4 us), and a last round of tiles that some waves have none of; a
// step costs a wave 75 to 120 vector instructions of four clocks for its 1 KB of codes, which memory takes some 460 clocks of the SIMD's for.  Two tiles a
// wave, sharing the reads of the rows' operands, had fewer waves in flight: 47.3 us for the first of these when one took 42.3.
#include "device_utils.h"
#include "ops.h"

namespace rnnlm {

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kStep = 128;                                   // units of a step: 16 bytes of codes a lane
constexpr size_t kLdsRows = 144 * 1024;                      // most LDS for the rows' operands
constexpr int kHeld = 4;                                     // eights of a thread that wait in registers while the rows' magnitudes are found

// Waves of a SIMD: six where their requests fit 80 registers, which is to say where there are few scales, no zero points, or rows of one term.  Us, four
// waves / six: V = 1000000, H = 256, groups of 128, 1 row 42.8 / 38.2; H = 100, groups of 32, 8 rows 34.3 / 31.8; V = 200000, H = 1024, groups of 64 with
// zero points, 16 rows in bf16 40.8 / 37.5, in fp32 45.4 / 57.4.
constexpr int waves_of(int TERMS, int MT, int G, bool zero) { return MT == 1 && (G == 128 || !zero || (G == 64 && TERMS == 1)) ? 6 : 4; }

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_any __attribute__((aligned(1)));         // rows of codes may start anywhere

typedef f32x4 f32x4_any __attribute__((aligned(4)));

// Elements k .. k + 7 of a row of H, 0 behind it, as they come from memory (so that several can be on their way).
template <bool BF16>
struct Eight {
    u32x4 w[BF16 ? 1 : 2] = {};
    __device__ __forceinline__ void load(const void *x, long long at, int k, int H) {
        if (BF16) {
            const uint16_t *p = static_cast<const uint16_t *>(x) + at + k;
            if (k + 8 <= H) w[0] = *reinterpret_cast<const u32x4_any *>(p);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) w[0][i >> 1] |= k + i < H ? (uint32_t)p[i] << (16 * (i & 1)) : 0;
        } else {
            const uint32_t *p = static_cast<const uint32_t *>(x) + at + k;
            if (k + 8 <= H) {
                w[0] = *reinterpret_cast<const u32x4_any *>(p);
                w[BF16 ? 0 : 1] = *reinterpret_cast<const u32x4_any *>(p + 4);
            } else
#pragma unroll
                for (int i = 0; i < 8; ++i) w[BF16 ? 0 : i >> 2][i & 3] = k + i < H ? p[i] : 0;
        }
    }
    __device__ __forceinline__ float operator[](int i) const {
        if (BF16) return __uint_as_float(i & 1 ? w[0][i >> 1] & 0xFFFF0000u : w[0][i >> 1] << 16);
        return __uint_as_float(w[BF16 ? 0 : i >> 2][i & 3]);
    }
    __device__ __forceinline__ uint32_t top(uint32_t t) const {            // the largest finite magnitude, and t
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t m = __float_as_uint((*this)[i]) & 0x7FFFFFFFu;
            if (m < 0x7F800000u && m > t) t = m;
        }
        return t;
    }
};

// What a wave needs of one step of a tile of 16 words, as it comes from memory.
template <int GROUPS, bool ZERO>
struct Codes {
    u32x4 w;
    uint32_t scale[GROUPS];              // of either type
    uint32_t zero[ZERO ? GROUPS : 1];
    float bias;                          // with the last step of a tile: a load behind the requests of later steps would have to wait for them
};

// (w & mask) | exponents in one instruction (of two literals it takes none, and the compiler makes two)
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t exponents) {
    uint32_t r;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(w), "s"(mask), "v"(exponents));
    return r;
}
// Eight codes of a dword less their zero, as fp16 in the order 0 4 1 5 2 6 3 7 (the rows are staged in that order too).  A code under
// the exponent of 1024 (of 64, four bits further up) is 1024 (64) more than itself; less1024 is -(1024 + zero), less64 -(64 + zero).
__device__ __forceinline__ f16x8 eight_codes(uint32_t w, f16x2 less1024, f16x2 less64) {
    f16x2 p[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t s = w >> (8 * i);
        p[2 * i] = __builtin_bit_cast(f16x2, and_or(s, 0x000F000Fu, 0x64006400u)) + less1024;
        p[2 * i + 1] = __builtin_bit_cast(f16x2, and_or(s, 0x00F000F0u, 0x54005400u)) + less64;
    }
    return f16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}

// dword i of the lanes 16 j + c goes to dword j of the lanes 16 i + c
__device__ __forceinline__ u32x4 transposed(u32x4 w) {
    auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return u32x4{c[0], c[1], d[0], d[1]};
}

// w without its first n bytes (the rest is of no account)
__device__ __forceinline__ u32x4 without(u32x4 w, uint32_t n) {
    const uint64_t lo = (uint64_t)w[1] << 32 | w[0], hi = (uint64_t)w[3] << 32 | w[2];
    const uint32_t bits = 8 * (n & 7);
    const uint64_t a = n & 8 ? hi : lo, b = n & 8 ? 0 : hi;
    const uint64_t x = n >= 16 ? 0 : bits ? a >> bits | b << (64 - bits) : a, y = n >= 16 ? 0 : b >> bits;
    return u32x4{(uint32_t)x, (uint32_t)(x >> 32), (uint32_t)y, (uint32_t)(y >> 32)};
}

template <int TERMS, int MT, int G, bool ZERO>
__global__ __launch_bounds__(kThreads, waves_of(TERMS, MT, G, ZERO)) void q4_kernel(Q4Args a, int chunk_steps, int rounds) {
    constexpr int kRows = 16 * MT, kGroups = kStep / G;
    // The second terms lie in LDS 2^11 times as large.  Where the registers of 16 rows allow their products have sums of their own, which take that factor off
    // where a group ends; else (forms of six waves a SIMD) the codes that they meet do, four instructions for 32 units.  Us, 1 row of V=65536 H=512, groups of 128:
    // 9.2 / 9.5; 16 rows of V=200000 H=1024, groups of 64 with zero points 45.4 / 46.3.  The same for any number of rows, so that a row's sums are.
    constexpr bool kApart = waves_of(TERMS, 1, G, ZERO) < 6 || (G == 128 && !ZERO);
    constexpr bool kFirst = G == 64;                                    // the first terms' product first: the order that 80 registers hold
    extern __shared__ __attribute__((aligned(1024))) char lds[];        // [units of a chunk / 32][MT][TERMS][64 lanes][8]
    __shared__ uint32_t row_top[kRows];                                 // the row's largest finite magnitude
    __shared__ int row_exp[kRows];                                      // the power of two that it is divided by
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const int r0 = blockIdx.y * kRows, rows = a.B - r0 < kRows ? a.B - r0 : kRows;
    const int steps = (a.H + kStep - 1) / kStep, last_group = (a.H + G - 1) / G - 1, stride = gridDim.x * kWaves;
    const int tiles = (a.V + 15) / 16, scale_size = a.scale_bf16 ? 2 : 4;
    const uint8_t *const end = a.codes + (long long)(a.V - 1) * a.code_ld + ((a.H + 1) >> 1), *const last = end - 16;

    // Tiles from here on may have loads that pass the end of the codes: a lane's last one ends up to 63 bytes behind its row.
    const int clear = (a.V - 64) / 16;
    // Requests run two steps ahead of the products, over the ends of tiles.
    int tile_r = blockIdx.x * kWaves + wave, step_r = 0;
    const uint8_t *word_r;
    uint32_t v_r;                                                       // a lane's word, in the array whatever the tile
    auto set_tile = [&]() {
        const int v = tile_r * 16 + c;
        v_r = (uint32_t)(v < a.V ? v : a.V - 1);
        word_r = a.codes + (long long)v_r * a.code_ld + 16 * g;
    };
    auto request = [&](Codes<kGroups, ZERO> &q) {
        if (tile_r < tiles) {
            const uint8_t *p = word_r + step_r * (kStep / 2);
            if (tile_r < clear) {                                       // behind a row come the next one's bytes, times zeros
                q.w = *reinterpret_cast<const u32x4_any *>(p);
            } else if (last >= a.codes) {                               // the codes end: from further in front, see below
                q.w = *reinterpret_cast<const u32x4_any *>(p > last ? last : p);
            } else {                                                    // less than 16 bytes of codes in all
                uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll 1
                for (int i = 0; i < 16 && p + i < end; ++i) {
                    const uint32_t byte = (uint32_t)p[i] << (8 * (i & 3));
#pragma unroll
                    for (int d = 0; d < 4; ++d) w[d] |= i >> 2 == d ? byte : 0;
                }
                q.w = u32x4{w[0], w[1], w[2], w[3]};
            }
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                const int grp = step_r * kGroups + i < last_group ? step_r * kGroups + i : last_group;
                const char *s = static_cast<const char *>(a.scale) + (long long)grp * a.V * scale_size;
                if (a.scale_bf16) q.scale[i] = *reinterpret_cast<const uint16_t *>(s + v_r * 2u);
                else q.scale[i] = *reinterpret_cast<const uint32_t *>(s + v_r * 4u);
                if (ZERO) q.zero[i] = (a.zero + (long long)grp * a.V)[v_r];
            }
            if (step_r + 1 == steps) q.bias = a.bias ? a.bias[v_r] : 0.f;
        }
        if (++step_r == steps) {
            step_r = 0;
            tile_r += stride;
            set_tile();
        }
    };

    set_tile();
    Codes<kGroups, ZERO> q[3];
    request(q[0]);
    request(q[1]);                                                      // on their way while the rows are staged

    // First unit of lane group g in product t of 32 units: as the codes are where a step is one group, else with the codes transposed.
    auto unit_of = [](int t, int g) { return G == kStep ? t / 4 * kStep + 32 * g + t % 4 * 8 : 32 * t + 8 * g; };
    // Eights of units in operand order; a thread's, kThreads apart, are of one row.
    const int my_row = wave % MT * 16 + c;
    auto load = [&](Eight<TERMS == 1> &x, int i, int k0, int n) {
        const int k = k0 + unit_of((i >> 6) / MT, g);
        if (i < n / 32 * MT * 64 && my_row < rows && k < a.H) x.load(a.x, (r0 + my_row) * a.x_ld, k, a.H);
    };
    auto put = [&](const Eight<TERMS == 1> &x, int i, int n, int e) {
        if (i >= n / 32 * MT * 64) return;
        const int frag = i >> 6;
        f16x8 t1, t2;
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const float y = ldexpf(x[(s >> 1) + 4 * (s & 1)], -e);
            t1[s] = (_Float16)y;
            t2[s] = (_Float16)(fabsf(y) < INFINITY ? 2048.f * (y - (float)t1[s]) : 0.f);       // (a NaN is in the first term)
        }
        *reinterpret_cast<f16x8 *>(lds + (size_t)frag * TERMS * 1024 + lane * 16) = t1;
        if (TERMS == 2) *reinterpret_cast<f16x8 *>(lds + (size_t)frag * 2048 + 1024 + lane * 16) = t2;
    };
    // The power of two of every row: its largest finite magnitude goes to [2^14, 2^15).  Rows that are kHeld eights a thread are requested at
    // once and stay in registers meanwhile; of longer ones each eight is read for the magnitude and again.  (Read twice, 1 row of V = 65536, H = 1024
    // took 16.0 us for 14.4, bf16 14.4 for 12.4.)
    const int units = steps * kStep, eights = units / 32 * MT * 64;
    const bool held = eights <= kHeld * kThreads && chunk_steps >= steps;
    Eight<TERMS == 1> x[kHeld];
    if (held)
#pragma unroll
        for (int j = 0; j < kHeld; ++j) load(x[j], tid + j * kThreads, 0, units);
    for (int r = tid; r < kRows; r += kThreads) row_top[r] = 0;
    __syncthreads();
    uint32_t top = 0;
    if (held) {
#pragma unroll
        for (int j = 0; j < kHeld; ++j) top = x[j].top(top);
    } else {
        for (int i = tid; i < eights; i += kThreads) {
            Eight<TERMS == 1> one;
            load(one, i, 0, units);
            top = one.top(top);
        }
    }
    atomicMax(&row_top[my_row], top);
    __syncthreads();
    auto exponent_of = [&](int r) { return row_top[r] ? ilogbf(__uint_as_float(row_top[r])) - 14 : 0; };
    for (int r = tid; r < kRows; r += kThreads) row_exp[r] = exponent_of(r);
    const int my_exp = exponent_of(my_row);
    if (held)
#pragma unroll
        for (int j = 0; j < kHeld; ++j) put(x[j], tid + j * kThreads, units, my_exp);
    __syncthreads();
    auto stage = [&](int k0, int n) {                                   // units k0 .. k0 + n - 1
        for (int i = tid; i < n / 32 * MT * 64; i += kThreads) {
            Eight<TERMS == 1> one;
            load(one, i, k0, n);
            put(one, i, n, my_exp);
        }
    };

    f32x4 acc[MT];
    int tile = blockIdx.x * kWaves + wave, step = 0, left = rounds * steps, in_chunk = 0;
    bool staged = held;
    auto body = [&](Codes<kGroups, ZERO> &now, Codes<kGroups, ZERO> &free) {
        if (in_chunk == 0 && !(staged && chunk_steps >= steps)) {       // (the same in all waves)
            if (staged) __syncthreads();                                // the chunk before has been read
            const int n = steps - step < chunk_steps ? steps - step : chunk_steps;
            stage(step * kStep, n * kStep);
            staged = true;
            __syncthreads();
        }
        request(free);
        if (tile < tiles) {
            if (step == 0)
#pragma unroll
                for (int m = 0; m < MT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
            const int v = tile * 16 + c;
            u32x4 w = now.w;
            if (tile >= clear) {                                        // loads that began too early
                const uint8_t *p = a.codes + (long long)(v < a.V ? v : a.V - 1) * a.code_ld + 16 * g + step * (kStep / 2);
                if (last >= a.codes && p > last) w = without(w, p - last < 16 ? (uint32_t)(p - last) : 16u);
            }
            if (G != kStep) w = transposed(w);
            f32x4 part[MT], rest[MT];
#pragma unroll
            for (int t = 0; t < 4; ++t) {                               // 32 units each
                constexpr int kPer = G / 32;
                const int grp = t / kPer;
                const uint32_t z = ZERO ? now.zero[grp] : 8u;
                const f16x2 less = __builtin_bit_cast(f16x2, 0xE400E400u | z * 0x00010001u);
                const f16x8 b = eight_codes(w[t], less, less + f16x2{(_Float16)960.f, (_Float16)960.f});
                const f16x8 b2 = kApart ? b : b * (_Float16)0x1p-11f;
                const float s = __uint_as_float(a.scale_bf16 ? now.scale[grp] << 16 : now.scale[grp]);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const char *at = lds + (size_t)((in_chunk * 4 + t) * MT + m) * TERMS * 1024 + lane * 16;
                    if (t % kPer == 0) part[m] = rest[m] = f32x4{0.f, 0.f, 0.f, 0.f};
                    f32x4 &to = kApart ? rest[m] : part[m];
                    if (TERMS == 2 && !kFirst) to = __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const f16x8 *>(at + 1024), b2, to, 0, 0, 0);
                    part[m] = __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const f16x8 *>(at), b, part[m], 0, 0, 0);
                    if (TERMS == 2 && kFirst) to = __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const f16x8 *>(at + 1024), b2, to, 0, 0, 0);
                    if (t % kPer == kPer - 1)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float sum = TERMS == 2 && kApart ? __builtin_fmaf(0x1p-11f, rest[m][i], part[m][i]) : part[m][i];
                            acc[m][i] = __builtin_fmaf(s, sum, acc[m][i]);
                        }
                }
            }
            if (step + 1 == steps && v < a.V)
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = m * 16 + 4 * g + i;
                        if (r >= rows) continue;
                        const float y = ldexpf(acc[m][i], row_exp[r]) + now.bias;
                        const long long at = (r0 + r) * a.y_ld + v;
                        if (a.y_bf16) static_cast<uint16_t *>(a.y)[at] = (uint16_t)pack_bf16x2(y, 0.f);
                        else static_cast<float *>(a.y)[at] = y;
                    }
        }
        if (++in_chunk == chunk_steps) in_chunk = 0;
        if (++step == steps) { step = in_chunk = 0; tile += stride; }
        // (the same in all lanes, which the compiler does not see)
        in_chunk = __builtin_amdgcn_readfirstlane(in_chunk);
        step = __builtin_amdgcn_readfirstlane(step);
        tile = __builtin_amdgcn_readfirstlane(tile);
    };
    while (true) {                                                      // the three sets of codes in turn, so that none is ever copied
        body(q[0], q[2]);
        if (--left == 0) break;
        body(q[1], q[0]);
        if (--left == 0) break;
        body(q[2], q[1]);
        if (--left == 0) break;
    }
}

template <int TERMS, int MT, int G, bool ZERO>
hipError_t launch(const Q4Args &a, hipStream_t stream) {
    static LdsLimit limit;
    const int steps = (a.H + kStep - 1) / kStep, step_bytes = 16 * MT * 2 * TERMS * kStep;
    int chunk = (int)(kLdsRows / step_bytes);
    if (chunk > steps) chunk = steps;
    const size_t bytes = (size_t)chunk * step_bytes;
    const auto kernel = q4_kernel<TERMS, MT, G, ZERO>;
    const hipError_t e = limit.ensure(reinterpret_cast<const void *>(kernel), bytes);
    if (e != hipSuccess) return e;
    const int row_blocks = (a.B + 16 * MT - 1) / (16 * MT), tiles = (a.V + 15) / 16, groups = (tiles + kWaves - 1) / kWaves;
    // workgroups of a compute unit: what its SIMDs' registers and its 160 KB of LDS hold
    const int by_lds = (int)(158 * 1024 / (bytes + 1024)), by_waves = waves_of(TERMS, MT, G, ZERO) * 4 / kWaves, resident = kChipGroups * (by_lds < 1 ? 1 : by_lds < by_waves ? by_lds : by_waves);
    for (int y0 = 0; y0 < row_blocks; y0 += 65535) {                    // (a grid has at most that many)
        const int ny = row_blocks - y0 < 65535 ? row_blocks - y0 : 65535;
        int gx = resident / ny;
        if (gx < 1) gx = 1;
        if (gx > groups) gx = groups;
        Q4Args b = a;
        const long long skip = (long long)y0 * 16 * MT;
        b.B = a.B - (int)skip;
        b.x = static_cast<const char *>(a.x) + skip * a.x_ld * (a.x_bf16 ? 2 : 4);
        b.y = static_cast<char *>(a.y) + skip * a.y_ld * (a.y_bf16 ? 2 : 4);
        kernel<<<dim3(gx, ny), kThreads, bytes, stream>>>(b, chunk, (tiles + gx * kWaves - 1) / (gx * kWaves));
    }
    return hipGetLastError();
}

template <int TERMS, int MT>
hipError_t by_group(const Q4Args &a, hipStream_t stream) {
    switch (a.group) {
        case 32: return a.zero ? launch<TERMS, MT, 32, true>(a, stream) : launch<TERMS, MT, 32, false>(a, stream);
        case 64: return a.zero ? launch<TERMS, MT, 64, true>(a, stream) : launch<TERMS, MT, 64, false>(a, stream);
        default: return a.zero ? launch<TERMS, MT, 128, true>(a, stream) : launch<TERMS, MT, 128, false>(a, stream);
    }
}
template <int TERMS>
hipError_t by_rows(const Q4Args &a, hipStream_t stream) {
    // Rows of a workgroup: 16 while all their tiles run at once (rows go to LDS by more workgroups), else 32; 64, whose operands need twice the
    // LDS, where every wave has several tiles and two such workgroups still share a compute unit's LDS and matrix cores (fp32 rows are two products
    // each).  Us, 16 / 32 / 64 rows, groups of 64 with zero points: 64 of V=2853 H=400 fp32 7.0 / 8.8 / 16.2; 40 of V=8000 H=1024 13.2 / 19.3 / 32.2; 64 of V=65536
    // H=512 25.4 / 21.4 / 30.1; 1024 of it 338 / 232 / 343; bf16: 64 of V=65536 H=512 21.7 / 17.0 / 19.8; 1024 of it 251 / 185 / 138; 512 of V=30000 H=512
    // 59.4 / 46.2 / 40.0; 64 of V=100000 H=1024 55.2 / 48.0 / 58.6.
    const long long tiles = (a.V + 15) / 16, at_once = 2 * kChipGroups * kWaves;
    if (a.B <= 16 || (a.B + 15) / 16 * tiles <= at_once) return by_group<TERMS, 1>(a, stream);
    if (a.B > 32 && TERMS * TERMS * a.H <= 512 && (a.B + 63) / 64 * tiles >= 2 * at_once) return by_group<TERMS, 4>(a, stream);
    return by_group<TERMS, 2>(a, stream);
}

}  // namespace

hipError_t launch_q4(const Q4Args &a, hipStream_t stream) { return a.x_bf16 ? by_rows<1>(a, stream) : by_rows<2>(a, stream); }

}  // namespace rnnlm
