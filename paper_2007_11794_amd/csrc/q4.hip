// Products with 4-bit weights: y[b][v] = bias[v] + sum_g scale[g][v] sum_{j in g} (code[v][j] - zero[g][v]) x[b][j].
//
// Few rows: the codes are read once, half a byte for every weight, and everything else has to keep out of their way.  A code less
// its zero is a small whole number, exact in fp16, so the matrix cores take it as it is, and the scale goes onto the fp32 sum of its
// group: no weight is ever rounded.  An fp32 x is two fp16 terms relative to its row's largest magnitude (two products instead of one), a
// bf16 x is one.
//
// One wave takes NT tiles of 16 words by 16 * MT rows.  Its B operand (16x16x32: lane = word, 8 units) comes straight from memory: a
// lane loads 16 bytes, 32 consecutive codes of its word, the four lanes of a word 64 consecutive bytes; a transpose of 4 x 4 dwords over
// those four lanes (four register swaps) turns "32 units of one group per lane" into "the same group in all four lanes", so that a matrix
// instruction never mixes two groups, whatever their size.  The A operand, the rows, lies in LDS in operand order, staged once per workgroup.
#include "device_utils.h"
#include "ops.h"

namespace rnnlm {

namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kStep = 128;                                   // units of a step: 16 bytes of codes a lane
constexpr size_t kLdsRows = 144 * 1024;                      // most LDS for the rows' operands

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_any __attribute__((aligned(1)));         // rows of codes may start anywhere

__device__ __forceinline__ float row_element(const void *x, long long i, bool bf16) {
    return bf16 ? bf16_to_f32(static_cast<const uint16_t *>(x)[i]) : static_cast<const float *>(x)[i];
}

// What a wave needs of one step of one tile of 16 words.
template <int GROUPS>
struct Codes {
    u32x4 w;
    uint32_t scale[GROUPS], zero[GROUPS];
};

// Eight codes of a dword less their zero, as fp16 in the order 0 4 1 5 2 6 3 7 (the rows are staged in that order too).  A code under
// the exponent of 1024 (of 64, four bits further up) is 1024 (64) more than itself; less1024 is -(1024 + zero), less64 -(64 + zero).
__device__ __forceinline__ f16x8 eight_codes(uint32_t w, f16x2 less1024, f16x2 less64) {
    f16x2 p[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t s = w >> (8 * i);
        p[2 * i] = __builtin_bit_cast(f16x2, (s & 0x000F000Fu) | 0x64006400u) + less1024;
        p[2 * i + 1] = __builtin_bit_cast(f16x2, (s & 0x00F000F0u) | 0x54005400u) + less64;
    }
    return f16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}

// dword i of the lanes 16 j + c goes to dword j of the lanes 16 i + c
__device__ __forceinline__ void transpose4(u32x4 &w) {
    auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    w = u32x4{c[0], c[1], d[0], d[1]};
}

template <int TERMS, int MT, int NT, int G, bool ZERO>
__global__ __launch_bounds__(kThreads, 4) void q4_kernel(Q4Args a, int chunk, int rounds) {
    constexpr int kRows = 16 * MT, kGroups = kStep / G;
    extern __shared__ __attribute__((aligned(1024))) char lds[];        // [chunk / 32][MT][TERMS][64 lanes][8]
    __shared__ int row_exp[kRows];                                      // power of two that the row was divided by
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const int r0 = blockIdx.y * kRows, rows = a.B - r0 < kRows ? a.B - r0 : kRows;
    const int row_bytes = (a.H + 1) >> 1, Hp = (a.H + kStep - 1) / kStep * kStep, last_group = (a.H + G - 1) / G - 1;
    const uint8_t *const end = a.codes + (long long)(a.V - 1) * a.code_ld + row_bytes;

    auto request = [&](int tile, int step, Codes<kGroups> (&q)[NT]) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            int v = (tile * NT + n) * 16 + c;
            if (v >= a.V) v = a.V - 1;
            const int off = step * (kStep / 2) + 16 * g;
            const uint8_t *p = a.codes + v * a.code_ld + off;
            q[n].w = u32x4{0, 0, 0, 0};
            if (off < row_bytes) {                                      // behind a row come the next one's bytes, times zeros
                if (p + 16 <= end) q[n].w = *reinterpret_cast<const u32x4_any *>(p);
                else
                    for (int i = 0; i < 16; ++i)
                        if (p + i < end) q[n].w[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
            }
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                int grp = step * kGroups + i;
                if (grp > last_group) grp = last_group;
                const long long at = (long long)grp * a.V + v;
                q[n].scale[i] = a.scale_bf16 ? (uint32_t)static_cast<const uint16_t *>(a.scale)[at] << 16 : static_cast<const uint32_t *>(a.scale)[at];
                q[n].zero[i] = ZERO ? a.zero[at] : 0;
            }
        }
    };

    const int tiles = (a.V + 16 * NT - 1) / (16 * NT);
    int tile = blockIdx.x * kWaves + wave;
    Codes<kGroups> q[NT];
    if (tile < tiles) request(tile, 0, q);                              // on their way while the rows are staged

    // the power of two of every row: its largest finite magnitude goes to [2^14, 2^15)
    for (int r = wave; r < kRows; r += kWaves) {
        float top = 0.f;
        if (r < rows)
            for (int j = lane; j < a.H; j += 64) {
                const float m = fabsf(row_element(a.x, (r0 + r) * a.x_ld + j, a.x_bf16));
                if (m < INFINITY) top = fmaxf(top, m);
            }
        top = wave_max(top);
        if (lane == 0) row_exp[r] = top > 0.f ? ilogbf(top) - 14 : 0;
    }
    __syncthreads();
    auto stage = [&](int k0, int n) {                                   // units k0 .. k0 + n - 1
        for (int i = tid; i < n / 32 * MT * 64; i += kThreads) {
            const int frag = i >> 6, l = i & 63, r = (frag % MT) * 16 + (l & 15), k = k0 + frag / MT * 32 + (l >> 4) * 8, e = row_exp[r];
            f16x8 t1, t2;
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const int j = k + (s >> 1) + 4 * (s & 1);
                const float x = r < rows && j < a.H ? ldexpf(row_element(a.x, (r0 + r) * a.x_ld + j, a.x_bf16), -e) : 0.f;
                t1[s] = (_Float16)x;
                t2[s] = (_Float16)(fabsf(x) < INFINITY ? x - (float)t1[s] : 0.f);       // (a NaN is in the first term)
            }
            *reinterpret_cast<f16x8 *>(lds + (size_t)frag * TERMS * 1024 + l * 16) = t1;
            if (TERMS == 2) *reinterpret_cast<f16x8 *>(lds + (size_t)frag * 2048 + 1024 + l * 16) = t2;
        }
    };

    for (int round = 0; round < rounds; ++round, tile += gridDim.x * kWaves) {
        f32x4 acc[MT][NT];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int k0 = 0; k0 < Hp; k0 += chunk) {
            const int now = Hp - k0 < chunk ? Hp - k0 : chunk;
            if (round == 0 || chunk < Hp) {
                if (round || k0) __syncthreads();                       // the chunk before has been read
                stage(k0, now);
                __syncthreads();
            }
            if (tile >= tiles) continue;
            for (int k = 0; k < now; k += kStep) {
                Codes<kGroups> cur[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) cur[n] = q[n];
                const bool row_ends = k0 + k + kStep >= Hp;
                const int next = row_ends ? tile + (int)gridDim.x * kWaves : tile;
                if (next < tiles) request(next, row_ends ? 0 : (k0 + k) / kStep + 1, q);
                f32x4 part[MT][NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) transpose4(cur[n].w);
#pragma unroll
                for (int t = 0; t < 4; ++t) {                           // 32 units each
                    const int grp = t * 32 / G;
                    f16x8 b[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint32_t z = ZERO ? cur[n].zero[grp] : 8u;
                        const f16x2 less = __builtin_bit_cast(f16x2, 0xE400E400u | z * 0x00010001u);
                        b[n] = eight_codes(cur[n].w[t], less, less + f16x2{(_Float16)960.f, (_Float16)960.f});
                    }
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const char *at = lds + (size_t)((k / 32 + t) * MT + m) * TERMS * 1024 + lane * 16;
                        const f16x8 x1 = *reinterpret_cast<const f16x8 *>(at);
                        f16x8 x2;
                        if (TERMS == 2) x2 = *reinterpret_cast<const f16x8 *>(at + 1024);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            if (t * 32 % G == 0) part[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
                            if (TERMS == 2) part[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x2, b[n], part[m][n], 0, 0, 0);
                            part[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x1, b[n], part[m][n], 0, 0, 0);
                            if ((t + 1) * 32 % G == 0) {
                                const float s = __uint_as_float(cur[n].scale[grp]);
#pragma unroll
                                for (int i = 0; i < 4; ++i) acc[m][n][i] = __builtin_fmaf(s, part[m][n][i], acc[m][n][i]);
                            }
                        }
                    }
                }
            }
        }
        if (tile >= tiles) continue;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int v = (tile * NT + n) * 16 + c;
            if (v >= a.V) continue;
            const float bias = a.bias ? a.bias[v] : 0.f;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = m * 16 + 4 * g + i;
                    if (r >= rows) continue;
                    const float y = ldexpf(acc[m][n][i], row_exp[r]) + bias;
                    const long long at = (r0 + r) * a.y_ld + v;
                    if (a.y_bf16) static_cast<uint16_t *>(a.y)[at] = (uint16_t)pack_bf16x2(y, 0.f);
                    else static_cast<float *>(a.y)[at] = y;
                }
        }
    }
}

template <int TERMS, int MT, int NT, int G, bool ZERO>
hipError_t launch(const Q4Args &a, hipStream_t stream) {
    static LdsLimit limit;
    const int Hp = (a.H + kStep - 1) / kStep * kStep, unit = 16 * MT * 2 * TERMS;          // bytes of LDS per unit
    int chunk = (int)(kLdsRows / unit) / kStep * kStep;
    if (chunk > Hp) chunk = Hp;
    const size_t bytes = (size_t)chunk * unit;
    const auto kernel = q4_kernel<TERMS, MT, NT, G, ZERO>;
    const hipError_t e = limit.ensure(reinterpret_cast<const void *>(kernel), bytes);
    if (e != hipSuccess) return e;
    const int row_blocks = (a.B + 16 * MT - 1) / (16 * MT), tiles = (a.V + 16 * NT - 1) / (16 * NT), groups = (tiles + kWaves - 1) / kWaves;
    const int resident = kChipGroups * (bytes > 72 * 1024 ? 1 : 2);
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

template <int TERMS, int MT, int NT>
hipError_t by_group(const Q4Args &a, hipStream_t stream) {
    switch (a.group) {
        case 32: return a.zero ? launch<TERMS, MT, NT, 32, true>(a, stream) : launch<TERMS, MT, NT, 32, false>(a, stream);
        case 64: return a.zero ? launch<TERMS, MT, NT, 64, true>(a, stream) : launch<TERMS, MT, NT, 64, false>(a, stream);
        default: return a.zero ? launch<TERMS, MT, NT, 128, true>(a, stream) : launch<TERMS, MT, NT, 128, false>(a, stream);
    }
}

template <int TERMS>
hipError_t by_rows(const Q4Args &a, hipStream_t stream) {
    // Tiles of 16 words where pairs of them would leave waves without any.
    const bool few_words = a.V < 32 * kWaves * kChipGroups;
    if (a.B <= 16) return few_words ? by_group<TERMS, 1, 1>(a, stream) : by_group<TERMS, 1, 2>(a, stream);
    if (a.B <= 32) return few_words ? by_group<TERMS, 2, 1>(a, stream) : by_group<TERMS, 2, 2>(a, stream);
    return few_words ? by_group<TERMS, 4, 1>(a, stream) : by_group<TERMS, 4, 2>(a, stream);
}

}  // namespace

hipError_t launch_q4(const Q4Args &a, hipStream_t stream) { return a.x_bf16 ? by_rows<1>(a, stream) : by_rows<2>(a, stream); }

}  // namespace rnnlm
