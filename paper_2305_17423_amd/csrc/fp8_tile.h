// Products of 8-bit rows with 8-bit weights on tiles: what fp8.hip and experts.hip share.  Internal.
//
// A block of 128 columns is one 16x16x128 matrix instruction, so the sum of a block's products comes out of it by itself and goes to the float accumulators times its two
// scales: one multiply-add for each value of a result, beside the matrix unit.  The weights' rows are the first index of the product: a lane has one token (its scale is
// the lane's) and four neighbouring outputs.
// The 8-bit instruction adds its products eight at a time and drops of each what is below 2^-13 of the largest of the eight (measured: eight of 2^14 and 2^1 add up exactly, those of 2^0
// are gone); 16x16x32, of half its rate, does the same.  That is up to 2^-10 of the magnitudes' sum, next to 2^-8 of a bf16 result, so bf16 results and the second product of experts of many rows take it; float results
// and the experts' other products (EXACT) are made of the same codes as bf16, whose instruction keeps all of a product, at half the rate.
// 8192 x 8192 x 8192, rows in 8 bits: 461 - 490 us by the card, 2.2 - 2.4 PFLOP/s (a library's product with one scale a matrix: 414), matrix units busy 56 % of the time.  Steps on the way there, us: products added up
// where they were made and the next block's loads waited for, 770; scales loaded a block ahead, 608; products added up two behind, 516; pieces without bank conflicts, 499; loads between the products, 470.
#pragma once
#include "common.h"
#include "latent.h"

namespace fise {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 fp8_bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int FP8_BLOCK = 128;                      // columns of a scale, bytes of a row in a tile

// exponent of the smallest power of two, 2^-126 at least, that leaves a magnitude (its bits; finite) at most 448 = 1.75 * 2^8
__device__ __forceinline__ int fp8_exponent(unsigned bits) {
    return max((int)(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u), -126);
}
__device__ __forceinline__ float fp8_power(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }
// The largest magnitude of N values (its bits); what is not finite does not count.  (NaN drops out of a maximum by itself, an infinity is looked for once.)
template <int N> __device__ __forceinline__ unsigned fp8_largest(const float* v) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) m = fmaxf(m, fabsf(v[i]));
    if (m > 3.402823466e38f) {
        m = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) m = fabsf(v[i]) <= 3.402823466e38f ? fmaxf(m, fabsf(v[i])) : m;
    }
    return __float_as_uint(m);
}
// the largest of such numbers over the LANES (4, 8 or 16) neighbouring lanes of a block of lanes
template <int LANES> __device__ __forceinline__ unsigned fp8_over(unsigned v) {
    int m = (int)v;                                                    // (not negative)
    m = max(m, __builtin_amdgcn_update_dpp(0, m, 0xb1, 0xf, 0xf, false));      // lane ^ 1
    m = max(m, __builtin_amdgcn_update_dpp(0, m, 0x4e, 0xf, 0xf, false));      // lane ^ 2
    if constexpr (LANES >= 8) m = max(m, __builtin_amdgcn_update_dpp(0, m, 0x141, 0xf, 0xf, false));      // eight lanes mirrored
    if constexpr (LANES >= 16) m = max(m, __builtin_amdgcn_update_dpp(0, m, 0x140, 0xf, 0xf, false));     // sixteen
    return (unsigned)m;
}
// Four values times `inverse`, a power of two that brings what is finite to 448 at most, as codes: rounded to the nearest, ties to even; the conversion makes NaN of what is beyond (there is no infinity).
__device__ __forceinline__ unsigned fp8_codes(float a, float b, float c, float d, float inverse) {
    int w = 0;
    w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, w, true);
    return (unsigned)w;
}
__device__ __forceinline__ float fp8_inverse(int e) { return fp8_power(-e); }      // (e is between -126 and 120, of values beyond 1.75 * 2^127: 2^-120 is a normal number)

__device__ __forceinline__ void fp8_load8(const float* p, float* v) {
    const f32x4_t a = *reinterpret_cast<const f32x4_t*>(p), b = *reinterpret_cast<const f32x4_t*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
__device__ __forceinline__ void fp8_load8(const bf16_t* p, float* v) {
    const u32x4_t a = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = lo16(a[i]); v[2 * i + 1] = hi16(a[i]); }
}

// What a tile kernel works on.  Rows of x are codes padded with zeros to whole blocks where the library made them.
enum { FP8_LINEAR = 0,      // y[m, n] of rows 0..M-1
       FP8_GATED = 1,       // rows of pairs, gate and up: silu(gate) * up in 8 bits again
       FP8_PAIRS = 2 };     // rows of those, in the same order
struct Fp8TileArgs {
    const unsigned char* x; long long x_stride; long long x_bytes;     // rows of codes (GATED: of tokens, in one buffer of x_bytes)
    const float* x_scale; long long x_scale_stride;                    // [block][row]
    const unsigned char* w; long long w_stride, w_expert;              // an expert's weights apart
    const float* w_scale; int w_scale_expert;
    int M, N, K;                                                       // N: rows of the weights (GATED: of the gate)
    int m_tiles, n_tiles;
    const void* bias; int bias_f32; const void* residual; long long residual_stride;
    void* y; long long y_stride; int y_f32;
    // experts
    const int* table; int pairs, k;                                    // a tile's first row, and its expert << 16 | rows
    const int* slots;
    unsigned char* h; long long h_stride; float* h_scale; long long h_scale_stride;
    unsigned char* row_exp;                                            // PAIRS that are not float: 16-bit floats times 2^(this - 127), for 64 outputs of a pair (32 where a wave has no more)
};
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ f32x4_t fp8_mfma(i32x8_t a, i32x8_t b) {
    const f32x4_t z = {0.f, 0.f, 0.f, 0.f};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, z, 0, 0, 0, 0, 0, 0);      // (no scales: the plain instruction)
}
// Sixteen bytes a lane to LDS as la_to_lds, `at` bytes (the same for all lanes) behind `off`.  `off` alone is held against the buffer's size: it is that of a row that is there, in which `at` stays.
__device__ __forceinline__ void fp8_to_lds(u32x4_t from, unsigned off, unsigned at, unsigned to) {
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(off), "s"(from), "s"(at), "s"(to) : "memory");
}
// A lane's 32 codes of a row; EXACT: as bf16, which holds every code.
template <bool EXACT> struct Fp8Operand;
template <> struct Fp8Operand<false> {
    i32x8_t v;
    __device__ __forceinline__ void ld(const unsigned char* row, int at0, int at1) {
        const i32x4_t lo = *reinterpret_cast<const i32x4_t*>(row + at0), hi = *reinterpret_cast<const i32x4_t*>(row + at1);
        of(lo, hi);
    }
    __device__ __forceinline__ void of(i32x4_t lo, i32x4_t hi) { v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); }
};
template <> struct Fp8Operand<true> {
    bf16x8_t v[4];
    __device__ __forceinline__ void ld(const unsigned char* row, int at0, int at1) { of(*reinterpret_cast<const i32x4_t*>(row + at0), *reinterpret_cast<const i32x4_t*>(row + at1)); }
    __device__ __forceinline__ void of(i32x4_t lo, i32x4_t hi) {
        const i32x4_t c[2] = {lo, hi};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            u32x4_t w;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int four = c[j >> 1][(j & 1) * 2 + i];
                w[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, 1.f, false));
                w[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, 1.f, true));
            }
            v[j] = __builtin_bit_cast(bf16x8_t, w);
        }
    }
};
__device__ __forceinline__ f32x4_t fp8_product(const Fp8Operand<false>& a, const Fp8Operand<false>& b) { return fp8_mfma(a.v, b.v); }
__device__ __forceinline__ f32x4_t fp8_product(const Fp8Operand<true>& a, const Fp8Operand<true>& b) {
    f32x4_t p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(fp8_bf16x8_t, a.v[j]), __builtin_bit_cast(fp8_bf16x8_t, b.v[j]), p, 0, 0, 0);
    return p;
}
__device__ __forceinline__ float fp8_value(const void* p, int f32, long long at) {
    return f32 ? reinterpret_cast<const float*>(p)[at] : bf2f(reinterpret_cast<const bf16_t*>(p)[at]);
}
#endif

// WN x WM waves, each with NF x MF pieces of 16 outputs x 16 tokens.  Two stages of LDS: the loads of the next block of columns run under the products of this one.  Rows of 128
// bytes lie with their pieces of 16 bytes at piece ^ (row / 2 & 7), and a lane reads the pieces lane / 16 and lane / 16 + 4: no bank is met twice (pieces 2 (lane / 16) and the next: a third of
// the LDS' time was conflicts).
template <int NF, int MF, int WN, int WM, int KIND, bool EXACT>
__global__ __launch_bounds__(64 * WN * WM) void fp8_tile_kernel(Fp8TileArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int WAVES = WN * WM, BN = NF * WN * 16, BM = MF * WM * 16, STAGE = (BN + BM) * FP8_BLOCK, LN = BN / 8 / WAVES, LM = BM / 8 / WAVES;
    static_assert(BN / 8 % WAVES == 0 && BM / 8 % WAVES == 0, "whole loads a wave");
    static_assert(KIND != FP8_GATED || (BN == 256 && NF % 2 == 0), "gate and up of one block of 128");
    extern __shared__ __align__(16) unsigned char fp8_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wn = wave / WM, wm = wave % WM;
    // workgroup w runs on XCD w mod 8, which gets a run of tiles: bands of a few tiles of tokens, all outputs of a band before the next, so that the tiles at work in an
    // XCD share rows of both sides in its L2 (8192 x 8192 x 8192, bands of 4, 6, 8: 469, 461, 470 us; 131072 pairs of 64 experts, where a band's tiles may be of two of them, both products on 256 rows, 3, 6, 12: 3.27, 3.33, 3.37 ms)
    int w = blockIdx.x;
    { const int chunk = gridDim.x >> 3; if (w < chunk << 3) w = (w & 7) * chunk + (w >> 3); }
    constexpr int BAND = KIND == FP8_LINEAR ? 6 : 3;
    const int band = w / (BAND * a.n_tiles), in = w - band * BAND * a.n_tiles, high = min(BAND, a.m_tiles - band * BAND), nt = in / high, mt = band * BAND + in - nt * high;
    int m0 = mt * BM, rows = min(BM, a.M - m0), expert = 0;
    if constexpr (KIND != FP8_LINEAR) {
        const int first = a.table[2 * mt], info = a.table[2 * mt + 1];
        m0 = __builtin_amdgcn_readfirstlane(first);
        rows = __builtin_amdgcn_readfirstlane(info) & 0xffff;
        expert = __builtin_amdgcn_readfirstlane(info) >> 16;
        if (rows == 0) return;
    }
    constexpr int TILE_N = KIND == FP8_GATED ? BN / 2 : BN;            // outputs, of gate and of up
    const int n0 = nt * TILE_N, n_rows = min(TILE_N, a.N - n0);
    const unsigned char* const wt = a.w + expert * a.w_expert;
    const auto w_bytes = (int)((n_rows - 1) * a.w_stride + a.K);
    const u32x4_t from_w = la_buffer(wt + n0 * a.w_stride, w_bytes);
    const u32x4_t from_up = la_buffer(wt + (KIND == FP8_GATED ? (long long)a.N + n0 : (long long)n0) * a.w_stride, w_bytes);
    const u32x4_t from_x = KIND == FP8_GATED ? la_buffer(a.x, (int)a.x_bytes) : la_buffer(a.x + m0 * a.x_stride, (int)((rows - 1) * a.x_stride + (KIND == FP8_LINEAR ? a.K : a.x_stride)));
    constexpr unsigned OOB = 0x80000000u;
    unsigned off_w[LN], off_x[LM];
    static_assert(WAVES % 2 == 0, "loads of a wave start at rows that are alike modulo 16");
    const int piece = (lane & 7) ^ (((wave & 1) * 4 + (lane >> 4)) & 7);      // of its row that a lane loads
#pragma unroll
    for (int j = 0; j < LN; ++j) {
        const int instr = j * WAVES + wave, row = instr * 8 + (lane >> 3), r = KIND == FP8_GATED ? row % TILE_N : row;
        off_w[j] = r < n_rows ? (unsigned)(r * (int)a.w_stride + piece * 16) : OOB;
    }
#pragma unroll
    for (int j = 0; j < LM; ++j) {
        const int instr = j * WAVES + wave, row = instr * 8 + (lane >> 3);
        unsigned off = OOB;
        if (row < rows) {
            if constexpr (KIND == FP8_GATED) {
                const unsigned p = (unsigned)a.slots[m0 + row];
                if (p < (unsigned)a.pairs) off = (p / (unsigned)a.k) * (unsigned)a.x_stride + piece * 16;
            } else off = (unsigned)(row * (int)a.x_stride + piece * 16);
        }
        off_x[j] = off;
    }
    const int blocks = (a.K + FP8_BLOCK - 1) / FP8_BLOCK;
    // load i of block s (a wave has LN of weights, then LM of tokens); columns past K are zeros on both sides (there is no telling what lies behind a row), and so are blocks past the last
    auto load = [&](int s, bool in, int i) {
        const unsigned to = (unsigned)((s & 1) * STAGE), at = (unsigned)(s * FP8_BLOCK);
        if (i < LN) {
            const int instr = i * WAVES + wave;
            fp8_to_lds(KIND == FP8_GATED && i >= LN / 2 ? from_up : from_w, in ? off_w[i] : OOB, at, to + (unsigned)instr * 1024u);
        } else {
            const int instr = (i - LN) * WAVES + wave;
            fp8_to_lds(from_x, in ? off_x[i - LN] : OOB, at, to + (unsigned)(BN * FP8_BLOCK + instr * 1024));
        }
    };
    auto inside = [&](int s) { return s * FP8_BLOCK + piece * 16 < a.K; };
    // a lane's token of each piece, and where its scales are
    const int l16 = lane & 15, lq = lane >> 4;
    long long scale_at[MF];
#pragma unroll
    for (int b = 0; b < MF; ++b) {
        const int row = wm * MF * 16 + b * 16 + l16;
        long long at = 0;
        if (row < rows) {
            at = m0 + row;
            if constexpr (KIND == FP8_GATED) {
                const unsigned p = (unsigned)a.slots[m0 + row];
                at = p < (unsigned)a.pairs ? p / (unsigned)a.k : 0;
            }
        }
        scale_at[b] = at;                                              // (of rows that are not there: a scale that is, times zeros)
    }
    // a wave's outputs lie in one block of the weights' scales (gate and up in one each)
    const int n_block = KIND == FP8_GATED ? n0 / FP8_BLOCK : min((n0 + wn * NF * 16) / FP8_BLOCK, (a.N - 1) / FP8_BLOCK);
    const float* const ws = a.w_scale + (long long)expert * a.w_scale_expert + (long long)n_block * blocks;
    const int up_scale = (a.N + FP8_BLOCK - 1) / FP8_BLOCK * blocks;   // (GATED: from the gate's scales to the up's)
    f32x4_t acc[NF][MF];
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int b = 0; b < MF; ++b) acc[f][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float xs[MF], wg, wu = 0.f;
    auto scales = [&](int s) {
#pragma unroll
        for (int b = 0; b < MF; ++b) xs[b] = a.x_scale[s * a.x_scale_stride + scale_at[b]];
        wg = ws[s];
        if (KIND == FP8_GATED) wu = ws[up_scale + s];
    };
#pragma unroll
    for (int i = 0; i < LN + LM; ++i) load(0, inside(0), i);
    scales(0);
    const int at0 = (lq ^ ((l16 >> 1) & 7)) * 16, at1 = at0 ^ 64;      // (which codes of the block a lane has is the same on both sides)
    constexpr int EVERY = NF * MF >= 2 * (LN + LM) ? 2 : 1;            // products from a load to the next
    for (int s = 0; s < blocks; ++s) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        const unsigned char* const stage = fp8_lds + (s & 1) * STAGE;
        const bool in = inside(s + 1);
        float sc[MF], su[MF];
#pragma unroll
        for (int b = 0; b < MF; ++b) {
            sc[b] = xs[b] * wg;
            asm volatile("" : "+v"(sc[b]));                            // here, in front of the next loads: behind them it would wait for those
            if (KIND == FP8_GATED) { su[b] = xs[b] * wu; asm volatile("" : "+v"(su[b])); }
        }
        Fp8Operand<EXACT> x[MF];
#pragma unroll
        for (int b = 0; b < MF; ++b) x[b].ld(stage + (BN + (wm * MF + b) * 16 + l16) * FP8_BLOCK, at0, at1);
        // a product is added up two products later, when it is there
        Fp8Operand<EXACT> v[2];
        f32x4_t p[3];
        auto row_of = [&](int f) {                                     // GATED: the first half of a wave's pieces are gate rows, the second the same rows of up
            return KIND == FP8_GATED ? (f < NF / 2 ? (wn * (NF / 2) + f) * 16 : BN / 2 + (wn * (NF / 2) + f - NF / 2) * 16) : (wn * NF + f) * 16;
        };
        auto add = [&](int j) {
            const int f = j / MF, b = j % MF;
            const float k = KIND == FP8_GATED && f >= NF / 2 ? su[b] : sc[b];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[f][b][i] = fmaf(p[j % 3][i], k, acc[f][b][i]);
        };
        v[0].ld(stage + (row_of(0) + l16) * FP8_BLOCK, at0, at1);
#pragma unroll
        for (int j = 0; j < NF * MF; ++j) {
            const int f = j / MF, b = j % MF;
            if (b == 0 && f + 1 < NF) v[(f + 1) & 1].ld(stage + (row_of(f + 1) + l16) * FP8_BLOCK, at0, at1);
            // the next block's loads between the products: issued together they keep the waves from their products until the last is taken
            if (j % EVERY == 0 && j / EVERY < LN + LM) load(s + 1, in, j / EVERY);
            p[j % 3] = fp8_product(v[f & 1], x[b]);
            if constexpr (!EXACT) __builtin_amdgcn_sched_barrier(0);   // (left alone, the compiler waits for each product where it is made)
            if (j >= 2) add(j - 2);
            if constexpr (!EXACT) __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = (NF * MF - 1) / EVERY + 1; i < LN + LM; ++i) load(s + 1, in, i);
        scales(min(s + 1, blocks - 1));                                // (no branch: behind one the compiler would gather all sums, and spill)
        if (NF * MF >= 2) add(NF * MF - 2);
        add(NF * MF - 1);
    }
    // the last block's step has sent for one more, of zeros: it must have arrived before LDS is used for something else, and all waves must be done with their operands
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if constexpr (KIND == FP8_GATED) {
        // silu(gate) * up, the largest magnitude of a token's 128 channels over pieces, lanes and waves, codes
        constexpr int PITCH = FP8_BLOCK + 16;
        static_assert(WN * BM * 4 + BM * PITCH <= 2 * STAGE, "magnitudes and codes in LDS");
        unsigned* const largest = reinterpret_cast<unsigned*>(fp8_lds);      // [WN][BM]
        unsigned char* const codes = fp8_lds + WN * BM * 4;            // [BM], rows 16 bytes off the banks' round
#pragma unroll
        for (int b = 0; b < MF; ++b) {
            float h[NF * 2];
#pragma unroll
            for (int f = 0; f < NF / 2; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) h[f * 4 + i] = acc[f][b][i] = silu_f(acc[f][b][i]) * acc[f + NF / 2][b][i];
            unsigned top = fp8_largest<NF * 2>(h);
            top = max(top, (unsigned)__shfl_xor((int)top, 16));
            top = max(top, (unsigned)__shfl_xor((int)top, 32));
            if (lq == 0) largest[wn * BM + (wm * MF + b) * 16 + l16] = top;
        }
        __syncthreads();
#pragma unroll
        for (int b = 0; b < MF; ++b) {
            const int row = (wm * MF + b) * 16 + l16;
            unsigned top = 0;
#pragma unroll
            for (int v = 0; v < WN; ++v) top = max(top, largest[v * BM + row]);
            const int e = fp8_exponent(top);
            if (row >= rows) continue;
            if (wn == 0 && lq == 0) a.h_scale[nt * a.h_scale_stride + m0 + row] = fp8_power(e);
            const float inv = fp8_inverse(e);
#pragma unroll
            for (int f = 0; f < NF / 2; ++f)
                *reinterpret_cast<unsigned*>(codes + row * PITCH + (wn * (NF / 2) + f) * 16 + lq * 4) = fp8_codes(acc[f][b][0], acc[f][b][1], acc[f][b][2], acc[f][b][3], inv);
        }
        __syncthreads();
        for (int i = tid; i < rows * 8; i += 64 * WAVES)               // a line of 128 bytes by eight lanes
            *reinterpret_cast<u32x4_t*>(a.h + (m0 + (i >> 3)) * a.h_stride + n0 + (i & 7) * 16) = *reinterpret_cast<const u32x4_t*>(codes + (i >> 3) * PITCH + (i & 7) * 16);
    } else {
        // sixteen tokens at a time through LDS, a part of it for each wave, so that a wave's outputs of a token are stored side by side; its rows are 16 bytes off the banks' round
        constexpr int W = NF * 16, PITCH = W * 4 + 16;
        static_assert(WAVES * 16 * PITCH <= 2 * STAGE, "the results of sixteen tokens in LDS");
        constexpr int SHARE = W < 64 ? W : 64;                         // (a power of two belongs to one row of a wave)
        unsigned char* const mine = fp8_lds + wave * 16 * PITCH;
        const int es = a.y_f32 ? 4 : 2, nw = n0 + wn * W, n_left = min(W, a.N - nw);      // (n_left may be negative)
        bool wide = (((uintptr_t)a.y | (uintptr_t)(a.y_stride * es)) & 15) == 0;
        float bias[NF][4];
        if constexpr (KIND == FP8_LINEAR) {
            if (a.residual) wide = wide && (((uintptr_t)a.residual | (uintptr_t)(a.residual_stride * es)) & 15) == 0;
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int n = f * 16 + lq * 4 + i;
                    bias[f][i] = a.bias && n < n_left ? fp8_value(a.bias, a.bias_f32, nw + n) : 0.f;
                }
        }
#pragma unroll
        for (int b = 0; b < MF; ++b) {
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                f32x4_t v = acc[f][b];
                if constexpr (KIND == FP8_LINEAR)
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] += bias[f][i];
                *reinterpret_cast<f32x4_t*>(mine + l16 * PITCH + (f * 16 + lq * 4) * 4) = v;
            }
            __builtin_amdgcn_wave_barrier();
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            auto row_to = [&](int r, long long& to) {                  // where the wave's row r goes
                const int row = (wm * MF + b) * 16 + r;
                to = m0 + row;
                return row < rows;
            };
            constexpr int LANES = W / 8, AT_ONCE = 64 / LANES;         // eight outputs a lane
            const int n = lane % LANES * 8;
#pragma unroll
            for (int r0 = 0; r0 < 16; r0 += AT_ONCE) {
                const int r = r0 + lane / LANES;
                long long to;
                const f32x4_t lo = *reinterpret_cast<const f32x4_t*>(mine + r * PITCH + n * 4), hi = *reinterpret_cast<const f32x4_t*>(mine + r * PITCH + n * 4 + 16);
                float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                if constexpr (KIND == FP8_PAIRS)
                    if (!a.y_f32) {
                        // Results that meet others in a sum keep eleven bits: 16-bit floats times a power of two for SHARE outputs, which brings the largest to 2^14 .. 2^15.  (bf16
                        // made the sums half as far again from 64 bits in the root mean square, where 1.7e-3 is their own rounding; floats move twice the bytes.)
                        const unsigned top = fp8_over<SHARE / 8>(fp8_largest<8>(v));
                        const int e = max((int)(top >> 23) - 141, -126);
                        const float inv = fp8_power(-e);
                        if (!row_to(r, to) || n >= n_left) continue;
                        f16x8_t half;
#pragma unroll
                        for (int i = 0; i < 8; ++i) half[i] = (_Float16)(v[i] * inv);
                        *reinterpret_cast<f16x8_t*>(reinterpret_cast<_Float16*>(a.y) + to * a.y_stride + nw + n) = half;
                        if ((lane & (SHARE / 8 - 1)) == 0) a.row_exp[to * ((a.N + SHARE - 1) / SHARE) + (nw + n) / SHARE] = (unsigned char)(e + 127);
                        continue;
                    }
                if (!row_to(r, to) || n >= n_left) continue;
                if (wide && n + 8 <= n_left) {
                    if constexpr (KIND == FP8_LINEAR)
                        if (a.residual) {
                            float res[8];
                            if (a.y_f32) fp8_load8(reinterpret_cast<const float*>(a.residual) + to * a.residual_stride + nw + n, res);
                            else fp8_load8(reinterpret_cast<const bf16_t*>(a.residual) + to * a.residual_stride + nw + n, res);
#pragma unroll
                            for (int i = 0; i < 8; ++i) v[i] += res[i];
                        }
                    if (a.y_f32) {
                        float* const p = reinterpret_cast<float*>(a.y) + to * a.y_stride + nw + n;
                        *reinterpret_cast<f32x4_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]};
                        *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
                    } else *reinterpret_cast<u32x4_t*>(reinterpret_cast<bf16_t*>(a.y) + to * a.y_stride + nw + n) = u32x4_t{f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7])};
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (n + i < n_left) {
                            if constexpr (KIND == FP8_LINEAR)
                                if (a.residual) v[i] += fp8_value(a.residual, a.y_f32, to * a.residual_stride + nw + n + i);
                            if (a.y_f32) reinterpret_cast<float*>(a.y)[to * a.y_stride + nw + n + i] = v[i];
                            else reinterpret_cast<bf16_t*>(a.y)[to * a.y_stride + nw + n + i] = f2bf(v[i]);
                        }
                }
            }
            __builtin_amdgcn_wave_barrier();                           // (LDS serves a wave in order: its next writes come behind these reads)
        }
    }
#endif
}

template <int NF, int MF, int WN, int WM, int KIND, bool EXACT = false> inline int launch_fp8_tile(const Fp8TileArgs& a, const char* fn, hipStream_t st) {
    constexpr int lds = 2 * (NF * WN + MF * WM) * 16 * FP8_BLOCK;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&fp8_tile_kernel<NF, MF, WN, WM, KIND, EXACT>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return fail(FISE_ERR_HIP, "%s: cannot raise the dynamic LDS limit", fn);
    hipLaunchKernelGGL((fp8_tile_kernel<NF, MF, WN, WM, KIND, EXACT>), dim3((unsigned)(a.m_tiles * a.n_tiles)), dim3(64 * WN * WM), lds, st, a);
    FISE_CHECK_LAUNCH(fn);
    return FISE_OK;
}

}  // namespace fise
