// Products of a few rows with 4-bit weights: y[m, n] = sum_k act(x[m, k]) s[n, k / g] q[n, k] + bias[n] (+ residual[m, n]), q a whole number from -8 to 7,
// s one bf16 number for g columns of an output.
//
// The weight bytes bound it (a byte holds two weights and is read once), and next to them the instructions that make bf16 of them.  So the weights are laid out
// once as operands of the matrix unit (w4_choice.h): a wave reads 1 KB of consecutive bytes, 16 outputs x 128 columns, and a lane's 16 bytes are its part of
// four 16x16x32 instructions.  A weight goes to float as q / 16 (v_cvt_off_f32_i4) and two of those to a bf16 pair; both are exact, and so are the
// products; they are added in float, a group at a time, and the group's scale is applied to that sum, in float too.  Nothing is added to the
// weights that would have to be taken off again, so an infinite x gives what the definition gives.
// x of a wave's columns stays in registers as operands, and the wave streams the weights of one tile of outputs after the other past it; nothing else is read again.
// Float x, and x behind SiLU, is split into three bf16 numbers that add up to it exactly: three rows of the
// instruction, of which a few rows of x leave most idle, added in the epilogue.
// 16 rows, 28672 outputs of 8192 columns: 31 us, 3.9 TB/s, with six sets of weights in turn, which no cache holds, and 28 us, 4.4 TB/s, with the same ones again and again (a sum over
// arrays of that size reads 3.2 and 4.5, over 1 GB 3.9); 2 float rows behind SiLU, 20160 outputs of 1280 columns: 10 and 8 us, of which the launch is the larger part.
#include "igemm.h"
#include "profile.h"
#include "w4_choice.h"

namespace fise {

// ---------------------------------------------------------------------------------------------------------------- packing
__device__ __forceinline__ float w4_value(const float* p) { return *p; }
__device__ __forceinline__ float w4_value(const bf16_t* p) { return bf2f(*p); }
__device__ __forceinline__ size_t w4_scale_at(int n, int k, int group, int tiles_k, int groups) {
    const size_t tn = n / W4_ROWS, row = n % W4_ROWS;
    if (group < W4_COLS) return ((tn * tiles_k + k / W4_COLS) * W4_ROWS + row) * (W4_COLS / group) + k % W4_COLS / group;
    return (tn * groups + k / group) * W4_ROWS + row;
}

// A lane packs eight columns of an output; the lanes of a group find its largest magnitude among them.  The scale is that / 7 in bf16, a weight the
// nearest multiple of it: at most half a scale off (7 scales are at least 7 / (7 (1 + 2^-8)) of the largest; below bf16's normal range, where its steps are a larger part,
// one step more if they are not).  Magnitudes are compared as
// whole numbers, so that a NaN wins: a group with a value that is not finite has a scale that is not, and comes back as NaN.
template <typename T>
__global__ __launch_bounds__(256) void w4_pack_kernel(const T* __restrict__ w, const bf16_t* __restrict__ given, int N, int K, int group, int tiles_k, int groups,
                                                      unsigned* __restrict__ tiles, bf16_t* __restrict__ scales) {
    const int n = blockIdx.y, k = (blockIdx.x * 256 + threadIdx.x) * 8, cols = tiles_k * W4_COLS;
    float v[8];
    unsigned top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = n < N && k + e < K ? w4_value(w + (size_t)n * K + k + e) : 0.f;
        top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
    }
    for (int o = 1; o < group / 8; o <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, o));
    if (k >= cols) return;
    bf16_t s = 0;
    if (n < N && k < K) {
        s = given ? given[(size_t)n * groups + k / group] : f2bf(__uint_as_float(top) / 7.f);
        if (!given && 7.5f * bf2f(s) < __uint_as_float(top)) ++s;
    }
    const float sf = bf2f(s);
    unsigned word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float r = rintf(v[e] / sf);
        const float lo = given ? -8.f : -7.f;
        const int q = sf != 0.f && r == r ? (int)fminf(fmaxf(r, lo), 7.f) : 0;
        word |= ((unsigned)q & 15u) << (4 * e);
    }
    const int in = k % W4_COLS / 8, j = in / 4, quarter = in % 4;
    tiles[(((size_t)(n / W4_ROWS) * tiles_k + k / W4_COLS) * 64 + quarter * 16 + n % W4_ROWS) * 4 + j] = word;
    if (k % group == 0 && (group < W4_COLS || k < K)) scales[w4_scale_at(n, k, group, tiles_k, groups)] = s;
}

template <typename T>
__global__ __launch_bounds__(256) void w4_unpack_kernel(const unsigned* __restrict__ tiles, const bf16_t* __restrict__ scales, int N, int K, int group, int tiles_k, int groups,
                                                        T* __restrict__ w) {
    const int n = blockIdx.y, k = (blockIdx.x * 256 + threadIdx.x) * 8;
    if (k >= K) return;
    const int in = k % W4_COLS / 8, j = in / 4, quarter = in % 4;
    const unsigned word = tiles[(((size_t)(n / W4_ROWS) * tiles_k + k / W4_COLS) * 64 + quarter * 16 + n % W4_ROWS) * 4 + j];
    const float s = bf2f(scales[w4_scale_at(n, k, group, tiles_k, groups)]);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (k + e < K) Elem<T>::st(w + (size_t)n * K + k + e, (float)((int)(word << (28 - 4 * e)) >> 28) * s);
}

// ---------------------------------------------------------------------------------------------------------------- product
struct W4Args {
    const void* x; long long x_stride; int x_f32, silu;
    const unsigned char* tiles; const bf16_t* scales; int N, K, tiles_k, groups, group_shift;      // group_shift: tile columns of a group as a power of two (wide groups)
    const void* bias; int bias_f32; const void* residual; long long residual_stride; void* y; long long y_stride; int y_f32;
    int M;
    W4Choice c;
};

#if defined(__HIP_DEVICE_COMPILE__)
// Eight weights / 16 of a word as the operand's four bf16 pairs: exact.  A conversion takes the lowest four bits of a byte that it picks itself.
__device__ __forceinline__ bf16x8_t w4_operand(unsigned w) {
    const unsigned odd = w >> 4;
    u32x4_t r;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
        float lo, hi;
        if (b == 0) asm("v_cvt_off_f32_i4_sdwa %0, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0\n\tv_cvt_off_f32_i4_sdwa %1, %3 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=&v"(lo), "=v"(hi) : "v"(w), "v"(odd));
        if (b == 1) asm("v_cvt_off_f32_i4_sdwa %0, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1\n\tv_cvt_off_f32_i4_sdwa %1, %3 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=&v"(lo), "=v"(hi) : "v"(w), "v"(odd));
        if (b == 2) asm("v_cvt_off_f32_i4_sdwa %0, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2\n\tv_cvt_off_f32_i4_sdwa %1, %3 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=&v"(lo), "=v"(hi) : "v"(w), "v"(odd));
        if (b == 3) asm("v_cvt_off_f32_i4_sdwa %0, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3\n\tv_cvt_off_f32_i4_sdwa %1, %3 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=&v"(lo), "=v"(hi) : "v"(w), "v"(odd));
        r[b] = f2bf2(lo, hi);
    }
    return *reinterpret_cast<const bf16x8_t*>(&r);
}
#endif

__device__ __forceinline__ void w4_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }      // (loads to registers that are on their way stay there)

// a value of x as three bf16 numbers that add up to it
__device__ __forceinline__ void w4_split(float v, bf16_t (&p)[3]) {    // truncated, not rounded: no piece of a finite number overflows, and what is left has 8 bits in the end
    const unsigned a = __float_as_uint(v) & 0xffff0000u;
    p[0] = (bf16_t)(a >> 16);
    const bool finite = (a & 0x7f800000u) != 0x7f800000u;
    const float r1 = finite ? v - __uint_as_float(a) : 0.f;
    const unsigned b = __float_as_uint(r1) & 0xffff0000u;
    p[1] = (bf16_t)(b >> 16);
    p[2] = (bf16_t)(__float_as_uint(r1 - __uint_as_float(b)) >> 16);
    if (v != v) p[0] |= 0x40;                                          // a NaN whose bits are all in the lower half stays one
}

struct W4Eight { uint4 a, b; };                                        // eight values of x as they lie in memory (bf16: the first half)
__device__ __forceinline__ W4Eight w4_load(const W4Args& g, int m, int k) {
    W4Eight r = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (k >= g.K || m >= g.M) return r;
    if (g.x_f32) {
        const uint4* const p = reinterpret_cast<const uint4*>((const float*)g.x + (size_t)m * g.x_stride + k);
        r.a = p[0]; r.b = p[1];
    } else r.a = *reinterpret_cast<const uint4*>((const bf16_t*)g.x + (size_t)m * g.x_stride + k);
    return r;
}
__device__ __forceinline__ void w4_pieces(const W4Args& g, const W4Eight& x, unsigned (&out)[3][4]) {
    const unsigned f[8] = {x.a.x, x.a.y, x.a.z, x.a.w, x.b.x, x.b.y, x.b.z, x.b.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float v = g.x_f32 ? __uint_as_float(f[e]) : e & 1 ? hi16(f[e >> 1]) : lo16(f[e >> 1]);
        bf16_t p[3];
        w4_split(g.silu ? silu_f(v) : v, p);
#pragma unroll
        for (int q = 0; q < 3; ++q) out[q][e >> 1] = e & 1 ? out[q][e >> 1] | (unsigned)p[q] << 16 : p[q];
    }
}
// What is left when the sums of an output are there (times 1/16, as the weights were): bias, residual, store
__device__ __forceinline__ void w4_store(const W4Args& a, int m, int n, float v) {
    v *= 16.f;
    if (a.bias) v += a.bias_f32 ? ((const float*)a.bias)[n] : bf2f(((const bf16_t*)a.bias)[n]);
    const size_t at = (size_t)m * a.y_stride + n;
    if (a.residual) {
        const size_t ar = (size_t)m * a.residual_stride + n;
        v += a.y_f32 ? ((const float*)a.residual)[ar] : bf2f(((const bf16_t*)a.residual)[ar]);
    }
    if (a.y_f32) ((float*)a.y)[at] = v; else ((bf16_t*)a.y)[at] = f2bf(v);
}

// MT: tiles of 16 rows of x; KT: tile columns of a wave; GS: matrix instructions a scale covers (1, 2, 4: groups of 32, 64, 128 and more); SPLIT: three pieces a value.
template <int MT, int KT, int GS, bool SPLIT>
__global__ __launch_bounds__(MT == 4 ? 512 : 1024) void w4_linear_kernel(const W4Args a) {
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), threads = blockDim.x;
    const W4Choice& c = a.c;
    const int l16 = lane & 15, lq = lane >> 4;
    const int m0 = blockIdx.y * c.slab, rows = min(c.slab, a.M - m0);
    const int all_n = (a.N + W4_ROWS - 1) / W4_ROWS, n0 = blockIdx.x * c.tiles_n, n_n = min(c.tiles_n, all_n - n0);
    float* const red = reinterpret_cast<float*>(lds);                  // [tile of outputs][wave][row of x][16]

    constexpr int NS = 4 / GS, SW = (NS + 1) / 2, U = 4 / KT;          // scales of a tile, words of them; tiles of outputs in flight
    u32x4_t w[U][KT];
    unsigned s[U][KT][SW];
    bf16x8_t xf[KT][4][MT];
    for (int chunk = 0; chunk < c.chunks; ++chunk) {
        const int t0 = (chunk * c.waves_k + wave) * KT, n_t = min(max(a.tiles_k - t0, 0), KT);      // this wave's tile columns
        auto fetch = [&](int slot, int n) {
#pragma unroll
            for (int t = 0; t < KT; ++t)
                if (t < n_t) {
                    w[slot][t] = *reinterpret_cast<const u32x4_t*>(a.tiles + ((size_t)(n0 + n) * a.tiles_k + t0 + t) * W4_TILE_BYTES + lane * 16);
                    const bf16_t* const st = a.scales + (size_t)(n0 + n) * (GS < 4 ? a.tiles_k * NS : a.groups) * W4_ROWS;
                    if constexpr (GS == 4) s[slot][t][0] = st[(size_t)((t0 + t) >> a.group_shift) * W4_ROWS + l16];
                    else if constexpr (GS == 2) s[slot][t][0] = *reinterpret_cast<const unsigned*>(st + ((size_t)(t0 + t) * W4_ROWS + l16) * 2);
                    else { const uint2 v = *reinterpret_cast<const uint2*>(st + ((size_t)(t0 + t) * W4_ROWS + l16) * 4); s[slot][t][0] = v.x; s[slot][t][SW - 1] = v.y; }
                }
        };
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < n_n) fetch(u, u);

        // ---- x of this wave's columns
        if constexpr (!SPLIT) {
            const auto from = buf((const bf16_t*)a.x + (size_t)m0 * a.x_stride, (unsigned)((rows - 1) * a.x_stride + a.K) * 2);
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int r = 0; r < MT; ++r) {                     // (rows and columns that do not exist: zeros)
                        const int k = (t0 + t) * W4_COLS + j * 32 + lq * 8, m = r * 16 + l16;
                        const u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(from, k < a.K && m < rows ? (m * (int)a.x_stride + k) * 2 : 0x7fffffff, 0, 0);
                        xf[t][j][r] = *reinterpret_cast<const bf16x8_t*>(&v);
                    }
        } else {
            // a tile column of every wave and 16 rows (pieces) at a time through LDS, so that a value is worked out once
            bf16_t* const xs = reinterpret_cast<bf16_t*>(lds + c.x_at);
            const int cols = c.waves_k * W4_COLS, pitch = cols + 8;
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int r = 0; r < MT; ++r) {
                    __syncthreads();
                    const int mlo = r * 16 / 3, mhi = min(rows, (r * 16 + 15) / 3 + 1);      // rows of x with a piece among these
                    for (int i = tid; i < (mhi - mlo) * (cols / 8); i += threads) {
                        const int m = mlo + i / (cols / 8), col = (i - (m - mlo) * (cols / 8)) * 8;
                        const int k = ((chunk * c.waves_k + col / W4_COLS) * KT + t) * W4_COLS + col % W4_COLS;
                        unsigned out[3][4];
                        w4_pieces(a, w4_load(a, m0 + m, k), out);
#pragma unroll
                        for (int q = 0; q < 3; ++q) {
                            const int row = m * 3 + q - r * 16;
                            if (row >= 0 && row < 16) *reinterpret_cast<uint4*>(xs + (size_t)row * pitch + col) = make_uint4(out[q][0], out[q][1], out[q][2], out[q][3]);
                        }
                    }
                    __syncthreads();
                    const int row = r * 16 + l16 < rows * 3 ? l16 : 0; // (pieces that do not exist: the first one's, not stored in the end)
#pragma unroll
                    for (int j = 0; j < 4; ++j) xf[t][j][r] = *reinterpret_cast<const bf16x8_t*>(xs + (size_t)row * pitch + wave * W4_COLS + j * 32 + lq * 8);
                }
            __syncthreads();                                           // the parts may take the same room
        }

        for (int i0 = 0; i0 < n_n; i0 += U) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int n = i0 + u;
                if (n < n_n) {
                    f32x4_t acc[MT];
#pragma unroll
                    for (int r = 0; r < MT; ++r) acc[r] = f32x4_t{0, 0, 0, 0};
#pragma unroll
                    for (int t = 0; t < KT; ++t)
                        if (t < n_t) {
                            f32x4_t part[MT];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const bf16x8_t b = w4_operand(w[u][t][j]);
#pragma unroll
                                for (int r = 0; r < MT; ++r) part[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[t][j][r], b, j % GS ? part[r] : f32x4_t{0, 0, 0, 0}, 0, 0, 0);
                                if (j % GS == GS - 1) {
                                    const unsigned sw = s[u][t][j / GS / 2];
                                    const float sc = GS < 4 && (j / GS) % 2 ? hi16(sw) : lo16(sw);
#pragma unroll
                                    for (int r = 0; r < MT; ++r)
#pragma unroll
                                        for (int e = 0; e < 4; ++e) acc[r][e] = fmaf(part[r][e], sc, acc[r][e]);
                                }
                            }
                        }
                    if (n + U < n_n) fetch(u, n + U);
                    float* const to = red + ((size_t)n * c.waves_k + wave) * (MT * 256) + lane * 4;      // [row tile][lane][4]: rows lq * 4 + (0..3), output l16
#pragma unroll
                    for (int r = 0; r < MT; ++r) {
                        f32x4_t* const at = reinterpret_cast<f32x4_t*>(to + r * 256);
                        *at = chunk ? *at + acc[r] : acc[r];
                    }
                }
            }
        }
    }
    // ---- the waves of an output tile and the pieces of a row, in order
    __syncthreads();
    for (int i = tid; i < n_n * rows * 16; i += threads) {
        const int col = i & 15, rest = i >> 4, g = rest / rows, m = rest - g * rows, n = (n0 + g) * W4_ROWS + col;
        if (n >= a.N) continue;
        float v = 0.f;
        for (int k = 0; k < c.waves_k; ++k)
#pragma unroll
            for (int q = SPLIT ? 2 : 0; q >= 0; --q) {
                const int row = SPLIT ? m * 3 + q : m;
                v += red[((size_t)g * c.waves_k + k) * (MT * 256) + (row >> 4) * 256 + ((row >> 2 & 3) * 16 + col) * 4 + (row & 3)];
            }
        w4_store(a, m0 + m, n, v);
    }
#endif
}

// The staged form.  Every wave has a tile of outputs (or waves_k waves share one and take turns with its tile columns) and all rows; x of the next four tile columns is on its
// way to registers while these are multiplied, and goes to the other half of LDS behind them.  Rows of the last tiles that three pieces a value leave over hold whatever LDS
// held: the matrix unit keeps rows apart, and theirs are not stored.
// 64 rows, 8192 outputs of 8192 columns: 35 us, five times what the bytes take.  No unit is full (of a CU's cycles the matrix units are busy 10 %, the vector units 38 %, LDS about
// half, a fifth of it bank conflicts): with one workgroup a CU, loads, the writes of x to LDS and the products of a chunk wait for one another at its barrier, and a CU moves 64 KB
// of x for every 8 KB of weights.
template <int MT, int GS, bool SPLIT>
__global__ __launch_bounds__(512) void w4_staged_kernel(const W4Args a) {
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    constexpr int ROWS = MT * 16, PITCH = W4_STAGE_PITCH, PIECES = W4_STAGE_COLS / 8, NS = 4 / GS, SW = (NS + 1) / 2;
    constexpr int SRC_ROWS = SPLIT ? (ROWS - 1) / 3 : ROWS, LOADS = (SRC_ROWS * PIECES + 511) / 512;      // rows of x of a slab, pieces of eight columns a lane
    bf16_t* const xs = reinterpret_cast<bf16_t*>(lds);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, lq = lane >> 4;
    const W4Choice& c = a.c;
    const int kw = wave % c.waves_k, nw = wave / c.waves_k, m0 = blockIdx.y * c.slab, rows = min(c.slab, a.M - m0);
    const int all_n = (a.N + W4_ROWS - 1) / W4_ROWS, n0 = blockIdx.x * c.tiles_n, tn = min(n0 + nw, all_n - 1);      // (behind the last tile: that one again, not stored)

    W4Eight raw[LOADS];
    auto load_x = [&](int chunk) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int p = tid + i * 512, m = p / PIECES, k = chunk * W4_STAGE_COLS + p % PIECES * 8;
            raw[i] = m < rows ? w4_load(a, m0 + m, k) : W4Eight{make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
        }
    };
    auto put_x = [&](int half) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int p = tid + i * 512, m = p / PIECES;
            if (m >= SRC_ROWS) continue;
            bf16_t* const to = xs + (size_t)(half * ROWS + (SPLIT ? m * 3 : m)) * PITCH + p % PIECES * 8;
            if constexpr (SPLIT) {
                unsigned out[3][4];
                w4_pieces(a, raw[i], out);
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<uint4*>(to + q * PITCH) = make_uint4(out[q][0], out[q][1], out[q][2], out[q][3]);
            } else *reinterpret_cast<uint4*>(to) = raw[i].a;
        }
    };
    // four tile columns of a chunk, of which this wave has every waves_k-th
    u32x4_t w[2][4];
    unsigned s[2][4][SW];
    auto load_w = [&](int set, int chunk) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = min(chunk * 4 + i, a.tiles_k - 1);           // (behind the last column: that one again; x is zeros there)
            if (i % c.waves_k == kw) {
                w[set][i] = *reinterpret_cast<const u32x4_t*>(a.tiles + ((size_t)tn * a.tiles_k + t) * W4_TILE_BYTES + lane * 16);
                const bf16_t* const st = a.scales + (size_t)tn * (GS < 4 ? a.tiles_k * NS : a.groups) * W4_ROWS;
                if constexpr (GS == 4) s[set][i][0] = st[(size_t)(t >> a.group_shift) * W4_ROWS + l16];
                else if constexpr (GS == 2) s[set][i][0] = *reinterpret_cast<const unsigned*>(st + ((size_t)t * W4_ROWS + l16) * 2);
                else { const uint2 v = *reinterpret_cast<const uint2*>(st + ((size_t)t * W4_ROWS + l16) * 4); s[set][i][0] = v.x; s[set][i][SW - 1] = v.y; }
            }
        }
    };
    f32x4_t acc[MT];
#pragma unroll
    for (int r = 0; r < MT; ++r) acc[r] = f32x4_t{0, 0, 0, 0};
    const bf16_t* const from = xs + (size_t)l16 * PITCH + lq * 8;
    auto multiply = [&](int set, int chunk) {
        const int half = chunk & 1;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i % c.waves_k == kw && chunk * 4 + i < a.tiles_k) {
                f32x4_t part[MT];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16x8_t b = w4_operand(w[set][i][j]);
#pragma unroll
                    for (int r = 0; r < MT; ++r) {
                        const bf16x8_t x = *reinterpret_cast<const bf16x8_t*>(from + (size_t)(half * ROWS + r * 16) * PITCH + i * W4_COLS + j * 32);
                        part[r] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, b, j % GS ? part[r] : f32x4_t{0, 0, 0, 0}, 0, 0, 0);
                    }
                    if (j % GS == GS - 1) {
                        const unsigned sw = s[set][i][j / GS / 2];
                        const float sc = GS < 4 && (j / GS) % 2 ? hi16(sw) : lo16(sw);
#pragma unroll
                        for (int r = 0; r < MT; ++r)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[r][e] = fmaf(part[r][e], sc, acc[r][e]);
                    }
                }
            }
    };
    load_x(0);
    load_w(0, 0);
    put_x(0);
    for (int chunk = 0; chunk < c.chunks; chunk += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int at = chunk + u;
            if (at >= c.chunks) break;
            w4_barrier();                                              // x of this chunk is there, that of the chunk before has been read
            if (at + 1 < c.chunks) { load_w(u ^ 1, at + 1); load_x(at + 1); }
            multiply(u, at);
            if (at + 1 < c.chunks) put_x((at + 1) & 1);
        }
    }
    __syncthreads();
    float* const red = reinterpret_cast<float*>(lds);                  // [wave][row tile][lane][4]
#pragma unroll
    for (int r = 0; r < MT; ++r) *reinterpret_cast<f32x4_t*>(red + (wave * MT + r) * 256 + lane * 4) = acc[r];
    __syncthreads();
    for (int i = tid; i < c.tiles_n * rows * 16; i += 512) {
        const int col = i & 15, rest = i >> 4, g = rest / rows, m = rest - g * rows, n = (n0 + g) * W4_ROWS + col;
        if (n >= a.N) continue;
        float v = 0.f;
        for (int k = 0; k < c.waves_k; ++k)
#pragma unroll
            for (int q = SPLIT ? 2 : 0; q >= 0; --q) {
                const int row = SPLIT ? m * 3 + q : m;
                v += red[((g * c.waves_k + k) * MT + (row >> 4)) * 256 + ((row >> 2 & 3) * 16 + col) * 4 + (row & 3)];
            }
        w4_store(a, m0 + m, n, v);
    }
#endif
}

template <int MT, int KT, int GS, bool SPLIT> static int launch_w4(const W4Args& a, hipStream_t st) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&w4_linear_kernel<MT, KT, GS, SPLIT>), hipFuncAttributeMaxDynamicSharedMemorySize, W4_LDS);
    if (attr != hipSuccess) return fail(FISE_ERR_HIP, "fise_w4_linear: cannot raise the dynamic LDS limit");
    const W4Choice& c = a.c;
    {
        const double bytes = (double)a.N * a.K / 2 + 2.0 * a.N * a.groups + (double)a.M * a.K * (a.x_f32 ? 4 : 2) + (double)a.M * a.N * (a.y_f32 ? 4 : 2);
        ProfileScope prof(PROF_ROWS_GEMM, 2.0 * a.M * a.N * a.K, bytes, st);
        hipLaunchKernelGGL((w4_linear_kernel<MT, KT, GS, SPLIT>), dim3((unsigned)c.groups_n, (unsigned)c.slabs), dim3(64u * c.waves_k), (size_t)c.lds, st, a);
    }
    FISE_CHECK_LAUNCH("fise_w4_linear");
    return FISE_OK;
}
template <int MT, int GS, bool SPLIT> static int launch_staged(const W4Args& a, hipStream_t st) {
    constexpr int lds = 2 * MT * 16 * W4_STAGE_PITCH * 2;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&w4_staged_kernel<MT, GS, SPLIT>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return fail(FISE_ERR_HIP, "fise_w4_linear: cannot raise the dynamic LDS limit");
    {
        const double bytes = (double)a.N * a.K / 2 + 2.0 * a.N * a.groups + (double)a.M * a.K * (a.x_f32 ? 4 : 2) + (double)a.M * a.N * (a.y_f32 ? 4 : 2);
        ProfileScope prof(PROF_ROWS_GEMM, 2.0 * a.M * a.N * a.K, bytes, st);
        hipLaunchKernelGGL((w4_staged_kernel<MT, GS, SPLIT>), dim3((unsigned)a.c.groups_n, (unsigned)a.c.slabs), dim3(512), lds, st, a);
    }
    FISE_CHECK_LAUNCH("fise_w4_linear");
    return FISE_OK;
}
template <int MT> static int launch_staged(const W4Args& a, int group, hipStream_t st) {
    if (a.c.pieces == 3) return group == 32 ? launch_staged<MT, 1, true>(a, st) : group == 64 ? launch_staged<MT, 2, true>(a, st) : launch_staged<MT, 4, true>(a, st);
    return group == 32 ? launch_staged<MT, 1, false>(a, st) : group == 64 ? launch_staged<MT, 2, false>(a, st) : launch_staged<MT, 4, false>(a, st);
}
template <int MT, int KT> static int launch_w4(const W4Args& a, int group, hipStream_t st) {
    if (a.c.pieces == 3) return group == 32 ? launch_w4<MT, KT, 1, true>(a, st) : group == 64 ? launch_w4<MT, KT, 2, true>(a, st) : launch_w4<MT, KT, 4, true>(a, st);
    return group == 32 ? launch_w4<MT, KT, 1, false>(a, st) : group == 64 ? launch_w4<MT, KT, 2, false>(a, st) : launch_w4<MT, KT, 4, false>(a, st);
}

// sizes that pack, unpack and product share; numbers of tiles have 31 bits
static int w4_check(const char* fn, int N, int K, int group) {
    if (N < 1 || K < 1 || !w4_group_ok(group)) return fail(FISE_ERR_SHAPE, "%s: N=%d K=%d group=%d (32, 64, 128 or 256)", fn, N, K, group);
    if (N > 1 << 20 || K > 1 << 20) return fail(FISE_ERR_SHAPE, "%s: N=%d K=%d beyond 2^20", fn, N, K);
    return FISE_OK;
}

}  // namespace fise

using namespace fise;

extern "C" size_t fise_w4_bytes(int N, int K, int group) {
    if (w4_check("fise_w4_bytes", N, K, group)) return 0;
    return (size_t)w4_layout(N, K, group).bytes;
}

extern "C" int fise_w4_pack(const void* w, int dtype, const void* scale, int N, int K, int group, void* packed, void* stream) {
    const char* fn = "fise_w4_pack";
    if (!w || !packed) return fail(FISE_ERR_NULL, "%s: null pointer", fn);
    if (dtype != FISE_F32 && dtype != FISE_BF16) return fail(FISE_ERR_DTYPE, "%s: dtype %d", fn, dtype);
    if (int e = w4_check(fn, N, K, group)) return e;
    if (!aligned16(w) || !aligned16(scale) || !aligned16(packed)) return fail(FISE_ERR_ALIGN, "%s: pointers must be 16-byte aligned", fn);
    const W4Layout l = w4_layout(N, K, group);
    const dim3 block(256);
    bf16_t* const scales = (bf16_t*)((unsigned char*)packed + l.scale_off);
    // outputs go in the grid's second dimension, which ends at 65535
    for (int n0 = 0; n0 < (int)l.tiles_n * W4_ROWS; n0 += 32768) {
        const int rows = std::min((int)l.tiles_n * W4_ROWS - n0, 32768);
        const dim3 grid((unsigned)ceil_div((int)l.tiles_k * W4_COLS, 2048), (unsigned)rows);
        const size_t per_row = (size_t)(group < W4_COLS ? l.tiles_k * (W4_COLS / group) : l.groups);
        unsigned* const t = (unsigned*)((unsigned char*)packed + (size_t)(n0 / W4_ROWS) * l.tiles_k * W4_TILE_BYTES);
        bf16_t* const s = scales + (size_t)n0 * per_row;
        const bf16_t* const given = scale ? (const bf16_t*)scale + (size_t)n0 * l.groups : nullptr;
        if (dtype == FISE_F32)
            hipLaunchKernelGGL(w4_pack_kernel<float>, grid, block, 0, as_stream(stream), (const float*)w + (size_t)n0 * K, given, N - n0, K, group, (int)l.tiles_k, (int)l.groups, t, s);
        else
            hipLaunchKernelGGL(w4_pack_kernel<bf16_t>, grid, block, 0, as_stream(stream), (const bf16_t*)w + (size_t)n0 * K, given, N - n0, K, group, (int)l.tiles_k, (int)l.groups, t, s);
        FISE_CHECK_LAUNCH(fn);
    }
    return FISE_OK;
}

extern "C" int fise_w4_unpack(const void* packed, int N, int K, int group, void* w, int dtype, void* stream) {
    const char* fn = "fise_w4_unpack";
    if (!w || !packed) return fail(FISE_ERR_NULL, "%s: null pointer", fn);
    if (dtype != FISE_F32 && dtype != FISE_BF16) return fail(FISE_ERR_DTYPE, "%s: dtype %d", fn, dtype);
    if (int e = w4_check(fn, N, K, group)) return e;
    if (!aligned16(w) || !aligned16(packed)) return fail(FISE_ERR_ALIGN, "%s: pointers must be 16-byte aligned", fn);
    const W4Layout l = w4_layout(N, K, group);
    const size_t per_row = (size_t)(group < W4_COLS ? l.tiles_k * (W4_COLS / group) : l.groups);
    for (int n0 = 0; n0 < N; n0 += 32768) {
        const dim3 grid((unsigned)ceil_div(K, 2048), (unsigned)std::min(N - n0, 32768)), block(256);
        const unsigned* const t = (const unsigned*)((const unsigned char*)packed + (size_t)(n0 / W4_ROWS) * l.tiles_k * W4_TILE_BYTES);
        const bf16_t* const s = (const bf16_t*)((const unsigned char*)packed + l.scale_off) + (size_t)n0 * per_row;
        if (dtype == FISE_F32)
            hipLaunchKernelGGL(w4_unpack_kernel<float>, grid, block, 0, as_stream(stream), t, s, N - n0, K, group, (int)l.tiles_k, (int)l.groups, (float*)w + (size_t)n0 * K);
        else
            hipLaunchKernelGGL(w4_unpack_kernel<bf16_t>, grid, block, 0, as_stream(stream), t, s, N - n0, K, group, (int)l.tiles_k, (int)l.groups, (bf16_t*)w + (size_t)n0 * K);
        FISE_CHECK_LAUNCH(fn);
    }
    return FISE_OK;
}

extern "C" int fise_w4_linear(const fise_w4_linear_args* g, void* stream) {
    const char* fn = "fise_w4_linear";
    if (!g || !g->x || !g->packed || !g->y) return fail(FISE_ERR_NULL, "%s: null pointer", fn);
    auto known = [](int d) { return d == FISE_F32 || d == FISE_BF16; };
    if (!known(g->x_dtype) || !known(g->y_dtype) || (g->bias && !known(g->bias_dtype)))
        return fail(FISE_ERR_DTYPE, "%s: dtypes x %d, y %d, bias %d", fn, g->x_dtype, g->y_dtype, g->bias_dtype);
    if (int e = w4_check(fn, g->N, g->K, g->group)) return e;
    if (g->M < 0 || g->M > 1 << 20 || g->x_stride < g->K || g->y_stride < g->N || (g->residual && g->residual_stride < g->N))
        return fail(FISE_ERR_SHAPE, "%s: M=%d, strides x %lld, y %lld, residual %lld", fn, g->M, (long long)g->x_stride, (long long)g->y_stride, (long long)g->residual_stride);
    if (g->x_stride > 1 << 23) return fail(FISE_ERR_SHAPE, "%s: rows of x %lld apart (at most 2^23)", fn, (long long)g->x_stride);      // a slab's offsets have 31 bits
    if (g->K % 8 || g->x_stride % 8 || !aligned16(g->x) || !aligned16(g->packed))
        return fail(FISE_ERR_ALIGN, "%s: K and the row stride of x must be multiples of 8, x and the weights 16-byte aligned", fn);
    const size_t ye = g->y_dtype == FISE_F32 ? 4 : 2, be = g->bias_dtype == FISE_F32 ? 4 : 2;
    if ((uintptr_t)g->y % ye || (uintptr_t)g->residual % ye || (g->bias && (uintptr_t)g->bias % be)) return fail(FISE_ERR_ALIGN, "%s: y, residual and bias must be aligned to their type", fn);
    if (g->M == 0) return FISE_OK;
    const W4Layout l = w4_layout(g->N, g->K, g->group);
    W4Args a{};
    a.x = g->x; a.x_stride = g->x_stride; a.x_f32 = g->x_dtype == FISE_F32; a.silu = g->silu_in != 0;
    a.tiles = (const unsigned char*)g->packed; a.scales = (const bf16_t*)((const unsigned char*)g->packed + l.scale_off);
    a.N = g->N; a.K = g->K; a.tiles_k = (int)l.tiles_k; a.groups = (int)l.groups; a.group_shift = g->group == 256 ? 1 : 0;
    a.bias = g->bias; a.bias_f32 = g->bias_dtype == FISE_F32;
    a.residual = g->residual; a.residual_stride = g->residual_stride; a.y = g->y; a.y_stride = g->y_stride; a.y_f32 = g->y_dtype == FISE_F32;
    a.M = g->M;
    a.c = w4_choose(g->M, g->N, g->K, a.x_f32 || a.silu);
    const hipStream_t st = as_stream(stream);
    if (a.c.staged) return a.c.mt == 2 ? launch_staged<2>(a, g->group, st) : launch_staged<4>(a, g->group, st);
    if (a.c.mt == 1) return a.c.kt == 1 ? launch_w4<1, 1>(a, g->group, st) : a.c.kt == 2 ? launch_w4<1, 2>(a, g->group, st) : launch_w4<1, 4>(a, g->group, st);
    if (a.c.mt == 2) return a.c.kt == 1 ? launch_w4<2, 1>(a, g->group, st) : launch_w4<2, 2>(a, g->group, st);
    return launch_w4<4, 1>(a, g->group, st);
}
