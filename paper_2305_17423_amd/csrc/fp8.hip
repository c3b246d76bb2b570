// 8-bit floating point (e4m3) with a scale for each block of 128 columns: rows and weights into codes, and the product of the two.
//
// Scales that the library makes are powers of two: dividing by one is exact, so a code is the value rounded once, and the largest of a block uses the format's range to
// within a factor of two, which costs none of the three bits of mantissa.  Rows into codes are bound by their bytes: 8192 x 8192 in bf16, 35 us (5.7 TB/s) among other launches.
#include "fp8_few.h"
#include "fp8_choice.h"

namespace fise {

template <typename T>
__global__ __launch_bounds__(256) void fp8_rows_kernel(const T* x, long long x_stride, int M, int K, int units, int written, unsigned char* codes, long long code_stride,
                                                       float* scale, long long scale_stride) {
    fp8_quantize_unit(x, x_stride, M, K, units, written, codes, code_stride, scale, scale_stride, (long long)blockIdx.x * 256 + threadIdx.x);
}

// A workgroup has 128 x 128 values: a lane eight columns of every sixteenth row.
template <typename T>
__global__ __launch_bounds__(256) void fp8_block_kernel(const T* x, long long x_stride, int M, int K, int blocks, unsigned char* codes, long long code_stride,
                                                        float* scale, long long scale_stride) {
    __shared__ unsigned largest[4];
    const int tid = threadIdx.x, bk = blockIdx.x % blocks, bm = blockIdx.x / blocks, col = bk * FP8_BLOCK + (tid & 15) * 8;
    const long long row0 = (long long)bm * FP8_BLOCK + (tid >> 4);
    float v[8][8];
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const long long row = row0 + 16 * j;
        if (row < M && col < K) fp8_load8(x + row * x_stride + col, v[j]);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = 0.f;
        top = max(top, fp8_largest<8>(v[j]));
    }
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) top = max(top, (unsigned)__shfl_xor((int)top, o));
    if ((tid & 63) == 0) largest[tid >> 6] = top;
    __syncthreads();
    const int e = fp8_exponent(max(max(largest[0], largest[1]), max(largest[2], largest[3])));
    const float inv = fp8_inverse(e);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const long long row = row0 + 16 * j;
        if (row < M && col < K)
            *reinterpret_cast<u32x2_t*>(codes + row * code_stride + col) =
                u32x2_t{fp8_codes(v[j][0], v[j][1], v[j][2], v[j][3], inv), fp8_codes(v[j][4], v[j][5], v[j][6], v[j][7], inv)};
    }
    if (tid == 0) scale[bm * scale_stride + bk] = fp8_power(e);
}

// At most 16 MT rows: a workgroup has sixteen outputs (fp8_few.h).  The products' sums keep everything, for bf16 results too: with the 8-bit instruction (fp8_tile.h) 54 rows, 1283 outputs of 5136
// columns take 14.7 us a call instead of 14.9, 32 rows, 8192 x 8192 25.4 instead of 27.1, and lose what is small beside products that cancel.
template <int MT, int X>
__global__ __launch_bounds__(1024) void fp8_few_kernel(Fp8TileArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __align__(16) float few_lds[];                   // [wave][MT][FP8_FEW_PIECE]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6, l16 = lane & 15, lq = lane >> 4;
    const int n0 = blockIdx.x * 16, blocks = (a.K + FP8_BLOCK - 1) / FP8_BLOCK;
    constexpr int es = X == FP8_X_CODES ? 1 : X == FP8_X_BF16 ? 2 : 4;
    const auto from_w = buf(a.w + (long long)n0 * a.w_stride, (unsigned)((min(16, a.N - n0) - 1) * a.w_stride + a.K));
    const auto from_x = buf(a.x, (unsigned)(((a.M - 1) * a.x_stride + a.K) * es));
    const unsigned w_row = n0 + l16 < a.N ? (unsigned)(l16 * a.w_stride) : FP8_FEW_NO_ROW;
    unsigned x_row[MT];
#pragma unroll
    for (int b = 0; b < MT; ++b) x_row[b] = b * 16 + l16 < a.M ? (unsigned)((b * 16 + l16) * a.x_stride * es) : FP8_FEW_NO_ROW;
    const float* const ws = a.w_scale + (long long)(n0 / FP8_BLOCK) * blocks;
    // what is added to a lane's first result: asked for at the start, not behind the sums
    auto added = [&](int i) {
        const int n = n0 + (i & 15), m = i >> 4;
        float v = 0.f;
        if (m >= a.M || n >= a.N) return v;
        if (a.bias) v += fp8_value(a.bias, a.bias_f32, n);
        if (a.residual) v += fp8_value(a.residual, a.y_f32, m * a.residual_stride + n);
        return v;
    };
    const float first = added(tid);
    f32x4_t acc[MT];
#pragma unroll
    for (int b = 0; b < MT; ++b) acc[b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // a block's weights are on their way while the one before is worked on (rows that are codes too: 32 rows, 8192 x 8192: 8 % slower)
    Fp8FewWeights w;
    if (wave < blocks) w.ld(from_w, w_row, ws, wave, lq, a.K);
    for (int kb = wave; kb < blocks; kb += waves) {
        Fp8Operand<true> v;
        const float wk = w.scale;
        v.of(w.lo, w.hi);
        if (kb + waves < blocks) w.ld(from_w, w_row, ws, kb + waves, lq, a.K);
        Fp8FewCodes c[X == FP8_X_CODES ? MT : 1];
        if constexpr (X == FP8_X_CODES)
#pragma unroll
            for (int b = 0; b < MT; ++b) c[b].ld(from_x, x_row[b], a.x_scale + kb * a.x_scale_stride, b * 16 + l16, b * 16 + l16 < a.M, kb, lq, a.K);
#pragma unroll
        for (int b = 0; b < MT; ++b) {
            Fp8Operand<true> x;
            float xk;
            if constexpr (X == FP8_X_CODES) { x.of(c[b].lo, c[b].hi); xk = c[b].scale; }
            else fp8_few_rows<X>(from_x, x_row[b], kb, lq, a.K, x, xk);
            const f32x4_t p = fp8_product(v, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[b][i] = fmaf(p[i], xk * wk, acc[b][i]);
        }
    }
#pragma unroll
    for (int b = 0; b < MT; ++b) *reinterpret_cast<f32x4_t*>(few_lds + (wave * MT + b) * FP8_FEW_PIECE + (lq * 17 + l16) * 4) = acc[b];
    __syncthreads();
    for (int i = tid; i < a.M * 16; i += blockDim.x) {
        const int n = i & 15, m = i >> 4;
        if (n0 + n >= a.N) continue;
        float v = 0.f;
        for (int k = 0; k < waves; ++k) v += few_lds[(k * MT + (m >> 4)) * FP8_FEW_PIECE + fp8_few_at(n, m & 15)];
        v += i == tid ? first : added(i);
        if (a.y_f32) reinterpret_cast<float*>(a.y)[m * a.y_stride + n0 + n] = v;
        else reinterpret_cast<bf16_t*>(a.y)[m * a.y_stride + n0 + n] = f2bf(v);
    }
#endif
}
template <int MT, int X> static int launch_few(const Fp8TileArgs& a, int waves, const char* fn, hipStream_t st) {
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&fp8_few_kernel<MT, X>), hipFuncAttributeMaxDynamicSharedMemorySize, 16 * MT * FP8_FEW_PIECE * 4);
    if (attr != hipSuccess) return fail(FISE_ERR_HIP, "%s: cannot raise the dynamic LDS limit", fn);
    hipLaunchKernelGGL((fp8_few_kernel<MT, X>), dim3((unsigned)ceil_div(a.N, 16)), dim3(64u * waves), (size_t)waves * MT * FP8_FEW_PIECE * 4, st, a);
    FISE_CHECK_LAUNCH(fn);
    return FISE_OK;
}
// (a launch has fewer than 2^32 lanes: more rows go in several)
static int fp8_rows(const char* fn, const void* x, int dtype, long long x_stride, int M, int K, int written, unsigned char* codes, long long code_stride, float* scale,
                    long long scale_stride, hipStream_t st) {
    const int units = (K + FP8_BLOCK - 1) / FP8_BLOCK * 16, step = std::max(1, (1 << 30) / units);
    for (int r0 = 0; r0 < M; r0 += std::min(step, M - r0)) {
        const int rows = std::min(step, M - r0);
        const dim3 grid((unsigned)(((long long)rows * units + 255) / 256));
        unsigned char* const c = codes + r0 * code_stride;
        if (dtype == FISE_F32) hipLaunchKernelGGL(fp8_rows_kernel<float>, grid, dim3(256), 0, st, (const float*)x + r0 * x_stride, x_stride, rows, K, units, written, c, code_stride, scale + r0, scale_stride);
        else hipLaunchKernelGGL(fp8_rows_kernel<bf16_t>, grid, dim3(256), 0, st, (const bf16_t*)x + r0 * x_stride, x_stride, rows, K, units, written, c, code_stride, scale + r0, scale_stride);
        FISE_CHECK_LAUNCH(fn);
    }
    return FISE_OK;
}

}  // namespace fise

using namespace fise;

extern "C" int fise_fp8_quantize(const void* x, int dtype, int64_t x_stride, int M, int K, int block_rows, uint8_t* codes, int64_t code_stride, float* scale, int64_t scale_stride,
                                 void* stream) {
    const char* fn = "fise_fp8_quantize";
    if (!x || !codes || !scale) return fail(FISE_ERR_NULL, "%s: null pointer", fn);
    if (dtype != FISE_F32 && dtype != FISE_BF16) return fail(FISE_ERR_DTYPE, "%s: dtype %d", fn, dtype);
    if (M < 0 || K < 1 || M > 1 << 30 || K > 1 << 20 || (block_rows != 1 && block_rows != 128)) return fail(FISE_ERR_SHAPE, "%s: M=%d K=%d, blocks of %d rows (1 or 128)", fn, M, K, block_rows);
    const long long blocks = (K + FP8_BLOCK - 1) / FP8_BLOCK;
    if (x_stride < K || code_stride < K || scale_stride < (block_rows == 1 ? M : blocks))
        return fail(FISE_ERR_SHAPE, "%s: strides x %lld, codes %lld, scales %lld", fn, (long long)x_stride, (long long)code_stride, (long long)scale_stride);
    if (K % 8 || x_stride % 8 || code_stride % 8 || !aligned16(x) || ((uintptr_t)codes & 7) || ((uintptr_t)scale & 3))
        return fail(FISE_ERR_ALIGN, "%s: K and the strides of x and of the codes must be multiples of 8, x 16-byte, codes 8-byte aligned", fn);
    if (M == 0) return FISE_OK;
    if (block_rows == 1) return fp8_rows(fn, x, dtype, x_stride, M, K, K, codes, code_stride, scale, scale_stride, as_stream(stream));
    const int high = (int)(((long long)M + 127) / 128), step = (int)std::max<long long>(1, (1 << 22) / blocks);      // rows of blocks, and those of a launch
    for (int b0 = 0; b0 < high; b0 += std::min(step, high - b0)) {
        const long long r0 = (long long)b0 * FP8_BLOCK;
        const dim3 grid((unsigned)(std::min(step, high - b0) * blocks));
        const int rows = (int)(M - r0);
        uint8_t* const c = codes + r0 * code_stride;
        float* const s = scale + b0 * scale_stride;
        if (dtype == FISE_F32) hipLaunchKernelGGL(fp8_block_kernel<float>, grid, dim3(256), 0, as_stream(stream), (const float*)x + r0 * x_stride, (long long)x_stride, rows, K, (int)blocks, c, (long long)code_stride, s, (long long)scale_stride);
        else hipLaunchKernelGGL(fp8_block_kernel<bf16_t>, grid, dim3(256), 0, as_stream(stream), (const bf16_t*)x + r0 * x_stride, (long long)x_stride, rows, K, (int)blocks, c, (long long)code_stride, s, (long long)scale_stride);
        FISE_CHECK_LAUNCH(fn);
    }
    return FISE_OK;
}

static int fp8_linear_sizes(const char* fn, const fise_fp8_linear_args* g) {
    if (g->x_dtype != FISE_F32 && g->x_dtype != FISE_BF16 && g->x_dtype != FISE_E4M3) return fail(FISE_ERR_DTYPE, "%s: dtype of x %d", fn, g->x_dtype);
    if (g->M < 0 || g->N < 1 || g->K < 1 || g->M > 1 << 20 || g->N > 1 << 20 || g->K > 1 << 20) return fail(FISE_ERR_SHAPE, "%s: M=%d N=%d K=%d", fn, g->M, g->N, g->K);
    return FISE_OK;
}

extern "C" size_t fise_fp8_linear_workspace_bytes(const fise_fp8_linear_args* g) {
    const char* fn = "fise_fp8_linear";
    if (!g) { fail(FISE_ERR_NULL, "%s: null pointer", fn); return 0; }
    if (fp8_linear_sizes(fn, g)) return 0;
    return fp8_choose(g->M, g->N, g->K, g->y_dtype == FISE_F32, g->x_dtype == FISE_E4M3).make_rows ? (size_t)fp8_space(g->M, g->K).bytes : 0;
}

extern "C" int fise_fp8_linear(const fise_fp8_linear_args* g, void* workspace, size_t workspace_bytes, void* stream) {
    const char* fn = "fise_fp8_linear";
    if (!g || !g->x || !g->w || !g->w_scale || !g->y) return fail(FISE_ERR_NULL, "%s: null pointer", fn);
    if (int e = fp8_linear_sizes(fn, g)) return e;
    auto known = [](int d) { return d == FISE_F32 || d == FISE_BF16; };
    if (!known(g->y_dtype) || (g->bias && !known(g->bias_dtype))) return fail(FISE_ERR_DTYPE, "%s: dtypes y %d, bias %d", fn, g->y_dtype, g->bias_dtype);
    const bool codes = g->x_dtype == FISE_E4M3;
    if (codes != (g->x_scale != nullptr)) return fail(FISE_ERR_NULL, "%s: codes have scales, other rows have none", fn);
    if (g->x_stride < g->K || g->w_stride < g->K || g->y_stride < g->N || (g->residual && g->residual_stride < g->N) || (codes && g->x_scale_stride < g->M) || g->x_stride > 1 << 22 || g->w_stride > 1 << 22)
        return fail(FISE_ERR_SHAPE, "%s: M=%d N=%d K=%d, strides x %lld, its scales %lld, w %lld, y %lld, residual %lld", fn, g->M, g->N, g->K, (long long)g->x_stride, (long long)g->x_scale_stride,
                    (long long)g->w_stride, (long long)g->y_stride, (long long)g->residual_stride);
    if (g->K % 16 || g->w_stride % 16 || g->x_stride % (codes ? 16 : 8) || !aligned16(g->x) || !aligned16(g->w))
        return fail(FISE_ERR_ALIGN, "%s: K and the strides of codes must be multiples of 16, that of other x of 8, x and w 16-byte aligned", fn);
    const size_t ye = g->y_dtype == FISE_F32 ? 4 : 2, be = g->bias_dtype == FISE_F32 ? 4 : 2;
    if ((uintptr_t)g->y % ye || (uintptr_t)g->residual % ye || (g->bias && (uintptr_t)g->bias % be) || ((uintptr_t)g->x_scale | (uintptr_t)g->w_scale) & 3)
        return fail(FISE_ERR_ALIGN, "%s: y, residual, bias and scales must be aligned to their type", fn);
    const Fp8Choice c = fp8_choose(g->M, g->N, g->K, g->y_dtype == FISE_F32, codes);
    const Fp8Space space = c.make_rows ? fp8_space(g->M, g->K) : Fp8Space{};
    if (space.bytes && (!workspace || workspace_bytes < (size_t)space.bytes)) return fail(FISE_ERR_CAPACITY, "%s: workspace of %zu bytes, %lld needed", fn, workspace ? workspace_bytes : 0, (long long)space.bytes);
    if (space.bytes && ((uintptr_t)workspace & 255)) return fail(FISE_ERR_ALIGN, "%s: workspace must be 256-byte aligned", fn);
    if (c.m_tiles * c.n_tiles >= 1 << 23) return fail(FISE_ERR_SHAPE, "%s: M=%d N=%d: more tiles than a launch holds", fn, g->M, g->N);
    if (g->M == 0) return FISE_OK;
    const hipStream_t st = as_stream(stream);
    Fp8TileArgs a{};
    a.x = (const unsigned char*)g->x; a.x_stride = g->x_stride; a.x_scale = g->x_scale; a.x_scale_stride = g->x_scale_stride;
    if (c.make_rows) {
        float* const scale = (float*)((unsigned char*)workspace + space.scale_off);
        if (int e = fp8_rows(fn, g->x, g->x_dtype, g->x_stride, g->M, g->K, (int)space.stride, (unsigned char*)workspace, space.stride, scale, g->M, st)) return e;
        a.x = (const unsigned char*)workspace; a.x_stride = space.stride; a.x_scale = scale; a.x_scale_stride = g->M;
    }
    a.w = g->w; a.w_stride = g->w_stride; a.w_scale = g->w_scale;
    a.M = g->M; a.N = g->N; a.K = g->K; a.m_tiles = (int)c.m_tiles; a.n_tiles = (int)c.n_tiles;
    a.bias = g->bias; a.bias_f32 = g->bias_dtype == FISE_F32; a.residual = g->residual; a.residual_stride = g->residual_stride;
    a.y = g->y; a.y_stride = g->y_stride; a.y_f32 = g->y_dtype == FISE_F32;
    ProfileScope prof(c.form == FP8_FORM_FEW ? PROF_ROWS_GEMM : PROF_IGEMM_WIDE, 2.0 * g->M * g->N * g->K, (double)g->N * g->K + (double)g->M * g->K + (double)g->M * g->N * ye, st);
    switch (c.form) {
        case FP8_FORM_256: return launch_fp8_tile<8, 4, 2, 4, FP8_LINEAR>(a, fn, st);
        case FP8_FORM_128: return a.y_f32 ? launch_fp8_tile<4, 4, 2, 2, FP8_LINEAR, true>(a, fn, st) : launch_fp8_tile<4, 4, 2, 2, FP8_LINEAR>(a, fn, st);
        case FP8_FORM_64: return a.y_f32 ? launch_fp8_tile<2, 4, 4, 1, FP8_LINEAR, true>(a, fn, st) : launch_fp8_tile<2, 4, 4, 1, FP8_LINEAR>(a, fn, st);
        case FP8_FORM_32: return a.y_f32 ? launch_fp8_tile<2, 2, 4, 1, FP8_LINEAR, true>(a, fn, st) : launch_fp8_tile<2, 2, 4, 1, FP8_LINEAR>(a, fn, st);
        default:
            if (!codes && !c.make_rows) return g->x_dtype == FISE_F32 ? launch_few<1, FP8_X_F32>(a, c.waves, fn, st) : launch_few<1, FP8_X_BF16>(a, c.waves, fn, st);
            return a.M <= 16 ? launch_few<1, FP8_X_CODES>(a, c.waves, fn, st) : a.M <= 32 ? launch_few<2, FP8_X_CODES>(a, c.waves, fn, st) : launch_few<4, FP8_X_CODES>(a, c.waves, fn, st);
    }
}
