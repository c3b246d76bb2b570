// The feed-forward of the chosen experts: h = silu(Wg x) * (Wu x) and Wo h for every pair (token, expert) in the experts' order, then a token's weighted sum.
//
// A few tokens: two launches that stream the weights past them (fp8_few.h), a workgroup a pair, then a token, h in float in between.  (Rows of an expert streamed past like that, 64 tokens of
// 6 among 64 experts: 303 us, 124 on tiles.)  More: four launches: rows of x into 8 bits, with the tables of tiles (a tile has rows of one expert); gate and up of a tile side by side in a wave, so that h leaves the
// accumulators in 8 bits with the scale of its 128 channels; Wo; and the sum, which reads a pair's row where it is in the experts' order (rows stored where the pair is among
// the tokens, 131072 rows of 4096: 1219 us instead of 1133).  No atomics: a result depends on its arguments only.
// Gate and up have exact sums (fp8_tile.h): h is put in 8 bits, and a code next to a border is moved by very little.
// One token, 2 of 16 experts, 1280 x 640: 9.2 us; 64 tokens, 6 of 64, 2048 x 1408: 124 us, 4.5 TB/s of weights; 16384 tokens, 8 of 64, 4096 x 1536: 4.55 ms, 1.1 PFLOP/s (gate and up 3.25 ms, 1.0 PFLOP/s of a
// library's 1.2 - 1.36 in bf16, the second product 1.0, the sum 0.28).
#include "fp8_few.h"
#include "fp8_choice.h"

namespace fise {

struct ExpertsArgs {
    const void* x; long long x_stride; int T, K, units;
    unsigned char* codes; long long code_stride; float* scale;
    const int* offsets; int E, pairs;
    int tables, bm[2], m_tiles[2]; int* table[2];                      // of the second product, and of gate and up where theirs is another
    const int* slots; int* place;                                      // place[pair]: where it is in the experts' order
    int place_blocks;
};

// table[2 t] = first row of tile t in the experts' order, table[2 t + 1] = expert << 16 | rows (0: no such tile).  Offsets that do not ascend or leave 0..pairs count as the nearest that do not.
__device__ void experts_table(const ExpertsArgs& a, int bm, int m_tiles, int* table) {
    __shared__ int sums[2][4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (a.E + 255) / 256, e0 = min(tid * each, a.E), e1 = min(e0 + each, a.E);
    // the offsets' running maximum
    int top = 0;
    for (int e = e0; e < e1; ++e) top = max(top, min(max(a.offsets[e], 0), a.pairs));
    int before = top;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int n = __shfl_up(before, o); if (lane >= o) before = max(before, n); }
    if (lane == 63) sums[0][wave] = before;
    __syncthreads();
    before = __shfl_up(before, 1);
    if (lane == 0) before = 0;
    for (int w = 0; w < wave; ++w) before = max(before, sums[0][w]);
    auto tiles_from = [&](int at, bool write) {
        int start = before;
        for (int e = e0; e < e1; ++e) {
            start = max(start, min(max(a.offsets[e], 0), a.pairs));
            const int end = max(start, min(max(a.offsets[e + 1], 0), a.pairs));
            for (int r = start; r < end; r += bm, ++at)
                if (write && at < m_tiles) { table[2 * at] = r; table[2 * at + 1] = e << 16 | min(bm, end - r); }
        }
        return at;
    };
    int n = tiles_from(0, false), upto = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int m = __shfl_up(upto, o); if (lane >= o) upto += m; }
    if (lane == 63) sums[1][wave] = upto;
    __syncthreads();
    int at = upto - n, all = 0;
    for (int w = 0; w < 4; ++w) { if (w < wave) at += sums[1][w]; all += sums[1][w]; }
    tiles_from(at, true);
    for (int t = all + tid; t < m_tiles; t += 256) { table[2 * t] = 0; table[2 * t + 1] = 0; }
}

template <typename T> __global__ __launch_bounds__(256) void experts_rows_kernel(ExpertsArgs a) {
    const int block = (int)blockIdx.x - a.tables;
    if (block < 0) {
        const int w = blockIdx.x;
        experts_table(a, w ? a.bm[1] : a.bm[0], w ? a.m_tiles[1] : a.m_tiles[0], w ? a.table[1] : a.table[0]);
        return;
    }
    if (block < a.place_blocks) {
        const int s = block * 256 + threadIdx.x;
        if (s < min(max(a.offsets[a.E], 0), a.pairs)) {
            const int p = a.slots[s];
            if ((unsigned)p < (unsigned)a.pairs) a.place[p] = s;
        }
        return;
    }
    fp8_quantize_unit((const T*)a.x, a.x_stride, a.T, a.K, a.units, a.units * 8, a.codes, a.code_stride, a.scale, (long long)a.T, (long long)(block - a.place_blocks) * 256 + threadIdx.x);
}

// ---- a few tokens ----
// silu(gate) * up of sixteen channels of one pair, the token in the first of the product's sixteen rows.
template <int X>
__global__ __launch_bounds__(1024) void experts_token_in_kernel(ExpertsFewArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __align__(16) float few_lds[];                   // [wave][gate, up][16]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6, l16 = lane & 15, lq = lane >> 4;
    const int i0 = blockIdx.x * 16, p = blockIdx.y, blocks = (a.K + FP8_BLOCK - 1) / FP8_BLOCK, i_blocks = (a.I + FP8_BLOCK - 1) / FP8_BLOCK;
    const int expert = __builtin_amdgcn_readfirstlane(a.ids[p]);
    if ((unsigned)expert >= (unsigned)a.E) return;
    constexpr int es = X == FP8_X_BF16 ? 2 : 4;
    const unsigned char* const wg = a.w_in + ((long long)expert * 2 * a.I + i0) * a.K;
    const unsigned w_bytes = (unsigned)(min(16, a.I - i0) * a.K);
    const auto from_g = buf(wg, w_bytes), from_u = buf(wg + (long long)a.I * a.K, w_bytes), from_x = buf(a.x, a.x_bytes);
    const unsigned w_row = i0 + l16 < a.I ? (unsigned)(l16 * a.K) : FP8_FEW_NO_ROW, x_row = l16 == 0 ? (unsigned)(p / a.k * a.x_stride * es) : FP8_FEW_NO_ROW;
    const float* const sg = a.w_in_scale + ((long long)expert * 2 * i_blocks + i0 / FP8_BLOCK) * blocks;
    const float* const su = sg + (long long)i_blocks * blocks;
    f32x4_t acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    Fp8FewWeights g, u;
    if (wave < blocks) { g.ld(from_g, w_row, sg, wave, lq, a.K); u.ld(from_u, w_row, su, wave, lq, a.K); }
    for (int kb = wave; kb < blocks; kb += waves) {
        Fp8Operand<true> vg, vu, x;
        vg.of(g.lo, g.hi);
        vu.of(u.lo, u.hi);
        const float kg = g.scale, ku = u.scale;
        if (kb + waves < blocks) { g.ld(from_g, w_row, sg, kb + waves, lq, a.K); u.ld(from_u, w_row, su, kb + waves, lq, a.K); }
        float xk;
        fp8_few_rows<X>(from_x, x_row, kb, lq, a.K, x, xk);
        const f32x4_t q = fp8_product(vg, x), r = fp8_product(vu, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) { acc[0][i] = fmaf(q[i], xk * kg, acc[0][i]); acc[1][i] = fmaf(r[i], xk * ku, acc[1][i]); }
    }
    if (l16 == 0)
#pragma unroll
        for (int j = 0; j < 2; ++j) *reinterpret_cast<f32x4_t*>(few_lds + (wave * 2 + j) * 16 + lq * 4) = acc[j];
    __syncthreads();
    if (tid < 16 && i0 + tid < a.I) {
        float gate = 0.f, up = 0.f;
        for (int k = 0; k < waves; ++k) { gate += few_lds[k * 32 + tid]; up += few_lds[k * 32 + 16 + tid]; }
        a.h[(long long)p * a.I + i0 + tid] = gate / (1.f + expf(-gate)) * up;
    }
#endif
}
// Sixteen outputs of one token, all its experts: the waves share (place, block of columns).
__global__ __launch_bounds__(1024) void experts_token_out_kernel(ExpertsFewArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __align__(16) float few_lds[];                   // [wave][16]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6, l16 = lane & 15, lq = lane >> 4;
    const int n0 = blockIdx.x * 16, t = blockIdx.y, blocks = (a.I + FP8_BLOCK - 1) / FP8_BLOCK, n_blocks = (a.N + FP8_BLOCK - 1) / FP8_BLOCK;
    const auto from_h = buf(a.h, a.h_bytes);
    const unsigned w_row = n0 + l16 < a.N ? (unsigned)(l16 * a.I) : FP8_FEW_NO_ROW;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    for (int it = wave; it < a.k * blocks; it += waves) {
        const int j = it / blocks, kb = it - j * blocks, p = t * a.k + j, expert = __builtin_amdgcn_readfirstlane(a.ids[p]);
        if ((unsigned)expert >= (unsigned)a.E) continue;
        const auto from_w = buf(a.w_out + ((long long)expert * a.N + n0) * a.I, (unsigned)(min(16, a.N - n0) * a.I));
        Fp8FewWeights w;
        w.ld(from_w, w_row, a.w_out_scale + ((long long)expert * n_blocks + n0 / FP8_BLOCK) * blocks, kb, lq, a.I);
        Fp8Operand<true> v, x;
        float xk;
        fp8_few_rows<FP8_X_F32>(from_h, l16 == 0 ? (unsigned)p * (unsigned)(a.I * 4) : FP8_FEW_NO_ROW, kb, lq, a.I, x, xk);
        v.of(w.lo, w.hi);
        const f32x4_t r = fp8_product(v, x);
        const float f = a.weights[p];
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = fmaf(f, r[i] * (xk * w.scale), acc[i]);
    }
    if (l16 == 0) *reinterpret_cast<f32x4_t*>(few_lds + wave * 16 + lq * 4) = acc;
    __syncthreads();
    if (tid < 16 && n0 + tid < a.N) {
        const int n = n0 + tid;
        float v = a.residual ? fp8_value(a.residual, a.y_f32, t * a.residual_stride + n) : 0.f;
        for (int j = 0; j < a.k; ++j) if ((unsigned)a.ids[t * a.k + j] >= (unsigned)a.E) v = fmaf(a.weights[t * a.k + j], 0.f, v);
        for (int k = 0; k < waves; ++k) v += few_lds[k * 16 + tid];
        if (a.y_f32) reinterpret_cast<float*>(a.y)[t * a.y_stride + n] = v;
        else reinterpret_cast<bf16_t*>(a.y)[t * a.y_stride + n] = f2bf(v);
    }
#endif
}

// ---- the sum ----
struct ExpertsSum {
    const void* rows; const unsigned char* row_exp; const int* place; int pairs; const int* ids; const float* weights; const void* residual; long long residual_stride; void* y; long long y_stride;
    int T, k, N, units, share;                                         // share: outputs with one power of two
};
template <typename T> __global__ __launch_bounds__(256) void experts_sum_kernel(ExpertsSum a) {
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x, t = id / a.units;
    const int n = (int)(id - t * a.units) * 8;
    if (t >= a.T) return;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.residual) fp8_load8((const T*)a.residual + t * a.residual_stride + n, v);
    for (int j = 0; j < a.k; ++j) {
        const long long p = t * a.k + j;
        const float w = a.weights[p];
        float r[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        const long long at = a.ids[p] >= 0 ? a.place[p] : -1;
        if (at >= 0 && at < a.pairs) {
            if constexpr (sizeof(T) == 4) fp8_load8((const float*)a.rows + at * a.N + n, r);
            else {                                                     // 16-bit floats times a power of two (fp8_tile.h)
                const f16x8_t half = *reinterpret_cast<const f16x8_t*>((const _Float16*)a.rows + at * a.N + n);
                const float f = fp8_power((int)a.row_exp[at * ((a.N + a.share - 1) / a.share) + n / a.share] - 127);
#pragma unroll
                for (int i = 0; i < 8; ++i) r[i] = (float)half[i] * f;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(w, r[i], v[i]);
    }
    T* const y = (T*)a.y + t * a.y_stride + n;
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<f32x4_t*>(y) = f32x4_t{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4_t*>(y + 4) = f32x4_t{v[4], v[5], v[6], v[7]};
    } else *reinterpret_cast<u32x4_t*>(y) = u32x4_t{f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7])};
}

static int expert_sizes(const char* fn, const fise_expert_mlp_args* g) {
    if ((g->x_dtype != FISE_F32 && g->x_dtype != FISE_BF16) || (g->y_dtype != FISE_F32 && g->y_dtype != FISE_BF16)) return fail(FISE_ERR_DTYPE, "%s: dtypes x %d, y %d", fn, g->x_dtype, g->y_dtype);
    if (g->T < 0 || g->K < 1 || g->I < 1 || g->N < 1 || g->K > 1 << 16 || g->I > 1 << 16 || g->N > 1 << 16 || g->E < 1 || g->E > 1024 || g->k < 1 || g->k > 64)
        return fail(FISE_ERR_SHAPE, "%s: T=%d K=%d I=%d N=%d E=%d k=%d", fn, g->T, g->K, g->I, g->N, g->E, g->k);
    if ((long long)g->T * g->k >= 1 << 24 || (long long)g->T * ((g->K + 127) / 128 * 128) >= 1 << 30)
        return fail(FISE_ERR_SHAPE, "%s: T=%d k=%d K=%d: T k below 2^24, T K below 2^30", fn, g->T, g->k, g->K);
    if (g->K % 16 || g->I % 16 || g->N % 8) return fail(FISE_ERR_ALIGN, "%s: K=%d, I=%d must be multiples of 16, N=%d of 8", fn, g->K, g->I, g->N);
    return FISE_OK;
}

}  // namespace fise

using namespace fise;

extern "C" size_t fise_expert_mlp_workspace_bytes(const fise_expert_mlp_args* g) {
    const char* fn = "fise_expert_mlp";
    if (!g) { fail(FISE_ERR_NULL, "%s: null pointer", fn); return 0; }
    if (expert_sizes(fn, g)) return 0;
    return (size_t)expert_choose(g->T, g->K, g->I, g->N, g->E, g->k, g->x_stride * (g->x_dtype == FISE_F32 ? 4 : 2), g->y_dtype == FISE_F32 ? 4 : 2).bytes;
}

extern "C" int fise_expert_mlp(const fise_expert_mlp_args* g, void* workspace, size_t workspace_bytes, void* stream) {
    const char* fn = "fise_expert_mlp";
    if (!g || !g->x || !g->ids || !g->weights || !g->offsets || !g->slots || !g->w_in || !g->w_in_scale || !g->w_out || !g->w_out_scale || !g->y) return fail(FISE_ERR_NULL, "%s: null pointer", fn);
    if (int e = expert_sizes(fn, g)) return e;
    if (g->x_stride < g->K || g->y_stride < g->N || (g->residual && g->residual_stride < g->N))
        return fail(FISE_ERR_SHAPE, "%s: strides x %lld, y %lld, residual %lld", fn, (long long)g->x_stride, (long long)g->y_stride, (long long)g->residual_stride);
    if (g->x_stride % 8 || g->y_stride % 8 || (g->residual && g->residual_stride % 8) || !aligned16(g->x) || !aligned16(g->y) || !aligned16(g->residual) || !aligned16(g->w_in) || !aligned16(g->w_out) ||
        ((uintptr_t)g->ids | (uintptr_t)g->weights | (uintptr_t)g->offsets | (uintptr_t)g->slots | (uintptr_t)g->w_in_scale | (uintptr_t)g->w_out_scale) & 3)
        return fail(FISE_ERR_ALIGN, "%s: rows and codes must be 16-byte aligned, strides multiples of 8, lists and scales aligned to their type", fn);
    const int es = g->y_dtype == FISE_F32 ? 4 : 2, xs = g->x_dtype == FISE_F32 ? 4 : 2;
    const ExpertChoice c = expert_choose(g->T, g->K, g->I, g->N, g->E, g->k, g->x_stride * xs, es);
    if (g->T && (!workspace || workspace_bytes < (size_t)c.bytes)) return fail(FISE_ERR_CAPACITY, "%s: workspace of %zu bytes, %lld needed", fn, workspace ? workspace_bytes : 0, (long long)c.bytes);
    if ((uintptr_t)workspace & 255) return fail(FISE_ERR_ALIGN, "%s: workspace must be 256-byte aligned", fn);
    if ((long long)g->T * g->N >= 1LL << 34) return fail(FISE_ERR_SHAPE, "%s: T=%d N=%d: more results than a launch holds", fn, g->T, g->N);
    if (g->T == 0) return FISE_OK;
    ExpertsSum s{};
    s.ids = g->ids; s.weights = g->weights; s.residual = g->residual; s.residual_stride = g->residual_stride; s.y = g->y; s.y_stride = g->y_stride;
    s.T = g->T; s.k = g->k; s.N = g->N; s.units = g->N / 8;
    const dim3 sum_grid((unsigned)(((long long)g->T * s.units + 255) / 256));
    const hipStream_t st = as_stream(stream);
    if (c.form == EXPERTS_TOKENS) {
        ExpertsFewArgs f{};
        f.x = g->x; f.x_stride = g->x_stride; f.x_bytes = (unsigned)(((g->T - 1) * g->x_stride + g->K) * xs);
        f.ids = g->ids; f.weights = g->weights; f.T = g->T; f.k = g->k; f.E = g->E; f.K = g->K; f.I = g->I; f.N = g->N;
        f.w_in = g->w_in; f.w_in_scale = g->w_in_scale; f.w_out = g->w_out; f.w_out_scale = g->w_out_scale;
        f.h = (float*)workspace; f.h_bytes = (unsigned)((long long)g->T * g->k * g->I * 4);
        f.residual = g->residual; f.residual_stride = g->residual_stride; f.y = g->y; f.y_stride = g->y_stride; f.y_f32 = es == 4;
        const int n = g->T * g->k;
        {
            ProfileScope prof(PROF_ROWS_GEMM, 4.0 * n * g->I * g->K, 2.0 * n * g->I * g->K + 4.0 * n * g->I, st);
            const dim3 grid((unsigned)ceil_div(g->I, 16), (unsigned)n), block(64u * c.waves_in);
            if (xs == 4) hipLaunchKernelGGL((experts_token_in_kernel<FP8_X_F32>), grid, block, (size_t)c.waves_in * 128, st, f);
            else hipLaunchKernelGGL((experts_token_in_kernel<FP8_X_BF16>), grid, block, (size_t)c.waves_in * 128, st, f);
            FISE_CHECK_LAUNCH(fn);
        }
        ProfileScope prof(PROF_ROWS_GEMM, 2.0 * n * g->I * g->N, (double)n * g->I * (g->N + 4.0), st);
        hipLaunchKernelGGL(experts_token_out_kernel, dim3((unsigned)ceil_div(g->N, 16), (unsigned)g->T), dim3(64u * c.waves_out), (size_t)c.waves_out * 64, st, f);
        FISE_CHECK_LAUNCH(fn);
        return FISE_OK;
    }
    const int blocks_i = (g->I + FP8_BLOCK - 1) / FP8_BLOCK, blocks_k = (g->K + FP8_BLOCK - 1) / FP8_BLOCK, blocks_n = (g->N + FP8_BLOCK - 1) / FP8_BLOCK, n_tiles = ceil_div(g->N, c.bm == 32 ? 128 : 256);      // (32 rows: more workgroups on their way at once)
    unsigned char* const ws = (unsigned char*)workspace;
    const int pairs = g->T * g->k;
    ExpertsArgs r{};
    r.x = g->x; r.x_stride = g->x_stride; r.T = g->T; r.K = g->K; r.units = blocks_k * 16; r.codes = ws; r.code_stride = c.x_stride; r.scale = (float*)(ws + c.x_scale_off);
    r.offsets = g->offsets; r.E = g->E; r.pairs = pairs;
    r.tables = c.bm_in == c.bm ? 1 : 2;
    r.bm[0] = c.bm; r.m_tiles[0] = (int)c.m_tiles; r.table[0] = (int*)(ws + c.table_off);
    r.bm[1] = c.bm_in; r.m_tiles[1] = (int)c.m_tiles_in; r.table[1] = (int*)(ws + c.table_in_off);
    r.slots = g->slots; r.place = (int*)(ws + c.place_off); r.place_blocks = ceil_div(pairs, 256);
    const dim3 rows_grid((unsigned)(r.tables + r.place_blocks + ((long long)g->T * r.units + 255) / 256));
    if (g->x_dtype == FISE_F32) hipLaunchKernelGGL(experts_rows_kernel<float>, rows_grid, dim3(256), 0, st, r);
    else hipLaunchKernelGGL(experts_rows_kernel<bf16_t>, rows_grid, dim3(256), 0, st, r);
    FISE_CHECK_LAUNCH(fn);
    Fp8TileArgs a{};
    // (a launch has fewer than 2^32 lanes: more tiles go in several)
    auto tiles = [&](const int* table, int64_t n, auto launch) {
        const int64_t step = (1 << 22) / a.n_tiles;
        for (int64_t t0 = 0; t0 < n; t0 += step) {
            a.table = table + 2 * t0; a.m_tiles = (int)std::min(step, n - t0);
            if (int e = launch()) return e;
        }
        return (int)FISE_OK;
    };
    a.pairs = pairs; a.k = g->k; a.slots = g->slots; a.M = pairs;
    a.x = ws; a.x_stride = c.x_stride; a.x_bytes = (long long)g->T * c.x_stride; a.x_scale = r.scale; a.x_scale_stride = g->T;
    a.w = g->w_in; a.w_stride = g->K; a.w_expert = 2LL * g->I * g->K; a.w_scale = g->w_in_scale; a.w_scale_expert = 2 * blocks_i * blocks_k;
    a.N = g->I; a.K = g->K; a.n_tiles = blocks_i;
    a.h = ws + c.h_off; a.h_stride = c.h_stride; a.h_scale = (float*)(ws + c.h_scale_off); a.h_scale_stride = pairs;
    {
        ProfileScope prof(PROF_IGEMM_GEGLU, 4.0 * pairs * g->I * g->K, 2.0 * std::min(g->E, pairs) * g->I * g->K + (double)pairs * (g->K + g->I), st);
        if (int e = tiles(r.table[1], c.m_tiles_in, [&] { return c.bm_in == 128 ? launch_fp8_tile<4, 4, 4, 2, FP8_GATED, true>(a, fn, st) : launch_fp8_tile<4, 2, 4, 1, FP8_GATED, true>(a, fn, st); })) return e;
    }
    a.x = a.h; a.x_stride = c.h_stride; a.x_scale = a.h_scale; a.x_scale_stride = pairs;
    a.w = g->w_out; a.w_stride = g->I; a.w_expert = (long long)g->N * g->I; a.w_scale = g->w_out_scale; a.w_scale_expert = blocks_n * blocks_i;
    a.N = g->N; a.K = g->I; a.n_tiles = n_tiles;
    a.y = ws + c.out_off; a.y_stride = g->N; a.y_f32 = es == 4; a.row_exp = ws + c.row_exp_off;
    {
        ProfileScope prof(PROF_IGEMM_WIDE, 2.0 * pairs * g->I * g->N, (double)std::min(g->E, pairs) * g->I * g->N + (double)pairs * (g->I + g->N * es), st);
        if (int e = tiles(r.table[0], c.m_tiles, [&] {
                return c.bm == 256 ? launch_fp8_tile<8, 4, 2, 4, FP8_PAIRS>(a, fn, st) : c.bm == 128 ? launch_fp8_tile<4, 4, 4, 2, FP8_PAIRS, true>(a, fn, st) : launch_fp8_tile<2, 2, 4, 1, FP8_PAIRS, true>(a, fn, st); }))
            return e;
    }
    s.rows = a.y; s.row_exp = a.row_exp; s.place = r.place; s.pairs = pairs; s.share = c.bm == 32 ? 32 : 64;
    if (es == 4) hipLaunchKernelGGL((experts_sum_kernel<float>), sum_grid, dim3(256), 0, st, s);
    else hipLaunchKernelGGL((experts_sum_kernel<bf16_t>), sum_grid, dim3(256), 0, st, s);
    FISE_CHECK_LAUNCH(fn);
    return FISE_OK;
}
