// The norms around a block with its gate and modulation, one pass over the rows:  r = a x + gate Npost(h),  y = Npre(r) (1 + scale) + shift.
//
// A row is read once and stays in registers through both norms: x and h come in with 16-byte loads that are all requested before the first sum, r and y go
// out, and nothing else moves.  Bound by those bytes where there are many rows, else by one trip to memory and four sums over lanes.  Sums are
// float: of the values, then of the squares of what is left when the mean is taken off (no difference of large sums).  4 x 4096 rows of 4096 channels, bf16: 107 us, 5.0 TB/s;
// 2 x 768 rows of 320: 5.1 us.
#include <algorithm>
#include "igemm.h"
#include "profile.h"

namespace fise {

constexpr int NG_MAX_C = 16384;

struct GatedNorm {
    const void* x; const void* h; void* r; void* y;
    const void* post_w; const void* post_b; const void* pre_w; const void* pre_b;
    const float* gate; const float* scale; const float* shift; long long mod_stride;
    const int* tile_idx; int tile, tiles_w, HW, W, M, rows, row0, C, pieces;  // M: rows of a batch element; row0: of this launch; pieces: of eight channels
    int post, pre, h_is_map, y_is_map;
    float res_scale, eps, channels;
    FastDiv d_M, d_tt, d_tile, d_tiles_w;
};

template <typename T> struct Eight;                                    // eight neighbouring channels as they lie in memory
template <> struct Eight<bf16_t> {
    uint4 a;
    __device__ __forceinline__ void load(const bf16_t* p) { a = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        v[0] = lo16(a.x); v[1] = hi16(a.x); v[2] = lo16(a.y); v[3] = hi16(a.y); v[4] = lo16(a.z); v[5] = hi16(a.z); v[6] = lo16(a.w); v[7] = hi16(a.w);
    }
    static __device__ __forceinline__ void store(bf16_t* p, const float (&v)[8]) {
        *reinterpret_cast<uint4*>(p) = make_uint4(f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7]));
    }
};
template <> struct Eight<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
    __device__ __forceinline__ void get(float (&v)[8]) const { v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w; }
    static __device__ __forceinline__ void store(float* p, const float (&v)[8]) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
};

// Sum over the lanes of a row: one wave, or the four waves of a workgroup (`slot` alternates, so that one barrier is enough).
template <int WAVES> __device__ __forceinline__ float row_sum(float v, float* lds, int& slot) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if constexpr (WAVES > 1) {
        float* const s = lds + slot * WAVES;
        slot ^= 1;
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += s[w];
    }
    return v;
}

// WAVES: that share a row (1: four rows a workgroup); J: pieces of eight channels a lane holds.
template <typename T, int WAVES, int J>
__global__ __launch_bounds__(256) void gated_norm_kernel(const GatedNorm a) {
    __shared__ float lds[2 * WAVES];
    int slot = 0;
    constexpr int LANES = 64 * WAVES;
    const int tid = threadIdx.x, lane = WAVES > 1 ? tid : tid & 63;
    const unsigned row = a.row0 + (WAVES > 1 ? blockIdx.x : blockIdx.x * 4 + (tid >> 6));
    if (row >= (unsigned)a.rows) return;                                         // (whole waves, and with WAVES > 1 none)
    const int b = (int)fdiv(row, a.d_M), m = (int)row - b * a.M;
    int token = m;
    if (a.tile) {
        const int ti = (int)fdiv((unsigned)m, a.d_tt), p = m - ti * a.tile * a.tile, t = a.tile_idx[ti];
        const int ty = (int)fdiv((unsigned)t, a.d_tiles_w), py = (int)fdiv((unsigned)p, a.d_tile);
        token = (ty * a.tile + py) * a.W + (t - ty * a.tiles_w) * a.tile + (p - py * a.tile);
    }
    const size_t on_map = ((size_t)b * a.HW + token) * a.C, compact = (size_t)row * a.C;
    const T* const x = (const T*)a.x + on_map;
    const T* const h = a.h ? (const T*)a.h + (a.h_is_map ? on_map : compact) : nullptr;

    Eight<T> xr[J], hr[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int p = lane + j * LANES;
        if (p < a.pieces) { xr[j].load(x + p * 8); if (h) hr[j].load(h + p * 8); }
    }
    float v[J][8];
    auto has = [&](int j) { return lane + j * LANES < a.pieces; };
    // v -> v normalised, weights applied
    auto norm = [&](int kind, const void* w_, const void* b_) {
        if (kind == FISE_NORM_NONE) return;
        if (kind == FISE_NORM_LAYER) {
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (has(j))
#pragma unroll
                    for (int e = 0; e < 8; ++e) s += v[j][e];
            const float mean = row_sum<WAVES>(s, lds, slot) / a.channels;      // (a reciprocal's rounding, times 1 / std, is what would be left of a constant row)
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[j][e] -= mean;
        }
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (has(j))
#pragma unroll
                for (int e = 0; e < 8; ++e) q = fmaf(v[j][e], v[j][e], q);
        const float rs = 1.0f / sqrtf(row_sum<WAVES>(q, lds, slot) / a.channels + a.eps);
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (has(j)) {
                const int c = (lane + j * LANES) * 8;
                float w[8], bb[8];
                if (w_) { Eight<T> t; t.load((const T*)w_ + c); t.get(w); }
                if (b_) { Eight<T> t; t.load((const T*)b_ + c); t.get(bb); }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float u = v[j][e] * rs;
                    if (w_) u *= w[e];
                    if (b_) u += bb[e];
                    v[j][e] = u;
                }
            }
    };
    if (h) {
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (has(j)) hr[j].get(v[j]);
        norm(a.post, a.post_w, a.post_b);
    }
    const size_t mod = (size_t)b * a.mod_stride;
#pragma unroll
    for (int j = 0; j < J; ++j)
        if (has(j)) {
            const int c = (lane + j * LANES) * 8;
            float xv[8], g[8];
            xr[j].get(xv);
            if (a.gate) { Eight<float> t; t.load(a.gate + mod + c); t.get(g); }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float br = h ? (a.gate ? g[e] * v[j][e] : v[j][e]) : 0.f;
                v[j][e] = h ? fmaf(a.res_scale, xv[e], br) : a.res_scale * xv[e];
            }
            if (a.r) Eight<T>::store((T*)a.r + on_map + c, v[j]);
        }
    if (!a.y) return;
    norm(a.pre, a.pre_w, a.pre_b);
    T* const y = (T*)a.y + (a.y_is_map ? on_map : compact);
#pragma unroll
    for (int j = 0; j < J; ++j)
        if (has(j)) {
            const int c = (lane + j * LANES) * 8;
            float sc[8], sh[8];
            if (a.scale) { Eight<float> t; t.load(a.scale + mod + c); t.get(sc); }
            if (a.shift) { Eight<float> t; t.load(a.shift + mod + c); t.get(sh); }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float u = v[j][e];
                if (a.scale) u *= 1.0f + sc[e];
                if (a.shift) u += sh[e];
                v[j][e] = u;
            }
            Eight<T>::store(y + c, v[j]);
        }
}

template <typename T, int WAVES, int J> static int launch_gated(GatedNorm a, hipStream_t st) {
    constexpr int per = WAVES > 1 ? 1 : 4, most = 1 << 23;             // rows of a workgroup; workgroups of a launch, whose lanes are counted in 32 bits
    for (long long row0 = 0; row0 < a.rows; row0 += (long long)most * per) {
        a.row0 = (int)row0;
        hipLaunchKernelGGL((gated_norm_kernel<T, WAVES, J>), dim3((unsigned)std::min<long long>((a.rows - row0 + per - 1) / per, most)), dim3(256), 0, st, a);
        FISE_CHECK_LAUNCH("fise_masked_gated_norm");
    }
    return FISE_OK;
}
// A wave for rows of up to 512 channels, which fill its lanes once (4096 rows of 320: 6.0 us, with four waves a row 10.2; 64 rows 4.4, 4.5), else the four of a workgroup, with as
// many pieces a lane as the row has.
template <typename T> static int launch_gated(const GatedNorm& a, hipStream_t st) {
    if (a.pieces <= 64) return launch_gated<T, 1, 1>(a, st);
    const int j = ceil_div(a.pieces, 256);
    return j <= 1 ? launch_gated<T, 4, 1>(a, st) : j <= 2 ? launch_gated<T, 4, 2>(a, st) : j <= 4 ? launch_gated<T, 4, 4>(a, st) : launch_gated<T, 4, 8>(a, st);
}

}  // namespace fise

using namespace fise;

extern "C" int fise_masked_gated_norm(const fise_gated_norm_args* g, void* stream) {
    const char* fn = "fise_masked_gated_norm";
    if (!g || !g->x || (!g->r && !g->y)) return fail(FISE_ERR_NULL, "%s: null pointer", fn);
    if (g->dtype != FISE_F32 && g->dtype != FISE_BF16) return fail(FISE_ERR_DTYPE, "%s: dtype %d", fn, g->dtype);
    auto kind = [](int k) { return k == FISE_NORM_NONE || k == FISE_NORM_LAYER || k == FISE_NORM_RMS; };
    if (!kind(g->post_norm) || !kind(g->pre_norm)) return fail(FISE_ERR_SHAPE, "%s: norms %d, %d", fn, g->post_norm, g->pre_norm);
    if (g->B < 1 || g->H < 1 || g->W < 1 || g->C < 1 || g->C > NG_MAX_C || g->tile < 0 || (g->tile && (g->H % g->tile || g->W % g->tile)))
        return fail(FISE_ERR_SHAPE, "%s: B%d H%d W%d C%d tile%d", fn, g->B, g->H, g->W, g->C, g->tile);
    if ((long long)g->B * g->H * g->W >= 1ll << 31) return fail(FISE_ERR_SHAPE, "%s: %d maps of %d x %d rows", fn, g->B, g->H, g->W);
    // what would be left out without a word
    if (!g->h && (g->post_norm != FISE_NORM_NONE || g->gate)) return fail(FISE_ERR_NULL, "%s: a norm or a gate of a branch that is not given", fn);
    if (!g->y && (g->pre_norm != FISE_NORM_NONE || g->mod_scale || g->mod_shift)) return fail(FISE_ERR_NULL, "%s: a norm or a modulation without an output y", fn);
    if ((g->post_b && g->post_norm != FISE_NORM_LAYER) || (g->pre_b && g->pre_norm != FISE_NORM_LAYER) || (g->post_w && g->post_norm == FISE_NORM_NONE) ||
        (g->pre_w && g->pre_norm == FISE_NORM_NONE))
        return fail(FISE_ERR_SHAPE, "%s: weights that this kind of norm does not have", fn);
    const bool modulated = g->gate || g->mod_scale || g->mod_shift;
    if (g->mod_stride < 0 || (modulated && g->B > 1 && g->mod_stride && g->mod_stride < g->C)) return fail(FISE_ERR_SHAPE, "%s: modulations of %d channels %lld apart", fn, g->C, (long long)g->mod_stride);
    if (g->C % 8 || (modulated && g->mod_stride % 4)) return fail(FISE_ERR_ALIGN, "%s: C must be a multiple of 8, the modulations' stride of 4", fn);
    for (const void* p : {g->x, g->h, (const void*)g->r, (const void*)g->y, g->post_w, g->post_b, g->pre_w, g->pre_b, (const void*)g->gate, (const void*)g->mod_scale, (const void*)g->mod_shift})
        if (!aligned16(p)) return fail(FISE_ERR_ALIGN, "%s: pointers must be 16-byte aligned", fn);
    if (g->r == g->y) return fail(FISE_ERR_SHAPE, "%s: r and y are the same buffer", fn);
    const int tiles = g->tile ? (g->H / g->tile) * (g->W / g->tile) : 0;
    if (g->tile && (g->n_active < 0 || g->n_active > tiles)) return fail(FISE_ERR_CAPACITY, "%s: n_active %d of %d", fn, g->n_active, tiles);
    if (g->tile && g->n_active == 0) return FISE_OK;
    if (g->tile && !g->tile_idx) return fail(FISE_ERR_NULL, "%s: null tile_idx", fn);
    GatedNorm a{};
    a.x = g->x; a.h = g->h; a.r = g->r; a.y = g->y;
    a.post_w = g->post_w; a.post_b = g->post_b; a.pre_w = g->pre_w; a.pre_b = g->pre_b;
    a.gate = g->gate; a.scale = g->mod_scale; a.shift = g->mod_shift; a.mod_stride = g->mod_stride;
    a.tile_idx = g->tile_idx; a.tile = g->tile; a.W = g->W; a.HW = g->H * g->W; a.C = g->C; a.pieces = g->C / 8;
    a.M = g->tile ? g->n_active * g->tile * g->tile : a.HW;
    a.rows = g->B * a.M;
    a.post = g->post_norm; a.pre = g->pre_norm; a.h_is_map = g->h_is_map; a.y_is_map = g->y_is_map;
    a.res_scale = g->res_scale; a.eps = g->eps; a.channels = (float)g->C;
    a.d_M = fast_div(a.M);
    if (g->tile) { a.tiles_w = g->W / g->tile; a.d_tt = fast_div(g->tile * g->tile); a.d_tile = fast_div(g->tile); a.d_tiles_w = fast_div(a.tiles_w); }
    return g->dtype == FISE_F32 ? launch_gated<float>(a, as_stream(stream)) : launch_gated<bf16_t>(a, as_stream(stream));
}
