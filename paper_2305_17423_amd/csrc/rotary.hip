// Rotary positions on several axes: pairs (u, v) of a head's channels are turned by a = (pos + offset) theta^(-2 j / n), a pair at a time.
//
// Every channel is read and written once, which bounds it.  A thread owns VE pairs (one 16-byte vector of each side; one pair where strides or alignment do not
// allow that) of one row, works out their sines and cosines once and turns those pairs of several heads with them.
// The angle is taken in 64 bits and in turns, so that its whole part drops out without error and what is left of a position of 10^6 is that of
// exact arithmetic to 2^-30 turns; rounded to float it is within 2^-26 turns, and sine and cosine are float.
// Queries and keys of 65536 tokens, 16 heads of 128 channels each, bf16 (1.07 GB): 205 us, 5.2 TB/s, which is a large copy's rate.
#include <cmath>
#include "common.h"

namespace fise {

struct RotaryPart {                                 // one tensor
    const unsigned char* x; unsigned char* y;
    long long x_batch, x_row, x_head, y_batch, y_row, y_head;          // elements
    int heads, start, x_is_map, y_is_map;
    int units, rot_units;                           // threads of a head: those that turn pairs, then those that copy VE channels
    int per_thread, slices;                         // heads of a thread, threads that share a row's heads
};
struct RotaryArgs {
    RotaryPart p[2];
    const void* pos; int pos_float, pos_shared;
    const int* tile_idx; int tile, tiles;           // tile 0: all tokens
    int M, rows, n_axes, half, pairing, shared_freq, inverse;
    int T, H, W;
    int begin[5];                                   // first pair of an axis, and half
    double log2_ratio[4], ratio[4], offset[4];      // theta^(-2 / n)
};

template <typename T, int VE> struct RotaryVec;
template <> struct RotaryVec<float, 4> {
    static __device__ __forceinline__ void ld(const float* p, float* v) { const f32x4_t w = *reinterpret_cast<const f32x4_t*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = w[e]; }
    static __device__ __forceinline__ void st(float* p, const float* v) { *reinterpret_cast<f32x4_t*>(p) = f32x4_t{v[0], v[1], v[2], v[3]}; }
};
template <> struct RotaryVec<bf16_t, 8> {
    static __device__ __forceinline__ void ld(const bf16_t* p, float* v) { const u32x4_t w = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[2 * e] = lo16(w[e]); v[2 * e + 1] = hi16(w[e]); } }
    static __device__ __forceinline__ void st(bf16_t* p, const float* v) { *reinterpret_cast<u32x4_t*>(p) = u32x4_t{f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7])}; }
};
template <typename T> struct RotaryVec<T, 1> {
    static __device__ __forceinline__ void ld(const T* p, float* v) { *v = Elem<T>::ld(p); }
    static __device__ __forceinline__ void st(T* p, const float* v) { Elem<T>::st(p, *v); }
};

// Position along an axis of a row whose place on the grid is t, y, x or whose positions start at `at`.
__device__ __forceinline__ double rotary_place(const RotaryArgs& a, int axis, long long at, int t, int y, int x) {
    if (a.pos) return a.offset[axis] + (a.pos_float ? (double)reinterpret_cast<const float*>(a.pos)[at + axis] : (double)reinterpret_cast<const int*>(a.pos)[at + axis]);
    const int place = axis + 3 - a.n_axes;                             // (two axes: y, x)
    return a.offset[axis] + (a.n_axes == 1 ? (double)(((long long)t * a.H + y) * a.W + x) : place == 0 ? (double)t : place == 1 ? (double)y : (double)x);
}

template <typename T, int VE>
__global__ __launch_bounds__(256) void rotary_kernel(RotaryArgs a) {
    const RotaryPart& p = a.p[blockIdx.y];
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int unit = (int)(id % p.units);
    const long long rest = id / p.units;
    const int slice = (int)(rest % p.slices);
    const long long row = rest / p.slices;                             // b * M + m
    if (row >= a.rows) return;
    const int b = (int)(row / a.M), m = (int)(row % a.M);
    int t = 0, y = 0, x = 0;
    if (a.tile) {
        const int per_row = a.W / a.tile, per_map = per_row * (a.H / a.tile), tt = a.tile * a.tile;
        const int id_ = a.tile_idx[m / tt], in = m % tt;
        if ((unsigned)id_ >= (unsigned)a.tiles) return;
        t = id_ / per_map;
        y = id_ % per_map / per_row * a.tile + in / a.tile;
        x = id_ % per_row * a.tile + in % a.tile;
    } else if (a.T) {
        x = m % a.W; y = m / a.W % a.H; t = m / a.W / a.H;
    }
    const long long token = ((long long)t * a.H + y) * a.W + x;
    const T* from = reinterpret_cast<const T*>(p.x) + b * p.x_batch + (p.x_is_map ? token : m) * p.x_row;
    T* to = reinterpret_cast<T*>(p.y) + b * p.y_batch + (p.y_is_map ? token : m) * p.y_row;
    const int h0 = slice * p.per_thread, h1 = min(p.heads, h0 + p.per_thread);
    if (unit >= p.rot_units) {                                         // channels that stay as they are
        int c = (unit - p.rot_units) * VE;
        if (c >= p.start) c += 2 * a.half;
        for (int h = h0; h < h1; ++h) {
            float v[VE];
            RotaryVec<T, VE>::ld(from + h * p.x_head + c, v);
            RotaryVec<T, VE>::st(to + h * p.y_head + c, v);
        }
        return;
    }
    // first pair of the unit and where its two sides are
    const int i0 = unit * VE;
    int ca, cb;
    if (a.pairing == FISE_ROTARY_ADJACENT) { ca = 2 * i0; cb = ca + VE; }
    else if (a.pairing == FISE_ROTARY_HALVES) { ca = i0; cb = i0 + a.half; }
    else {
        int axis = 0;
#pragma unroll
        for (int j = 1; j < 4; ++j) axis += j < a.n_axes && i0 >= a.begin[j];
        ca = i0 + a.begin[axis]; cb = ca + a.begin[axis + 1] - a.begin[axis];
    }
    ca += p.start; cb += p.start;
    float c[VE], s[VE];
    const long long at = ((long long)(a.pos_shared ? 0 : b) * a.M + m) * a.n_axes;
    // A pair's frequency in turns is the one before times the axis' ratio, or the axis' first: one power a thread (eight of them: 1.5 us of the smallest call)
    constexpr double TURN = 0.15915494309189533577;                    // 1 / (2 pi)
    int axis = 0;
#pragma unroll
    for (int j = 1; j < 4; ++j) axis += j < a.n_axes && i0 >= a.begin[j];
    const int of = a.shared_freq ? 0 : axis;
    double f = exp2(a.log2_ratio[of] * (double)(a.shared_freq ? i0 : i0 - a.begin[axis])) * TURN, ratio = a.ratio[of], place = rotary_place(a, axis, at, t, y, x);
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        const double turns = place * f;
        sincospif(2.f * (float)(turns - rint(turns)), &s[e], &c[e]);
        if (a.inverse) s[e] = -s[e];
        f *= ratio;
        if (e + 1 < VE && i0 + e + 1 == a.begin[axis + 1] && axis + 1 < a.n_axes) {
            ++axis;
            place = rotary_place(a, axis, at, t, y, x);
            if (!a.shared_freq) { f = TURN; ratio = a.ratio[axis]; }
        }
    }
    const bool adjacent = a.pairing == FISE_ROTARY_ADJACENT;
#pragma unroll 4
    for (int h = h0; h < h1; ++h) {
        float u[VE], v[VE], w[2 * VE];
        RotaryVec<T, VE>::ld(from + h * p.x_head + ca, u);
        RotaryVec<T, VE>::ld(from + h * p.x_head + cb, v);
        if (adjacent) {                                                // pairs lie side by side: sides 2e and 2e + 1 of both vectors
#pragma unroll
            for (int e = 0; e < VE; ++e) { w[e] = u[e]; w[VE + e] = v[e]; }
#pragma unroll
            for (int e = 0; e < VE; ++e) { u[e] = w[2 * e]; v[e] = w[2 * e + 1]; }
        }
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float r = u[e] * c[e] - v[e] * s[e];
            v[e] = u[e] * s[e] + v[e] * c[e];
            u[e] = r;
        }
        if (adjacent) {
#pragma unroll
            for (int e = 0; e < VE; ++e) { w[2 * e] = u[e]; w[2 * e + 1] = v[e]; }
#pragma unroll
            for (int e = 0; e < VE; ++e) { u[e] = w[e]; v[e] = w[VE + e]; }
        }
        RotaryVec<T, VE>::st(to + h * p.y_head + ca, u);
        RotaryVec<T, VE>::st(to + h * p.y_head + cb, v);
    }
}

}  // namespace fise

using namespace fise;

extern "C" int fise_rotary(const fise_rotary_args* g, void* stream) {
    const char* fn = "fise_rotary";
    if (!g) return fail(FISE_ERR_NULL, "%s: null pointer", fn);
    if (g->n_tensors < 1 || g->n_tensors > 2) return fail(FISE_ERR_SHAPE, "%s: %d tensors (1 or 2)", fn, g->n_tensors);
    for (int i = 0; i < g->n_tensors; ++i)
        if (!g->t[i].x || !g->t[i].y) return fail(FISE_ERR_NULL, "%s: null pointer in tensor %d", fn, i);
    if (g->dtype != FISE_F32 && g->dtype != FISE_BF16) return fail(FISE_ERR_DTYPE, "%s: dtype %d", fn, g->dtype);
    if (g->n_axes < 1 || g->n_axes > 4) return fail(FISE_ERR_SHAPE, "%s: %d axes (1 to 4)", fn, g->n_axes);
    if (g->pairing < 0 || g->pairing > 2) return fail(FISE_ERR_SHAPE, "%s: pairing %d", fn, g->pairing);
    RotaryArgs a{};
    for (int j = 0; j < g->n_axes; ++j) {
        const int n = g->axis_dim[j];
        if (n < 2 || n % 2 || n > 1024) return fail(FISE_ERR_SHAPE, "%s: axis %d of %d channels (an even number up to 1024)", fn, j, n);
        if (!(g->theta[j] > 0.0) || std::isinf(g->theta[j]) || !std::isfinite(g->offset[j])) return fail(FISE_ERR_SHAPE, "%s: theta %g, offset %g of axis %d", fn, g->theta[j], g->offset[j], j);
        a.begin[j + 1] = a.begin[j] + n / 2;
        a.offset[j] = g->offset[j];
    }
    a.half = a.begin[g->n_axes];
    for (int j = 0; j < g->n_axes; ++j) {
        a.log2_ratio[j] = -2.0 * std::log2(g->theta[j]) / (g->shared_freq ? 2.0 * a.half : (double)g->axis_dim[j]);
        a.ratio[j] = std::exp2(a.log2_ratio[j]);
    }
    if (a.half > 512) return fail(FISE_ERR_SHAPE, "%s: %d rotated channels (at most 1024)", fn, 2 * a.half);
    if (g->B < 1 || g->M < 0 || (long long)g->B * g->M > 0x7fffffffLL) return fail(FISE_ERR_SHAPE, "%s: B=%d M=%d", fn, g->B, g->M);
    bool maps = false;
    for (int i = 0; i < g->n_tensors; ++i) maps = maps || g->t[i].x_is_map || g->t[i].y_is_map;
    const bool grid = !g->pos || maps || g->tile;
    if (grid) {
        if (g->T < 1 || g->H < 1 || g->W < 1 || (long long)g->T * g->H > 0x7fffffffLL || (long long)g->T * g->H * g->W > 0x7fffffffLL) return fail(FISE_ERR_SHAPE, "%s: grid %d x %d x %d", fn, g->T, g->H, g->W);
        if (!g->pos && g->n_axes > 3) return fail(FISE_ERR_SHAPE, "%s: a grid has at most 3 axes", fn);
        if (g->tile < 0 || (g->tile && (g->H % g->tile || g->W % g->tile))) return fail(FISE_ERR_SHAPE, "%s: tile %d on a %d x %d map", fn, g->tile, g->H, g->W);
        const long long tokens = (long long)g->T * g->H * g->W;
        if (g->tile) {
            const long long tt = (long long)g->tile * g->tile;
            if (g->n_active < 0 || g->n_active > tokens / tt) return fail(FISE_ERR_CAPACITY, "%s: %d active tiles of %lld", fn, g->n_active, tokens / tt);
            if (g->M != g->n_active * tt) return fail(FISE_ERR_SHAPE, "%s: M=%d, %d tiles have %lld rows", fn, g->M, g->n_active, g->n_active * tt);
            if (g->n_active && !g->tile_idx) return fail(FISE_ERR_NULL, "%s: tile_idx NULL", fn);
            a.tiles = (int)(tokens / tt);
        } else if (g->M != tokens) return fail(FISE_ERR_SHAPE, "%s: M=%d, the grid has %lld tokens", fn, g->M, tokens);
        a.T = g->T; a.H = g->H; a.W = g->W;
    }
    if (g->pos && ((uintptr_t)g->pos & 3)) return fail(FISE_ERR_ALIGN, "%s: positions must be aligned to their type", fn);
    if (g->pos && g->pos_B != 1 && g->pos_B != g->B) return fail(FISE_ERR_SHAPE, "%s: positions of %d batch elements (1 or %d)", fn, g->pos_B, g->B);
    const int es = g->dtype == FISE_F32 ? 4 : 2, wide = 16 / es, rot = 2 * a.half;
    bool vec = g->pairing == FISE_ROTARY_ADJACENT ? rot % (2 * wide) == 0 : g->pairing == FISE_ROTARY_HALVES ? a.half % wide == 0 : true;
    if (g->pairing == FISE_ROTARY_AXIS_HALVES)
        for (int j = 0; j < g->n_axes; ++j) vec = vec && (g->axis_dim[j] / 2) % wide == 0 && g->axis_dim[j] % wide == 0;
    for (int i = 0; i < g->n_tensors; ++i) {
        const fise_rotary_tensor& t = g->t[i];
        if (t.heads < 1 || t.d < 1 || t.start < 0 || (long long)t.start + rot > t.d) return fail(FISE_ERR_SHAPE, "%s: tensor %d has %d heads of %d channels, rotated %d from %d on", fn, i, t.heads, t.d, rot, t.start);
        for (long long s : {(long long)t.x_batch, (long long)t.x_row, (long long)t.x_head, (long long)t.y_batch, (long long)t.y_row, (long long)t.y_head})
            if (s < 0) return fail(FISE_ERR_SHAPE, "%s: a negative stride in tensor %d", fn, i);
        if ((uintptr_t)t.x % es || (uintptr_t)t.y % es) return fail(FISE_ERR_ALIGN, "%s: tensor %d must be aligned to its type", fn, i);
        if (t.x == t.y && (t.x_batch != t.y_batch || t.x_row != t.y_row || t.x_head != t.y_head || !t.x_is_map != !t.y_is_map))
            return fail(FISE_ERR_SHAPE, "%s: tensor %d in place needs the same strides and form on both sides", fn, i);
        vec = vec && aligned16(t.x) && aligned16(t.y) && t.start % wide == 0 && t.d % wide == 0;
        for (long long s : {(long long)t.x_batch, (long long)t.x_row, (long long)t.x_head, (long long)t.y_batch, (long long)t.y_row, (long long)t.y_head}) vec = vec && s % wide == 0;
    }
    if (g->M == 0) return FISE_OK;
    const int ve = vec ? wide : 1;
    a.M = g->M; a.rows = g->B * g->M; a.n_axes = g->n_axes; a.pairing = g->pairing; a.shared_freq = g->shared_freq != 0; a.inverse = g->inverse != 0;
    a.pos = g->pos; a.pos_float = g->pos_is_float != 0; a.pos_shared = g->pos_B == 1; a.tile_idx = g->tile_idx; a.tile = g->tile;
    long long blocks = 0;
    for (int i = 0; i < g->n_tensors; ++i) {
        const fise_rotary_tensor& t = g->t[i];
        RotaryPart& p = a.p[i];
        p.x = (const unsigned char*)t.x; p.y = (unsigned char*)t.y;
        p.x_batch = t.x_batch; p.x_row = t.x_row; p.x_head = t.x_head; p.y_batch = t.y_batch; p.y_row = t.y_row; p.y_head = t.y_head;
        p.heads = t.heads; p.start = t.start; p.x_is_map = t.x_is_map != 0; p.y_is_map = t.y_is_map != 0;
        p.rot_units = a.half / ve;
        p.units = p.rot_units + (t.x == t.y ? 0 : (t.d - rot) / ve);
        // heads that share a thread's sines: as many as leave two waves on each of the 1024 SIMDs, up to eight (65536 tokens, 16 heads of 128, us at 2, 4, 8, 16: 211, 202, 205, 234)
        const long long all = (long long)a.rows * p.units * t.heads;
        p.per_thread = (int)std::min<long long>(std::min(t.heads, 8), std::max<long long>(1, all / 131072));
        p.slices = ceil_div(t.heads, p.per_thread);
        const long long n = ((long long)a.rows * p.units * p.slices + 255) / 256;
        blocks = std::max(blocks, n);
    }
    if (blocks >= 1 << 24) return fail(FISE_ERR_SHAPE, "%s: more pairs than a launch holds", fn);
    const dim3 dims((unsigned)blocks, (unsigned)g->n_tensors);
    const hipStream_t st = as_stream(stream);
    if (g->dtype == FISE_F32) {
        if (vec) hipLaunchKernelGGL((rotary_kernel<float, 4>), dims, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((rotary_kernel<float, 1>), dims, dim3(256), 0, st, a);
    } else {
        if (vec) hipLaunchKernelGGL((rotary_kernel<bf16_t, 8>), dims, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((rotary_kernel<bf16_t, 1>), dims, dim3(256), 0, st, a);
    }
    FISE_CHECK_LAUNCH(fn);
    return FISE_OK;
}
