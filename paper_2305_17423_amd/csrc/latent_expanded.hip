// Attention over a cache of latent vectors, expanded form (many queries): the keys and values of every head are made first, one product with W_uk and one with W_uv,
// and then met by the queries of their head; 2 (d + dr + dv) operations a (query, key) pair where the absorbed form has 2 (2 r + dr).
#include <algorithm>
#include "latent.h"

namespace fise {

// ---------------------------------------------------------------------------------------------------------------- keys and values
// Tiles of 128 keys x 128 weight rows of one batch element on 32x32x16 products, four waves of 64 x 64; both operands run along the latent channels, 64 a step,
// loaded directly to LDS, a step ahead.  Rows of 128 bytes, sixteen-byte pieces at piece ^ (row / 2 & 7): sixteen rows read at
// once lie in different banks.  The first index of the product is the one that runs along the
// result's memory (a key's channels; a value channel's keys), so that a lane has four neighbours.  Keys that do not exist are zeros.
constexpr int LE_STEP = 64, LE_STAGE = 2 * 128 * LE_STEP * 2;
__global__ __launch_bounds__(256, 2) void latent_expand_kernel(const LatentArgs a, int KD, int key_tiles, int k_tiles, int v_tiles, FastDiv d_key_tiles, FastDiv d_tiles) {
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, hl = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave >> 1, wc = wave & 1;
    // weight tile slowest within an element: a key tile's workgroups follow one another in an XCD
    int w = blockIdx.x;
    { const int chunk = gridDim.x >> 3; if (w < chunk << 3) w = (w & 7) * chunk + (w >> 3); }
    const int kt_b = (int)fdiv((unsigned)w, d_tiles), wt = w - kt_b * (k_tiles + v_tiles), b = (int)fdiv((unsigned)kt_b, d_key_tiles), kt = kt_b - b * key_tiles;
    const int len = __builtin_amdgcn_readfirstlane(la_len(a, b)), key0 = kt * LX_KEYS;
    if (key0 >= len) return;                                           // nobody reads it
    const bool values = wt >= k_tiles;
    const int w0 = (values ? wt - k_tiles : wt) * 128, n_w = a.heads * (values ? a.dv : a.d), row_bytes = (a.r + a.dr) * 2;
    const auto keys = buf((const unsigned char*)a.cache + ((size_t)b * a.cache_tokens + key0) * row_bytes, (unsigned)(min(len - key0, 128) * row_bytes));
    const auto weights = buf((values ? a.w_uv : a.w_uk) + (size_t)w0 * a.r, (unsigned)(min(n_w - w0, 128) * a.r * 2));

    // a wave loads 32 rows of each operand in four loads of eight rows
    unsigned key_off[4], w_off[4];
    int piece[2];                                                      // of loads of even and odd number
#pragma unroll
    for (int j = 0; j < 2; ++j) piece[j] = (lane & 7) ^ ((j * 8 + (lane >> 3)) >> 1);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = wave * 32 + j * 8 + (lane >> 3);
        key_off[j] = (unsigned)(row * row_bytes + piece[j & 1] * 16);
        w_off[j] = (unsigned)(row * a.r * 2 + piece[j & 1] * 16);
    }
    const int steps = (a.r + LE_STEP - 1) / LE_STEP;
    auto load = [&](int s) {
        unsigned char* const to = lds + (s & 1) * LE_STAGE + wave * 4096;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool ok = s * LE_STEP + piece[j & 1] * 8 < a.r;      // channels past r: zeros on both sides
            __builtin_amdgcn_raw_ptr_buffer_load_lds(keys, (FISE_AS3 void*)(to + j * 1024), 16, (int)(ok ? key_off[j] + s * (LE_STEP * 2) : 0x40000000u), 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(weights, (FISE_AS3 void*)(to + 16384 + j * 1024), 16, (int)(ok ? w_off[j] + s * (LE_STEP * 2) : 0x40000000u), 0, 0, 0);
        }
    };
    f32x16_t acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    load(0);
    const int first = values ? 0 : 16384, second = 16384 - first;      // operand whose index runs along the result: keys for values, weights for keys
    for (int s = 0; s < steps; ++s) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (s + 1 < steps) load(s + 1);
        const unsigned char* const stage = lds + (s & 1) * LE_STAGE;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            bf16x8_t x[2], y[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int at = ((ks * 2 + hl) ^ ((l32 >> 1) & 7)) * 16;
                x[i] = *reinterpret_cast<const bf16x8_t*>(stage + first + (wr * 64 + i * 32 + l32) * 128 + at);
                y[i] = *reinterpret_cast<const bf16x8_t*>(stage + second + (wc * 64 + i * 32 + l32) * 128 + at);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], y[j], acc[i][j], 0, 0, 0);
        }
    }
    // through LDS, column by column of the product (its pieces of eight rows at piece ^ (column & 15)), so that sixteen lanes store 256 bytes side by side
    const int width = KD * 16;
    la_barrier();
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int piece = wr * 8 + i * 4 + q, col = wc * 64 + j * 32 + l32;
                *reinterpret_cast<uint2*>(lds + col * 256 + (piece ^ (col & 15)) * 16 + hl * 8) =
                    make_uint2(f2bf2(acc[i][j][4 * q], acc[i][j][4 * q + 1]), f2bf2(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]));
            }
    la_barrier();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int col = i * 16 + (tid >> 4), row = (tid & 15) * 8;
        const uint4 v = *reinterpret_cast<const uint4*>(lds + col * 256 + ((tid & 15) ^ (col & 15)) * 16);
        if (values) {
            if (w0 + col < n_w) *reinterpret_cast<uint4*>(a.v + ((size_t)b * n_w + w0 + col) * a.n_pad + key0 + row) = v;
        } else if (w0 + row < n_w) {
            const int c = w0 + row, h = c / a.d;
            *reinterpret_cast<uint4*>(a.k + (((size_t)b * a.heads + h) * a.n_pad + key0 + col) * width + (c - h * a.d)) = v;
        }
    }
    if (!values) {
        // the shared key (and zeros) behind the channels of the heads that begin in this tile
        const int h0 = (w0 + a.d - 1) / a.d, h1 = min((w0 + 127) / a.d + 1, a.heads), tail = (width - a.d) / 8;
        for (int i = tid; i < (h1 - h0) * 128 * tail; i += 256) {
            const int c = (i % tail) * 8, key = i / tail % 128, h = h0 + i / (tail * 128);
            uint4 v = make_uint4(0, 0, 0, 0);
            if (c < a.dr && key0 + key < len) v = *reinterpret_cast<const uint4*>(a.cache + ((size_t)b * a.cache_tokens + key0 + key) * (a.r + a.dr) + a.r + c);
            *reinterpret_cast<uint4*>(a.k + (((size_t)b * a.heads + h) * a.n_pad + key0 + key) * width + a.d + c) = v;
        }
    }
#endif
}

// ---------------------------------------------------------------------------------------------------------------- attention
// A wave has 32 queries of a head; keys come in blocks of 64 through LDS, loaded directly, a block ahead.  Scores are computed transposed (a lane keeps one query),
// from key rows in the order that makes a lane's eight scores of a 16-key step those of eight consecutive keys: they are the operand of the second product as
// they stand.  A row's pieces are placed so that sixteen rows read at once lie in different banks, by what 256 leaves of the row's bytes.
template <int KD, int DB>
__global__ __launch_bounds__(256, 2) void latent_expanded_kernel(const LatentArgs a, int nqt, int heads_xcd) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int PIECES = 2 * KD, PITCH = PIECES * 16, KB = LX_BLOCK * PITCH, VB = DB * 32 * 128, STAGE = KB + VB, KL = KB / 4096, VL = VB / 4096;
    static_assert(KB % 4096 == 0 && KD % 2 == 0 && (PITCH % 256 || PIECES % 16 == 0), "whole loads of four waves");
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, hl = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // an XCD gets whole heads (where their number allows), the tiles of all of them with most keys first; where all are on the CUs at once, two a CU, the second half
    // the other way round, so that the two that share a CU have as many keys as any other two
    const int per_xcd = (gridDim.x & 7) == 0 && heads_xcd, i_xcd = per_xcd ? blockIdx.x >> 3 : blockIdx.x, heads_here = per_xcd ? heads_xcd : a.B * a.heads;
    const int rank = i_xcd / heads_here, local = i_xcd - rank * heads_here, half = nqt >> 1;
    const int bh = (per_xcd ? (blockIdx.x & 7) * heads_xcd : 0) + local, b = (int)fdiv((unsigned)bh, a.d_heads), h = bh - b * a.heads;
    const int qt = gridDim.x <= 2 * LA_CUS && rank >= nqt - half ? rank - (nqt - half) : nqt - 1 - rank;
    const int len = __builtin_amdgcn_readfirstlane(la_len(a, b));
    const int m = qt * LX_QUERIES + wave * 32 + l32;
    const bool ok = m < a.M;
    const int limit = la_limit(a, len, min(m, a.M - 1)), limit_first = la_limit(a, len, qt * LX_QUERIES), limit_last = la_limit(a, len, min(qt * LX_QUERIES + LX_QUERIES, a.M) - 1);
    const int blocks = (limit_last + LX_BLOCK - 1) / LX_BLOCK;

    auto swizzle = [](int row) { return PITCH % 128 ? (row >> 2) & 3 : PITCH % 256 ? (row >> 1) & 7 : row & 15; };
    unsigned k_off[KL], v_off[VL];
#pragma unroll
    for (int j = 0; j < KL; ++j) {
        const int p = (wave * KL + j) * 64 + lane, row = p / PIECES, piece = (p - row * PIECES) ^ swizzle(row);
        const int key = (row & 32) + 16 * (row >> 4 & 1) + 8 * (row >> 2 & 1) + 4 * (row >> 3 & 1) + (row & 3);
        k_off[j] = (unsigned)(key * PITCH + piece * 16);
    }
    const bf16_t* const k = a.k + (size_t)bh * a.n_pad * (KD * 16);
    const bf16_t* const v = a.v + (size_t)bh * a.dv * a.n_pad;
#pragma unroll
    for (int j = 0; j < VL; ++j) {
        const int row = (wave * VL + j) * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
        v_off[j] = row < a.dv ? (unsigned)((lane >> 3) * a.n_pad * 2 + piece * 16) : 0x40000000u;
    }
    auto load = [&](int blk) {
        const auto kr = buf(k + (size_t)blk * LX_BLOCK * (KD * 16), KB);
        unsigned char* const to = lds + (blk & 1) * STAGE;
#pragma unroll
        for (int j = 0; j < KL; ++j) __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (FISE_AS3 void*)(to + (wave * KL + j) * 1024), 16, (int)k_off[j], 0, 0, 0);
#pragma unroll
        for (int j = 0; j < VL; ++j) {                                 // eight rows a load, each with a base of its own: rows of a long cache lie far apart
            const auto vr = buf(v + (size_t)(wave * VL + j) * 8 * a.n_pad + blk * LX_BLOCK, 0x40000000u);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (FISE_AS3 void*)(to + KB + (wave * VL + j) * 1024), 16, (int)v_off[j], 0, 0, 0);
        }
    };
    bf16x8_t qf[KD];
    {
        const bf16_t* const q = a.q + (((size_t)b * a.M + min(m, a.M - 1)) * a.heads + h) * (a.d + a.dr);
#pragma unroll
        for (int ks = 0; ks < KD; ++ks) {
            uint4 x = make_uint4(0, 0, 0, 0);
            const int c = ks * 16 + hl * 8;
            if (c < a.d + a.dr) x = *reinterpret_cast<const uint4*>(q + c);
            qf[ks] = *reinterpret_cast<const bf16x8_t*>(&x);
        }
    }
    f32x16_t o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    if (blocks > 0) load(0);
#pragma unroll
    for (int ks = 0; ks < KD; ++ks) asm volatile("" ::"v"(qf[ks]));
    for (int blk = 0; blk < blocks; ++blk) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (blk + 1 < blocks) load(blk + 1);
        unsigned char* const stage = lds + (blk & 1) * STAGE;
        const int k0 = blk * LX_BLOCK;
        f32x16_t s[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int e = 0; e < 16; ++e) s[kb][e] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KD; ++ks) {
                const bf16x8_t kf = *reinterpret_cast<const bf16x8_t*>(stage + (kb * 32 + l32) * PITCH + ((ks * 2 + hl) ^ swizzle(l32)) * 16);
                s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], s[kb], 0, 0, 0);
            }
        }
        const bool partial = k0 + LX_BLOCK > limit_first;
        if (partial) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (k0 + kb * 32 + (e >> 3) * 16 + hl * 8 + (e & 7) >= limit) s[kb][e] = -INFINITY;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[kb][e]);
        {
            const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            mx = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
        }
        mx = fmaxf(m_run, mx * a.scale_log2e);
        const float base = mx == -INFINITY ? 0.f : mx;
        const float alpha = __builtin_amdgcn_exp2f(m_run - base);
        float sum = 0.f;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float p = __builtin_amdgcn_exp2f(fmaf(s[kb][e], a.scale_log2e, -base));
                s[kb][e] = p;
                sum += p;
            }
        l_run = fmaf(l_run, alpha, sum);
        m_run = mx;
        if (__any(alpha != 1.0f)) {
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[i][e] *= alpha;
        }
        if (a.causal && partial) {                                     // uniform: what a key holds that a query does not see must not matter
            la_barrier();
#pragma unroll
            for (int j = 0; j < DB; ++j) {
                uint4* const at = reinterpret_cast<uint4*>(stage + KB + (j * 256 + tid) * 16);
                *at = la_finite(*at);
            }
            la_barrier();
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {                                  // steps of 16 keys
            const int kb = u >> 1, e0 = (u & 1) * 8;
            uint4 pw = make_uint4(f2bf2(s[kb][e0], s[kb][e0 + 1]), f2bf2(s[kb][e0 + 2], s[kb][e0 + 3]), f2bf2(s[kb][e0 + 4], s[kb][e0 + 5]), f2bf2(s[kb][e0 + 6], s[kb][e0 + 7]));
            const bf16x8_t pf = *reinterpret_cast<const bf16x8_t*>(&pw);
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const bf16x8_t vf = *reinterpret_cast<const bf16x8_t*>(stage + KB + (i * 32 + l32) * 128 + ((u * 2 + hl) ^ ((l32 >> 1) & 7)) * 16);
                o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[i], 0, 0, 0);
            }
        }
    }
    {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
        l_run = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if (!ok) return;
    const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;               // no key seen: zeros
    bf16_t* const out = a.out + (((size_t)b * a.M + m) * a.heads + h) * a.dv;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = i * 32 + q * 8 + hl * 4;
            if (c < a.dv) *reinterpret_cast<uint2*>(out + c) = make_uint2(f2bf2(o[i][4 * q] * inv, o[i][4 * q + 1] * inv), f2bf2(o[i][4 * q + 2] * inv, o[i][4 * q + 3] * inv));
        }
#endif
}

template <int TILE> static int launch_tile(const LatentArgs& a, hipStream_t st) {
    constexpr int KD = kExpandedTiles[TILE].KD, DB = kExpandedTiles[TILE].DB, lds = 2 * (LX_BLOCK * KD * 32 + DB * 32 * 128);
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&latent_expanded_kernel<KD, DB>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return fail(FISE_ERR_HIP, "fise_latent_attention: cannot raise the dynamic LDS limit");
    const int key_tiles = (int)(a.n_pad / LX_KEYS), k_tiles = ceil_div(a.heads * a.d, 128), v_tiles = ceil_div(a.heads * a.dv, 128);
    if (key_tiles) {
        ProfileScope prof(PROF_IGEMM_WIDE, 2.0 * a.B * a.n * a.heads * (double)a.r * (a.d + a.dv), 2.0 * a.B * a.n * (a.r + a.heads * (double)(a.d + a.dv)), st);
        hipLaunchKernelGGL(latent_expand_kernel, dim3((unsigned)(a.B * key_tiles * (k_tiles + v_tiles))), dim3(256), 2 * LE_STAGE, st, a, KD, key_tiles, k_tiles, v_tiles,
                           fast_div(key_tiles), fast_div(k_tiles + v_tiles));
    }
    FISE_CHECK_LAUNCH("fise_latent_attention: keys and values");
    const int nqt = ceil_div(a.M, LX_QUERIES);
    {
        ProfileScope prof(PROF_ATTENTION, 2.0 * a.B * a.M * a.heads * (double)a.n * (a.d + a.dr + a.dv), 2.0 * a.B * a.n * a.heads * (double)(a.d + a.dr + a.dv), st);
        hipLaunchKernelGGL((latent_expanded_kernel<KD, DB>), dim3((unsigned)(a.B * a.heads * nqt)), dim3(256), lds, st, a, nqt, a.B * a.heads % 8 ? 0 : a.B * a.heads / 8);
    }
    FISE_CHECK_LAUNCH("fise_latent_attention: expanded");
    return FISE_OK;
}

int launch_expanded(const LatentArgs& a, int tile, hipStream_t st) {
    static_assert(sizeof(kExpandedTiles) / sizeof(kExpandedTiles[0]) == 7, "one case each");
    switch (tile) {
    case 0: return launch_tile<0>(a, st);
    case 1: return launch_tile<1>(a, st);
    case 2: return launch_tile<2>(a, st);
    case 3: return launch_tile<3>(a, st);
    case 4: return launch_tile<4>(a, st);
    case 5: return launch_tile<5>(a, st);
    default: return launch_tile<6>(a, st);
    }
}

}  // namespace fise
