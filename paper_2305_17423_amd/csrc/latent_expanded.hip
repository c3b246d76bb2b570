// Attention over a cache of latent vectors, expanded form (many queries): the keys and values of every head are made first, one product with W_uk and one with W_uv,
// and then met by the queries of their head; 2 (d + dr + dv) operations a (query, key) pair where the absorbed form has 2 (2 r + dr).
#include <algorithm>
#include "latent.h"

namespace fise {

// ---------------------------------------------------------------------------------------------------------------- keys and values
// Tiles of 128 keys x 128 weight rows of one batch element on 32x32x16 products, four waves of 64 x 64; both operands run along the latent channels, 64 a step,
// loaded directly to LDS, a step ahead.  Rows of 128 bytes, sixteen-byte pieces at piece ^ (row / 2 & 7): sixteen rows read at
// once lie in different banks.  The first index of the product is the one that runs along the
// result's memory (a key's channels; a value channel's keys), so that a lane has four neighbours.  Keys that do not exist are zeros.  Keys and values are rounded to bf16, as the
// library's caches of them are; in two numbers each their products would double and LDS would not hold two workgroups' blocks.  16 heads of 4096 keys, r 512: 30 us, bound by
// what it reads from the L2 caches again (268 MB); 8 heads of 2 x 4096 keys, r 128: 11 us.
// Group g of the line: (element, head) and one of its tiles of queries.
struct LxGroup { int b, h, tile; };
__device__ __forceinline__ LxGroup lx_group(const LatentArgs& a, int g) {
    const int bh = (int)fdiv((unsigned)g, a.d_tiles), i = g - bh * a.tiles, b = (int)fdiv((unsigned)bh, a.d_heads);
    return {b, bh - b * a.heads, expanded_line_tile(i, a.tiles)};
}
typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
constexpr int LE_STEP = 64, LE_STAGE = 2 * 128 * LE_STEP * 2;
__global__ __launch_bounds__(256, 2) void latent_expand_kernel(const LatentArgs a, int KD, int key_tiles, int k_tiles, int v_tiles, FastDiv d_key_tiles, FastDiv d_tiles) {
#if defined(__HIP_DEVICE_COMPILE__)
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, hl = lane >> 5, l32 = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wr = wave >> 1, wc = wave & 1;
    int w = blockIdx.x;
    if (w == (int)gridDim.x - 1) {                                     // the line of key blocks
        la_line(a.table, a.groups, reinterpret_cast<int*>(lds), [&](int g) {
            const LxGroup p = lx_group(a, g);
            return (la_limit(a, la_len(a, p.b), min(a.M, (p.tile + 1) * LX_QUERIES) - 1) + LX_BLOCK - 1) / LX_BLOCK;
        });
        return;
    }
    // weight tile slowest within an element: a key tile's workgroups follow one another in an XCD
    { const int chunk = (gridDim.x - 1) >> 3; if (w < chunk << 3) w = (w & 7) * chunk + (w >> 3); }
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
    u16x2_t largest = {0, 0};                                          // bits of the largest magnitude: infinity and NaN are at least 0x7f80
    la_barrier();
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int piece = wr * 8 + i * 4 + q, col = wc * 64 + j * 32 + l32;
                const uint2 v = make_uint2(f2bf2(acc[i][j][4 * q], acc[i][j][4 * q + 1]), f2bf2(acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]));
                const uint2 bits = make_uint2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu);
                largest = __builtin_elementwise_max(largest, __builtin_elementwise_max(*reinterpret_cast<const u16x2_t*>(&bits.x), *reinterpret_cast<const u16x2_t*>(&bits.y)));
                *reinterpret_cast<uint2*>(lds + col * 256 + (piece ^ (col & 15)) * 16 + hl * 8) = v;
            }
    if (values) {
        const bool odd = __any(largest[0] >= 0x7f80 || largest[1] >= 0x7f80);
        if (lane == 0) reinterpret_cast<unsigned char*>(a.flags + ((size_t)b * v_tiles + wt - k_tiles) * key_tiles + kt)[wave] = odd;
        if (odd) {
            // Where the latent vector itself is not finite, every channel is NaN: the score of its key is NaN or infinite, and the probability 0 of a score of -inf meets
            // an infinite value.  (What is infinite without that has overflown, and stays.)
            bool bad = false;
            for (int c = 0; c < a.r; c += 8) {
                const u32x4_t x = __builtin_amdgcn_raw_buffer_load_b128(keys, (wr * 64 + lane) * row_bytes + c * 2, 0, 0);
                bad |= la_odd(make_uint4(x[0], x[1], x[2], x[3]));
            }
            const int col = wc * 64 + lane;
            asm volatile("" ::: "memory");                             // behind the writes above, of other types
            for (unsigned long long left = __ballot(bad); left; left &= left - 1) {
                const int key = wr * 64 + __ffsll(left) - 1;
                *reinterpret_cast<unsigned short*>(lds + col * 256 + ((key >> 3) ^ (col & 15)) * 16 + (key & 7) * 2) = 0x7fc0;
            }
        }
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
        // the shared key (and zeros) behind the channels of the heads that begin in this tile: four pieces on their way at once, each stored for every head
        const int h0 = (w0 + a.d - 1) / a.d, h1 = min((w0 + 127) / a.d + 1, a.heads), tail = (width - a.d) / 8;
        for (int i0 = tid; i0 < 128 * tail; i0 += 1024) {
            u32x4_t v[4];
            bf16_t* to[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * 256, key = i / tail, c = (i - key * tail) * 8;
                v[u] = __builtin_amdgcn_raw_buffer_load_b128(keys, c < a.dr ? key * row_bytes + (a.r + c) * 2 : 0x7fffffff, 0, 0);      // (zeros behind the last key)
                to[u] = a.k + (((size_t)b * a.heads + h0) * a.n_pad + key0 + key) * width + a.d + c;
            }
            for (int h = h0; h < h1; ++h)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (i0 + u * 256 < 128 * tail) *reinterpret_cast<u32x4_t*>(to[u]) = v[u];
                    to[u] += a.n_pad * width;
                }
        }
    }
#endif
}

// ---------------------------------------------------------------------------------------------------------------- attention
// A wave has 32 queries of a head; keys come in blocks of 64 through LDS, loaded directly, a block ahead.  Scores are computed transposed (a lane keeps one query),
// from key rows in the order that makes a lane's eight scores of a 16-key step those of eight consecutive keys: they are the operand of the second product as
// they stand.  A row's pieces are placed so that sixteen rows read at once lie in different banks, by what 256 leaves of the row's bytes.
// A turn is: scores of the next block, with the exponentials of this block between the products; sums of this block, with the maximum of the next between them.  So
// neither product waits for a softmax, nor the vector unit for a product; the order is written down, as the compiler's own keeps them apart.
// Probabilities are two bf16 numbers, as in the absorbed form: that took 16 heads of 4096 causal queries from 148 to 169 us, their root mean square error from 2.7e-3 to 2.4e-3 (1.7e-3 is
// the result's own rounding, the rest that of keys and values).
// The prompt's 16 x 1056 pairs of a tile and a block take this kernel 137 us with a pause between calls and 154 without, as the clock falls; at 0.6 PFLOP/s it is bound by what a SIMD
// issues: while it has waves its matrix unit is busy 53 % of the time (56 products a turn) and vector instructions take 44 % (32 exponentials and what turns scores into operands),
// so two waves a SIMD overlap little; LDS is busy a third of it.  768 queries on 4096 keys, twice, 8 heads of 40: 35 us, 12 or 13 turns a workgroup, matrix units 34 %, vector instructions 52 %.
// Few tiles: the workgroups share the line of key blocks evenly (latent.h), and latent_join_kernel adds up what a cut tile's parts came to.
[[maybe_unused]] constexpr int LX_AHEAD = 4;

// Values that are not finite, added to what a wave's queries have (a query sees the keys below `limit`, none that does not exist; part: its partial result, else `out` holds it): the first key
// of +inf, of -inf and of NaN in each channel tells what a query gets, and parts that find the same ones add the same.  Lanes share the keys; rare, so it is
// made to be short, not fast.
__device__ __forceinline__ void lx_add_odd(const LatentArgs& a, int bh, int lane, int limit, float* part, bf16_t* out) {
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");                   // the finite sums are where they belong
    const int none = 0x7fffffff;
    auto first = [&](int key) {                                        // over the wave (addresses of shuffles would stay in registers through all blocks)
        int least = none;
#pragma unroll 1
        for (int l = 0; l < 64; ++l) least = min(least, __builtin_amdgcn_readlane(key, l));
        return least;
    };
    const int end = -first(-limit);                                    // the first key that none of them sees
    for (int c = 0; c < a.dv; ++c) {
        const bf16_t* const v = a.v + ((size_t)bh * a.dv + c) * a.n_pad;
        int plus = none, minus = none, nan = none;
        for (int at = lane * 8; at < end; at += 512) {
            const uint4 x = *reinterpret_cast<const uint4*>(v + at);
            if (!la_odd(x)) continue;
            const unsigned words[4] = {x.x, x.y, x.z, x.w};
            for (int e = 0; e < 8; ++e) {
                const unsigned bits = words[e >> 1] >> (e & 1) * 16 & 0xffff;
                int& to = (bits & 0x7fff) > 0x7f80 ? nan : bits == 0x7f80 ? plus : minus;
                if ((bits & 0x7f80) == 0x7f80) to = min(to, at + e);
            }
        }
        plus = first(plus); minus = first(minus); nan = first(nan);
        if ((c >> 2 & 1) != lane >> 5 || limit <= min(min(plus, minus), nan)) continue;
        const float add = limit > nan || (limit > plus && limit > minus) ? NAN : limit > plus ? INFINITY : -INFINITY;
        if (part) part[c] += add;
        else out[c] = f2bf(bf2f(out[c]) + add);
    }
#endif
}

template <int KD, int DB>
__global__ __launch_bounds__(256, expanded_per_cu(KD)) void latent_expanded_kernel(const LatentArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int PIECES = 2 * KD, PITCH = PIECES * 16, KB = LX_BLOCK * PITCH, VB = DB * 32 * 128, KL = KB / 4096, VL = VB / 4096;
    static_assert(KB % 4096 == 0 && KD % 2 == 0 && (PITCH % 256 || PIECES % 16 == 0), "whole loads of four waves");
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];                  // keys, keys, values, values
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    const unsigned lds0 = (unsigned)(size_t)(FISE_AS3 unsigned char*)(FISE_AS3 void*)lds;
    const int tid = threadIdx.x, lane = tid & 63, hl = lane >> 5, l32 = lane & 31, wave = uniform(tid >> 6);
    // consecutive workgroups go to the eight XCDs in turn: give each XCD one run of the line
    int w = blockIdx.x, g, line0, line1;
    if (a.whole) {
        const ExpandedPlace p = expanded_place(w, a.B * a.heads, a.tiles, expanded_per_cu(KD));
        g = uniform(p.head * a.tiles + expanded_line_place(p.tile, a.tiles));
        line0 = uniform(a.table[g]); line1 = uniform(a.table[g + 1]);
        if (line0 == line1) {                                          // no query of the tile sees a key: zeros
            const LxGroup p = lx_group(a, g);
            const int quads = a.dv / 4;
            for (int e = tid; e < LX_QUERIES * quads; e += 256) {
                const int m = p.tile * LX_QUERIES + e / quads;
                if (m < a.M) *reinterpret_cast<uint2*>(a.out + (((size_t)p.b * a.M + m) * a.heads + p.h) * a.dv + e % quads * 4) = make_uint2(0, 0);
            }
            return;
        }
    } else {
        const int total = uniform(a.table[a.groups]), workgroups = min(a.workgroups, total);
        if (w >= workgroups) return;
        const int chunk = workgroups >> 3;
        if (w < chunk << 3) w = (w & 7) * chunk + (w >> 3);
        line0 = uniform((int)((long long)w * total / workgroups)); line1 = uniform((int)((long long)(w + 1) * total / workgroups));
        g = la_group(a.table, a.groups, line0);
    }

    // ---- places that depend on the lane only
    auto swizzle = [](int row) { return PITCH % 128 ? (row >> 2) & 3 : PITCH % 256 ? (row >> 1) & 7 : row & 15; };
    unsigned k_off[KL], v_off[2];
#pragma unroll
    for (int j = 0; j < KL; ++j) {
        const int p = (wave * KL + j) * 64 + lane, row = p / PIECES, piece = (p - row * PIECES) ^ swizzle(row);
        const int key = (row & 32) + 16 * (row >> 4 & 1) + 8 * (row >> 2 & 1) + 4 * (row >> 3 & 1) + (row & 3);
        k_off[j] = (unsigned)(key * PITCH + piece * 16);
    }
    const unsigned v_pitch = (unsigned)(a.n_pad * 2);
#pragma unroll
    for (int j = 0; j < 2; ++j) v_off[j] = (unsigned)(lane >> 3) * v_pitch + (unsigned)((lane & 7) ^ ((j * 8 + (lane >> 3)) >> 1)) * 16;
    // operands: key row l32 of a 32-key block (swizzle(l32 + 32) is that of l32), value row l32
    constexpr int KU = PITCH % 256 ? (PITCH % 128 ? 2 : 4) : 8;        // steps after which the places repeat
    unsigned k_at[KU], v_at[4];
#pragma unroll
    for (int u = 0; u < KU; ++u) k_at[u] = (unsigned)(l32 * PITCH + ((u * 2 + hl) ^ swizzle(l32)) * 16);
#pragma unroll
    for (int u = 0; u < 4; ++u) v_at[u] = (unsigned)(l32 * 128 + ((u * 2 + hl) ^ ((l32 >> 1) & 7)) * 16);

    constexpr int NK = 2 * KD, NV = 4 * DB, AHEAD = LX_AHEAD, RING = AHEAD + 1, NE = 32;      // products of the scores, of the sums; reads ahead of them; scores a lane
    for (int at = line0; at < line1; ++g) {
        const int g_at = uniform(a.table[g]), g_end = uniform(a.table[g + 1]), end = min(line1, g_end);
        if (end <= at) continue;
        const LxGroup place = lx_group(a, uniform(g));
        const int b = uniform(place.b), h = uniform(place.h), m0 = uniform(place.tile) * LX_QUERIES, bh = b * a.heads + h;
        const int blk0 = at - g_at, blk1 = end - g_at, len = uniform(la_len(a, b));
        const bool whole = blk0 == 0 && end == g_end;
        const int m = m0 + wave * 32 + l32;
        // (behind this part's last block: nothing)
        const int limit = min(la_limit(a, len, min(m, a.M - 1)), blk1 * LX_BLOCK), limit_first = min(la_limit(a, len, m0), blk1 * LX_BLOCK);

        const unsigned char* const k = (const unsigned char*)(a.k + (size_t)bh * a.n_pad * (KD * 16));
        const unsigned char* const v = (const unsigned char*)(a.v + (size_t)bh * a.dv * a.n_pad);
        auto load_k = [&](int blk) {                                   // (behind the last block: nothing)
            const u32x4_t from = la_buffer(k + (size_t)blk * KB, blk < blk1 ? KB : 0);
#pragma unroll
            for (int j = 0; j < KL; ++j) la_to_lds(from, k_off[j], lds0 + (blk & 1) * KB + (wave * KL + j) * 1024);
        };
        auto load_v = [&](int blk) {                                   // eight rows a load, each with a base of its own: rows of a long cache lie far apart
#pragma unroll
            for (int j = 0; j < VL; ++j) {
                const int row = (wave * VL + j) * 8;                   // rows past dv (a multiple of 8): zeros
                const u32x4_t from = la_buffer(v + (size_t)row * v_pitch + (size_t)blk * (LX_BLOCK * 2), blk < blk1 && row < a.dv ? 0x7fffffff : 0);
                la_to_lds(from, v_off[(wave * VL + j) & 1], lds0 + 2 * KB + (blk & 1) * VB + (wave * VL + j) * 1024);
            }
        };
        // Values that are not finite are in none of the sums (times what rounding left of a probability, or 0 of a key that a query does not see, they would be NaN), but added
        // behind them: a part with such a tile of values knows it before its first block.
        const int row_v = h * a.dv, tile_v = row_v >> 7, tiles_v = ((row_v + a.dv - 1) >> 7) - tile_v + 1, key_tiles = (int)(a.n_pad / LX_KEYS);
        const unsigned* const flags = a.flags + ((size_t)b * ((a.heads * a.dv + 127) >> 7) + tile_v) * key_tiles;
        auto odd_of = [&](int t0) {                                    // 64 tiles of keys from t0 on, the last one again behind it
            const int t = min(t0 + lane, (blk1 - 1) >> 1);
            return flags[t] | flags[(size_t)min(1, tiles_v - 1) * key_tiles + t] | flags[(size_t)(tiles_v - 1) * key_tiles + t];
        };
        unsigned odd_bits = odd_of(blk0 >> 1);                         // (on its way with the first blocks)
        bool odd;
        la_barrier();                                                  // the group before has been read to its end
        load_k(blk0);
        load_k(blk0 + 1);
        load_v(blk0);
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
        float m_run = -INFINITY, l_run = 0.f, alpha = 1.f, scale = a.scale_log2e, base = 0.f, top = 0.f;
        bf16x8_t fr[RING];
        auto read_k = [&](const unsigned char* tile, int p) {          // product p: step p % KD of the 32 keys p / KD
            const int ks = p % KD;
            return *reinterpret_cast<const bf16x8_t*>(tile + k_at[ks % KU] + (ks / KU) * (KU * 32) + p / KD * (32 * PITCH));
        };
        auto read_v = [&](const unsigned char* tile, int p) { return *reinterpret_cast<const bf16x8_t*>(tile + v_at[p / DB] + p % DB * 4096); };      // 16 keys p / DB, rows of block p % DB
        auto score = [&](f32x16_t& s, int p) {
            if (p % KD == 0) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 0.f;
            }
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[p % RING], qf[p % KD], s, 0, 0, 0);
        };
        auto mask = [&](f32x16_t& s, f32x16_t& t, int blk) {
            if (blk * LX_BLOCK + LX_BLOCK > limit_first) {             // uniform: some query of the tile does not see all of the block
#pragma unroll
                for (int e = 0; e < NE; ++e)
                    if (blk * LX_BLOCK + (e >> 3) * 16 + hl * 8 + (e & 7) >= limit) (e < 16 ? s : t)[e % 16] = -INFINITY;
            }
        };
        auto maximum = [&](const f32x16_t& s, const f32x16_t& t, int step) {      // in eight steps
            if (step == 0) top = s[0];
#pragma unroll
            for (int e = step * 4; e < step * 4 + 4; ++e) top = fmaxf(top, (e < 16 ? s : t)[e % 16]);
        };
        // a query's reference moves only when a score lies 8 powers of two above it (see the absorbed form)
        auto reference = [&](f32x16_t& s, f32x16_t& t) {
            const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            const float mx = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1])) * a.scale_log2e;
            const float to = mx > m_run + 8.f ? mx : m_run;
            base = to == -INFINITY ? 0.f : to;
            alpha = __builtin_amdgcn_exp2f(m_run - base);
            m_run = to;
            l_run *= alpha;
            // The exponentials' fma has the scores' products unrounded, the reference is a rounded one: from 2^31 on they are more than 127 apart.  There the scores are
            // rounded too before the reference is taken off.
            scale = a.scale_log2e;
            if (__builtin_expect(__any(fabsf(base) > 0x1p29f), 0)) {
#pragma unroll
                for (int e = 0; e < NE; ++e) {
                    float x = (e < 16 ? s : t)[e % 16] * a.scale_log2e;
                    asm volatile("" : "+v"(x));                        // (not one fma again)
                    (e < 16 ? s : t)[e % 16] = x - base;
                }
                scale = 1.f;
                base = 0.f;
            }
        };
        // c0, c1: scores of this block; n0: those of the next block's first 32 keys, the others' take c0, which has been used up by then
        f32x16_t sa, sb, sc;
        auto turn = [&](f32x16_t& c0, f32x16_t& c1, f32x16_t& n0, int blk) {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            load_k(blk + 2);
            load_v(blk + 1);
            unsigned char* const values = lds + 2 * KB + (blk & 1) * VB;
            const unsigned char* const keys = lds + ((blk + 1) & 1) * KB;
            if (odd) {
#pragma unroll
                for (int j = 0; j < DB; ++j) {
                    uint4* const at16 = reinterpret_cast<uint4*>(values + (j * 256 + tid) * 16);
                    *at16 = la_finite(*at16);
                }
                la_barrier();
            }
            if (__any(alpha != 1.0f)) {
#pragma unroll
                for (int i = 0; i < DB; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[i][e] *= alpha;
            }
            auto fetch = [&](int q) {                                  // the operand of product q of the turn
                if (q < NK) fr[q % RING] = read_k(keys, q);
                else if (q < NK + NV) fr[q % RING] = read_v(values, q - NK);
            };
            u32x4_t p[4], rest[4];                                     // probabilities, the operands of the sums, and what their rounding left
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int q = 0; q < AHEAD; ++q) fetch(q);
#pragma unroll
            for (int q = 0; q < NK; ++q) {
                fetch(q + AHEAD);
                __builtin_amdgcn_sched_barrier(0);
                score(q < KD ? n0 : c0, q);
#pragma unroll
                for (int e = NE * q / NK; e < NE * (q + 1) / NK; ++e) {
                    f32x16_t& c = e < 16 ? c0 : c1;
                    const float x = __builtin_amdgcn_exp2f(fmaf(c[e % 16], scale, -base));
                    c[e % 16] = x;
                    l_run += x;
                    if (e & 1) {
                        unsigned pair = f2bf2(c[e % 16 - 1], x);
                        asm volatile("" : "+v"(pair), "+v"(l_run));    // here, not behind the branch in front of their use
                        p[e / 8][e / 2 % 4] = pair;
                        unsigned less = f2bf2(c[e % 16 - 1] - lo16(pair), x - hi16(pair));
                        asm volatile("" : "+v"(less));
                        rest[e / 8][e / 2 % 4] = less;
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            mask(n0, c0, blk + 1);
#pragma unroll
            for (int q = 0; q < NV; ++q) {
                fetch(NK + q + AHEAD);
                __builtin_amdgcn_sched_barrier(0);
                const bf16x8_t pf = *reinterpret_cast<const bf16x8_t*>(&p[q / DB]);
                const bf16x8_t rf = *reinterpret_cast<const bf16x8_t*>(&rest[q / DB]);
                o[q % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[(NK + q) % RING], pf, o[q % DB], 0, 0, 0);
                o[q % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[(NK + q) % RING], rf, o[q % DB], 0, 0, 0);
                // the score products' results are there once a few of these have gone out
#pragma unroll
                for (int st = 0; st < 8; ++st)
                    if (st * (NV - 1) / 8 + 1 == q) maximum(n0, c0, st);
                __builtin_amdgcn_sched_barrier(0);
            }
            reference(n0, c0);
        };
#pragma unroll
        for (int ks = 0; ks < KD; ++ks) asm volatile("" ::"v"(qf[ks]));
        for (int t0 = (blk0 >> 1) + 64; t0 <= (blk1 - 1) >> 1; t0 += 64) odd_bits |= odd_of(t0);
        odd = __any(odd_bits != 0);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        {
            const unsigned char* const keys = lds + (blk0 & 1) * KB;
#pragma unroll
            for (int q = 0; q < NK; ++q) { fr[q % RING] = read_k(keys, q); score(q < KD ? sa : sb, q); }
        }
        mask(sa, sb, blk0);
#pragma unroll
        for (int st = 0; st < 8; ++st) maximum(sa, sb, st);
        reference(sa, sb);
        for (int blk = blk0;;) {
            turn(sa, sb, sc, blk);
            if (++blk >= blk1) break;
            turn(sc, sa, sb, blk);
            if (++blk >= blk1) break;
            turn(sb, sc, sa, blk);
            if (++blk >= blk1) break;
        }
        at = end;
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        {
            const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
            l_run = __uint_as_float(p[0]) + __uint_as_float(p[1]);
        }
        // (places anew: kept through the blocks they would not leave room for these)
        int again = threadIdx.x & 63;
        asm volatile("" : "+v"(again));
        const int half = again >> 5, query = m0 + wave * 32 + (again & 31);
        if (query >= a.M && !odd) continue;
        bf16_t* const out = a.out + (((size_t)b * a.M + query) * a.heads + h) * a.dv;
        const size_t row = ((size_t)w + g) * LX_QUERIES + wave * 32 + (again & 31);
        float* const part = a.part + row * (DB * 32);
        if (query < a.M && whole) {
            const float inv = l_run == 0.f ? 0.f : 1.0f / l_run;       // no key seen: zeros
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = i * 32 + q * 8 + half * 4;
                    if (c < a.dv) *reinterpret_cast<uint2*>(out + c) = make_uint2(f2bf2(o[i][4 * q] * inv, o[i][4 * q + 1] * inv), f2bf2(o[i][4 * q + 2] * inv, o[i][4 * q + 3] * inv));
                }
        } else if (query < a.M) {
            if (half == 0) a.ml[row] = make_float2(m_run, l_run);
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<float4*>(part + i * 32 + q * 8 + half * 4) = make_float4(o[i][4 * q], o[i][4 * q + 1], o[i][4 * q + 2], o[i][4 * q + 3]);
        }
        if (odd) lx_add_odd(a, bh, again, query < a.M ? limit : 0, whole ? nullptr : part, out);
    }
#endif
}

// Tiles that several workgroups had blocks of: their parts, each with its weight exp2(m - max), divided by the sum.  Tiles without a key: zeros.  DB * 8 lanes a query, four
// channels each.  480 parts of 128 queries x 64 channels: 7 us, bound by their 16 MB and one launch.
template <int DB>
__global__ __launch_bounds__(256) void latent_join_kernel(const LatentArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int QUADS = DB * 8, QUERIES = 256 / QUADS;
    const int g = blockIdx.x, total = a.table[a.groups], workgroups = min(a.workgroups, total), g0 = a.table[g], g1 = a.table[g + 1];
    const int w0 = g1 > g0 ? la_owner(g0, workgroups, total) : 0, n = g1 > g0 ? la_owner(g1 - 1, workgroups, total) - w0 + 1 : 0;
    if (n == 1) return;                                                // the workgroup that had it has written it
    const LxGroup place = lx_group(a, g);
    const int sub = threadIdx.x / QUADS, c = (threadIdx.x - sub * QUADS) * 4;
    if (sub >= QUERIES || c >= a.dv) return;
    for (int i = blockIdx.y * QUERIES + sub; i < LX_QUERIES; i += gridDim.y * QUERIES) {
        const int m = place.tile * LX_QUERIES + i;
        if (m >= a.M) return;
        const size_t row = ((size_t)w0 + g) * LX_QUERIES + i;
        float top = -INFINITY;
#pragma unroll 4
        for (int p = 0; p < n; ++p) top = fmaxf(top, a.ml[row + (size_t)p * LX_QUERIES].x);
        const float base = top == -INFINITY ? 0.f : top;
        float l = 0.f;
        float4 o = make_float4(0, 0, 0, 0);
#pragma unroll 4
        for (int p = 0; p < n; ++p) {
            const float2 ml = a.ml[row + (size_t)p * LX_QUERIES];
            const float4 v = *reinterpret_cast<const float4*>(a.part + (row + (size_t)p * LX_QUERIES) * (DB * 32) + c);
            const float f = __builtin_amdgcn_exp2f(ml.x - base);
            l = fmaf(f, ml.y, l);
            o.x = fmaf(f, v.x, o.x); o.y = fmaf(f, v.y, o.y); o.z = fmaf(f, v.z, o.z); o.w = fmaf(f, v.w, o.w);
        }
        if (!(fabsf(o.x) + fabsf(o.y) + fabsf(o.z) + fabsf(o.w) < INFINITY)) {      // what is infinite stays so however little its part weighs
            o = make_float4(0, 0, 0, 0);
            for (int p = 0; p < n; ++p) {
                const float f = __builtin_amdgcn_exp2f(a.ml[row + (size_t)p * LX_QUERIES].x - base);
                const float4 v = *reinterpret_cast<const float4*>(a.part + (row + (size_t)p * LX_QUERIES) * (DB * 32) + c);
                auto add = [&](float& to, float x) { to = fabsf(x) < INFINITY ? fmaf(f, x, to) : to + x; };
                add(o.x, v.x); add(o.y, v.y); add(o.z, v.z); add(o.w, v.w);
            }
        }
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        *reinterpret_cast<uint2*>(a.out + (((size_t)place.b * a.M + m) * a.heads + place.h) * a.dv + c) = make_uint2(f2bf2(o.x * inv, o.y * inv), f2bf2(o.z * inv, o.w * inv));
    }
#endif
}

template <int TILE> static int launch_tile(const LatentArgs& a, hipStream_t st) {
    constexpr int KD = kExpandedTiles[TILE].KD, DB = kExpandedTiles[TILE].DB, lds = 2 * (LX_BLOCK * KD * 32 + DB * 32 * 128);
    static_assert(expanded_per_cu(KD) * lds <= 160 * 1024, "LDS of a CU");
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&latent_expanded_kernel<KD, DB>), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (attr != hipSuccess) return fail(FISE_ERR_HIP, "fise_latent_attention: cannot raise the dynamic LDS limit");
    const int key_tiles = (int)(a.n_pad / LX_KEYS), k_tiles = ceil_div(a.heads * a.d, 128), v_tiles = ceil_div(a.heads * a.dv, 128);
    {
        ProfileScope prof(PROF_IGEMM_WIDE, 2.0 * a.B * a.n * a.heads * (double)a.r * (a.d + a.dv), 2.0 * a.B * a.n * (a.r + a.heads * (double)(a.d + a.dv)), st);
        hipLaunchKernelGGL(latent_expand_kernel, dim3((unsigned)(a.B * key_tiles * (k_tiles + v_tiles) + 1)), dim3(256), 2 * LE_STAGE, st, a, KD, key_tiles, k_tiles, v_tiles,
                           fast_div(std::max(key_tiles, 1)), fast_div(k_tiles + v_tiles));
    }
    FISE_CHECK_LAUNCH("fise_latent_attention: keys and values");
    {
        ProfileScope prof(PROF_ATTENTION, 2.0 * a.B * a.M * a.heads * (double)a.n * (a.d + a.dr + a.dv), 2.0 * a.B * a.n * a.heads * (double)(a.d + a.dr + a.dv), st);
        hipLaunchKernelGGL((latent_expanded_kernel<KD, DB>), dim3((unsigned)a.workgroups), dim3(256), lds, st, a);
    }
    FISE_CHECK_LAUNCH("fise_latent_attention: expanded");
    if (!a.whole) {
        ProfileScope prof(PROF_ATTENTION_MERGE, 0, 0, st);
        hipLaunchKernelGGL(latent_join_kernel<DB>, dim3((unsigned)a.groups, 4), dim3(256), 0, st, a);      // (fewer tiles than workgroups on the CUs: four for each)
    }
    FISE_CHECK_LAUNCH("fise_latent_attention: parts");
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
