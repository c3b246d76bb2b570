// Attention whose keys and values come from one latent vector c_j (r channels) and one shared key (dr channels) a token:
//   k[j, h] = [W_uk[h] c_j | k_pe_j],   v[j, h] = W_uv[h] c_j,   o[m, h] = softmax_j(q[m, h] . k[j, h] scale) v[j, h].
//
// Absorbed form (few queries): q . W_uk c = (W_uk^T q) . c, so W_uk goes to the queries once and W_uv to the sums at the end; in between every head reads the same
// rows [c | k_pe], which come in from the cache once for 64 rows (query, head).  Three launches: latent_query_kernel, latent_absorbed_kernel,
// latent_values_kernel.  Expanded form: latent_expanded.hip.
#include <algorithm>
#include "latent.h"

namespace fise {

// ---------------------------------------------------------------------------------------------------------------- queries
// qa[b, m, h] = [W_uk[h]^T q_c | q_pe | 0]: a workgroup has 128 latent channels of a head (a wave 32 of them) and takes 64 tokens at a time; W_uk's rows run along the
// result, so they are turned on the way out of LDS.  The result is rounded to bf16, which is what makes a result of this form 2.3e-3 off in the root mean square instead of the
// 1.66e-3 of its own rounding.  Two bf16 numbers would end that, and cost as many score products again: 16 elements of 16 rows on 8192 keys 40 -> 43 us, 32 of 64 rows on
// 20480 keys 205 -> 240.  All loads of a round go out together: few
// tokens wait for one trip to memory, not for one a step.  64 tokens of 32 heads, r 512: 9 us, bound by that trip; 128 tokens of 128 heads 24 us (41 MB).
// The last workgroup writes the line of key blocks instead: table[g] = blocks of all groups before g.
constexpr int LQ_COLS = 128, LQ_TOKENS = 64;
[[maybe_unused]] constexpr int LQ_STEPS = 5;                           // steps of 32 channels of d, at most 160
__global__ __launch_bounds__(256) void latent_query_kernel(const LatentArgs a, int R, int DR, int rounds) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int LQ_PITCH = LQ_COLS * 2 + 32;                         // four rows of a block side by side in the banks
    __shared__ __attribute__((aligned(16))) unsigned char lds[LQ_STEPS * 32 * LQ_PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, lq = lane >> 4;
    if (blockIdx.x == gridDim.x - 1) {
        if (blockIdx.y) return;
        la_line(a.table, a.groups, reinterpret_cast<int*>(lds), [&](int g) {
            const int b = (int)fdiv((unsigned)g, a.d_tiles), t = g - b * a.tiles;
            const int last = min(a.M * a.heads, (t + 1) * LA_ROWS) - 1;
            return (la_limit(a, la_len(a, b), (int)fdiv((unsigned)last, a.d_heads)) + LA_KEYS - 1) / LA_KEYS;
        });
        return;
    }
    const int cols = R / LQ_COLS, h = blockIdx.x / cols, c0 = (blockIdx.x - h * cols) * LQ_COLS, tokens = a.B * a.M, width = R + DR;
    const int steps = (a.d + 31) / 32;
    // (loads through buffers, which bring zeros for what does not exist: a condition would be a branch each)
    u32x4_t qv[LQ_TOKENS / 16][LQ_STEPS];
    const unsigned token_bytes = (unsigned)(a.heads * (a.d + a.dr) * 2);
    auto queries = [&](int t0) {
        const auto from = buf(a.q + ((size_t)t0 * a.heads + h) * (a.d + a.dr), (unsigned)(min(tokens - t0, LQ_TOKENS) - 1) * token_bytes + (unsigned)a.d * 2);
#pragma unroll
        for (int tt = 0; tt < LQ_TOKENS / 16; ++tt)
#pragma unroll
            for (int ks = 0; ks < LQ_STEPS; ++ks) {
                const int c = ks * 32 + lq * 8;
                qv[tt][ks] = __builtin_amdgcn_raw_buffer_load_b128(from, c < a.d ? (int)((unsigned)(tt * 16 + l16) * token_bytes + c * 2) : 0x7fffffff, 0, 0);
            }
    };
    {
        u32x4_t w[LQ_STEPS * 2];
        const int c = (tid & 15) * 8;
        const auto from = buf(a.w_uk + (size_t)h * a.d * a.r, (unsigned)(a.d * a.r * 2));
#pragma unroll
        for (int i = 0; i < LQ_STEPS * 2; ++i) w[i] = __builtin_amdgcn_raw_buffer_load_b128(from, c0 + c < a.r ? ((i * 16 + (tid >> 4)) * a.r + c0 + c) * 2 : 0x7fffffff, 0, 0);
        queries(blockIdx.y * LQ_TOKENS);
#pragma unroll
        for (int i = 0; i < LQ_STEPS * 2; ++i) *reinterpret_cast<u32x4_t*>(lds + (i * 16 + (tid >> 4)) * LQ_PITCH + c * 2) = w[i];
    }
    __syncthreads();
    const unsigned char* const from = lds + (lq * 8 + l16 / 4) * LQ_PITCH + (wave * 32 + (l16 % 4) * 4) * 2;
    for (int round = 0; round < rounds; ++round) {
        const int t0 = (round * gridDim.y + blockIdx.y) * LQ_TOKENS;
        if (t0 >= tokens) return;
        if (round) queries(t0);
#pragma unroll
        for (int tt = 0; tt < LQ_TOKENS / 16; ++tt) {
            if (t0 + tt * 16 >= tokens) return;
            const int t = t0 + tt * 16 + l16;
            f32x4_t acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
            for (int ks = 0; ks < LQ_STEPS; ++ks)
                if (ks < steps) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(la_turned(from + ks * 32 * LQ_PITCH + j * 32, 4 * LQ_PITCH), *reinterpret_cast<const bf16x8_t*>(&qv[tt][ks]),
                                                                         acc[j], 0, 0, 0);
                }
            if (t >= tokens) continue;
            bf16_t* const to = a.qa + ((size_t)t * a.heads + h) * width;
#pragma unroll
            for (int j = 0; j < 2; ++j)
                *reinterpret_cast<uint2*>(to + c0 + wave * 32 + j * 16 + lq * 4) = make_uint2(f2bf2(acc[j][0], acc[j][1]), f2bf2(acc[j][2], acc[j][3]));
            if (c0 == 0 && wave == 0)
                for (int c = lq * 8; c < DR; c += 32)
                    *reinterpret_cast<uint4*>(to + R + c) = c < a.dr ? *reinterpret_cast<const uint4*>(a.q + ((size_t)t * a.heads + h) * (a.d + a.dr) + a.d + c) : make_uint4(0, 0, 0, 0);
        }
    }
#endif
}

// ---------------------------------------------------------------------------------------------------------------- sums over the latent vectors
// A workgroup of four waves has 64 rows (query, head) and goes through its blocks of 32 keys; a block's rows [c | k_pe] lie in LDS, in a ring, loaded there
// directly two or three blocks ahead.  Scores: a wave has 16 rows, whose operands stay in registers, against all keys of the block.  The first index of the product is
// the key, and a lane reads the key rows in the order that makes its eight scores those of eight consecutive keys: its probabilities are
// then, as they stand, its part of the second product's operand.  Sums: the waves exchange probabilities and a wave has all 64 rows x a quarter
// of the latent channels, whose operand is the same block read turned, so nothing is read twice from memory and no transposed copy exists.
// Probabilities go in as two bf16 numbers, the second what rounding leaves of the first, for half as many products again: one number's rounding (2^-9 of each term, root mean
// square) would show as much as that of the result itself.  A long cache still waits for its bytes (32 tokens on 32768 keys: 189 -> 194 us for the whole call).
// A turn is the scores of one block and the sums of the block before, so that one barrier serves both and neither product waits for the softmax of its own block.
// 32 elements of 20480 keys on average, 64 rows, r 512: 162 - 197 us, 3.8 - 4.7 TB/s (the clock under load differs from card to card); the cache's bytes alone take 147, the matrix
// units are busy 39 % of the time, and a block of 32 keys for 64 rows takes 1.9 us a CU, a little more than its bytes do.
// A row's reference moves only when a score lies 8 powers of two above it: any reference gives the same quotient, probabilities stay below 256 (a bf16 and a float have
// the same relative steps there) and the factor for the sums before is 1 almost always.
template <int R_, int DR_, int NT> struct LaTile {
    static constexpr int R = R_, DR = DR_, PIECES = (R + DR) / 8, PITCH = PIECES * 16, TILE = LA_KEYS * PITCH, PER_CU = latent_per_cu(R);
    static constexpr int RING = R <= 256 || (R == 512 && DR && NT == 4) ? 3 : 4, AHEAD = RING - 1, LPW = TILE / 4096, RT = R / 64, KS = (R + DR) / 32;
    static constexpr int P = RING * TILE, PB = NT * 16 * LA_KEYS * 4, ALPHA = P + 2 * PB, AB = NT * 16 * 4, BAD = ALPHA + 2 * AB, LDS = BAD + 16;      // probabilities and factors: two of each; first key that is not finite
    // Place of a row's pieces.  A sixteen-byte read takes lanes 0-3, 12-15, 20-23, 24-27 at once (then the other sixteen of a half wave), which are sixteen keys of the
    // score product's operand, two neighbouring pieces alternating with key / 8; half a turned read takes two pieces of keys k .. k + 3 and k + 8 .. k + 11.  Both
    // meet every bank once.  (Where rows are 128 bytes off a multiple of 256, odd keys are in the other half of the banks anyway.)
    static constexpr int PERIOD = PITCH % 256 ? 8 : 16;
    static __device__ __forceinline__ int swizzle(int key) { return (PITCH % 256 ? 0 : (key & 1) << 3) | (key & 2) << 1 | (key & 8) >> 2; }
    static_assert(TILE % 4096 == 0 && PIECES % PERIOD == 0 && PER_CU * LDS <= 160 * 1024, "whole loads of four waves; LDS of a CU");
};

// NT: tiles of 16 rows that there are (4 but where a token's heads are few): the waves past them have no scores, and the sums are over those only.  16 elements of 16 rows, 8192 keys,
// whole call: 40 us, with four tiles 45; 32 rows and 1000 keys, r 256: 26, 27.5.
template <int R, int DR, int NT>
__global__ __launch_bounds__(256, latent_per_cu(R)) void latent_absorbed_kernel(const LatentArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    using T = LaTile<R, DR, NT>;
    constexpr int RT = T::RT, KS = T::KS, PITCH = T::PITCH, LPW = T::LPW, AHEAD = T::AHEAD;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, lq = lane >> 4;
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    const int wave = uniform(tid >> 6);
    // consecutive workgroups go to the eight XCDs in turn: give each XCD one run of the line
    const int total = uniform(a.table[a.groups]), workgroups = min(a.workgroups, total);      // each has a block
    int w = blockIdx.x;
    if (w >= workgroups) return;
    { const int chunk = workgroups >> 3; if (w < chunk << 3) w = (w & 7) * chunk + (w >> 3); }
    const int line0 = uniform((int)((long long)w * total / workgroups)), line1 = uniform((int)((long long)(w + 1) * total / workgroups));
    int g = la_group(a.table, a.groups, line0);
    const int row_bytes = (a.r + a.dr) * 2, rows = a.M * a.heads;

    // ---- places that depend on the lane only: loads (offset of a piece in a block of the cache; pieces that do not exist past its end), operands
    unsigned off[LPW];
#pragma unroll
    for (int j = 0; j < LPW; ++j) {
        const int p = (wave * LPW + j) * 64 + lane, key = p / T::PIECES, piece = (p - key * T::PIECES) ^ T::swizzle(key);
        const int c = piece * 8, pe = c - R;
        off[j] = c < R ? (c < a.r ? (unsigned)(key * row_bytes + c * 2) : 0x40000000u) : (pe < a.dr ? (unsigned)(key * row_bytes + (a.r + pe) * 2) : 0x40000000u);
    }
    const int my_key = (l16 >> 2) * 8 + (l16 & 3);                     // of the first half of a block's scores; the second half's is 4 further
    constexpr int KB = T::PERIOD / 4;                                  // steps after which the places repeat
    unsigned kat[KB];
#pragma unroll
    for (int j = 0; j < KB; ++j) kat[j] = (unsigned)(my_key * PITCH + ((j * 4 + lq) ^ T::swizzle(my_key)) * 16);
    constexpr int VB = RT < T::PERIOD / 2 ? RT : T::PERIOD / 2;
    unsigned vat[VB];
    {
        const int key = lq * 8 + l16 / 4;
#pragma unroll
        for (int j = 0; j < VB; ++j) vat[j] = (unsigned)(key * PITCH + (((wave * RT + j) * 2 + (l16 % 4) / 2) ^ T::swizzle(key)) * 16 + (l16 & 1) * 8);
    }
    const unsigned lds0 = (unsigned)(size_t)(FISE_AS3 unsigned char*)(FISE_AS3 void*)lds;

    for (int at = line0; at < line1; ++g) {
        const int b = uniform((int)fdiv((unsigned)g, a.d_tiles)), row0 = (g - b * a.tiles) * LA_ROWS;
        const int2 of_g = make_int2(a.table[g], a.table[g + 1]);       // (with the length: one trip)
        const int len = uniform(la_len(a, b)), g_at = uniform(of_g.x), end = min(line1, uniform(of_g.y));
        if (end <= at) continue;
        const int blk0 = at - g_at, blk1 = end - g_at;
        const int row = row0 + wave * 16 + l16;
        const int sees = row < rows ? la_limit(a, len, (int)fdiv((unsigned)row, a.d_heads)) : len;
        const int limit = min(sees, blk1 * LA_KEYS);                   // (behind this part's last block: nothing)
        const int limit_first = la_limit(a, len, (int)fdiv((unsigned)row0, a.d_heads));       // the fewest keys that a row of the tile sees
        const unsigned char* const keys = (const unsigned char*)a.cache + (size_t)b * a.cache_tokens * row_bytes;

        int put = 0, get = 0;                                          // places in the ring
        auto next = [](int x) { return x == AHEAD * T::TILE ? 0 : x + T::TILE; };
        auto load = [&](int blk) {                                     // (behind the last block: nothing but zeros, no traffic, the same count of loads)
            const int k0 = blk * LA_KEYS, left = min(max(len - k0, 0), LA_KEYS);
            const u32x4_t from = la_buffer(keys + (size_t)k0 * row_bytes, blk < blk1 ? left * row_bytes : 0);
            const unsigned to = uniform(lds0 + put + wave * LPW * 1024);
            put = next(put);
#pragma unroll
            for (int j = 0; j < LPW; ++j) la_to_lds(from, off[j], to + j * 1024);
        };
        bf16x8_t qf[KS];
        {
            const bf16_t* const q = a.qa + ((size_t)b * rows + min(row, rows - 1)) * (R + DR) + lq * 8;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const bf16x8_t*>(q + ks * 32);
        }
        la_barrier();                                                  // the group before has been read to its end
        int* const bad = reinterpret_cast<int*>(lds + T::BAD);
        if (tid == 0) *bad = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) load(blk0 + i);
        // the queries have arrived before the loop (the compiler's count would otherwise wait for every load in flight)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" ::"v"(qf[ks]));

        const bool has_rows = NT == 4 || wave < NT;
        f32x4_t acc[RT][NT];
#pragma unroll
        for (int j = 0; j < RT; ++j)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[j][t] = f32x4_t{0, 0, 0, 0};
        float m_run = -INFINITY, l_run = 0.f;                          // l: of this lane's keys until the end

        // Product m of the scores takes key rows of half m & 1, step m >> 1; reads go out LA_AHEAD products before theirs.
        constexpr int LA_AHEAD = 6, NK = 2 * KS, RK = LA_AHEAD + 1;
        f32x4_t s[2][2];
        bf16x8_t kf[RK];
        auto read_k = [&](const unsigned char* tile, int m) { return *reinterpret_cast<const bf16x8_t*>(tile + kat[(m >> 1) % KB] + (m >> 1) / KB * (T::PERIOD * 16) + (m & 1) * 4 * PITCH); };
        auto score = [&](int m) {
            f32x4_t& to = s[m & 1][(m >> 1) & 1];
            to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[m % RK], qf[m >> 1], m < 4 ? f32x4_t{0, 0, 0, 0} : to, 0, 0, 0);
        };
        // softmax of a block in five pieces: scores of eight keys a lane, k0 + lq * 8 + (0..7); their maximum; the reference and the factor for the sums before;
        // probabilities; those and the factor to LDS
        float p[8], mx, alpha;
        auto softmax = [&](int piece, int k0, int which) {
            if (piece == 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    p[e] = (s[e >> 2][0][e & 3] + s[e >> 2][1][e & 3]) * a.scale_log2e;
                    if (k0 + lq * 8 + e >= limit) p[e] = -INFINITY;
                }
            } else if (piece == 1) {
                mx = la_max4(fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7]))));
            } else if (piece == 2) {
                mx = mx > m_run + 8.f ? mx : m_run;                    // (the first block: above -inf)
                const float base = mx == -INFINITY ? 0.f : mx;         // nothing seen yet: every probability is exp2(-inf) = 0
                alpha = __builtin_amdgcn_exp2f(m_run - base);
                m_run = mx;
#pragma unroll
                for (int e = 0; e < 8; ++e) p[e] -= base;
            } else if (piece == 3) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) { p[e] = __builtin_amdgcn_exp2f(p[e]); sum += p[e]; }
                l_run = fmaf(l_run, alpha, sum);
            } else {
                unsigned high[4], low[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    high[e] = f2bf2(p[2 * e], p[2 * e + 1]);
                    low[e] = f2bf2(p[2 * e] - lo16(high[e]), p[2 * e + 1] - hi16(high[e]));
                }
                *reinterpret_cast<uint4*>(lds + T::P + which * T::PB + tid * 16) = make_uint4(high[0], high[1], high[2], high[3]);
                *reinterpret_cast<uint4*>(lds + T::P + which * T::PB + T::PB / 2 + tid * 16) = make_uint4(low[0], low[1], low[2], low[3]);
                if (lq == 0) *reinterpret_cast<float*>(lds + T::ALPHA + which * T::AB + (wave * 16 + l16) * 4) = alpha;
            }
        };
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((AHEAD - 1) * LPW) : "memory");
        if (has_rows) {
#pragma unroll
            for (int m = 0; m < NK; ++m) { kf[m % RK] = read_k(lds, m); score(m); }
#pragma unroll
            for (int i = 0; i < 5; ++i) softmax(i, blk0 * LA_KEYS, 0);
        }
        int which = 0;
        for (int blk = blk0; blk < blk1; ++blk, which ^= 1) {
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((AHEAD - 2) * LPW) : "memory");
            load(blk + AHEAD);                                         // over the block before, which all waves are done with
            const unsigned char* const tile = lds + get;
            get = next(get);
            if (a.causal && blk * LA_KEYS + LA_KEYS > limit_first) {
                // a key that a row does not see takes part with probability 0: what is not finite in it must not.  A row that does see it is NaN (its score is NaN or
                // infinite, and the probability 0 of a score of -inf meets a value that is not finite)
                int first = 0x7fffffff;
                for (int i = tid; i < LA_KEYS * (R / 8); i += 256) {
                    const int key = i / (R / 8), piece = (i - key * (R / 8)) ^ T::swizzle(key);
                    uint4* const at16 = reinterpret_cast<uint4*>(const_cast<unsigned char*>(tile) + key * PITCH + piece * 16);
                    const uint4 v = *at16;
                    if (la_odd(v)) { *at16 = la_finite(v); first = min(first, blk * LA_KEYS + key); }
                }
                if (first != 0x7fffffff) atomicMin(bad, first);
                la_barrier();
                if (*bad < limit) l_run = NAN;
            }
            if (has_rows) {
#pragma unroll
                for (int m = 0; m < LA_AHEAD; ++m) kf[m] = read_k(lds + get, m);
            }
            float al[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) al[t] = *reinterpret_cast<const float*>(lds + T::ALPHA + which * T::AB + (t * 16 + l16) * 4);
            bool moved = false;
#pragma unroll
            for (int t = 0; t < NT; ++t) moved |= al[t] != 1.0f;
            if (__any(moved)) {                                        // a reference has moved, which becomes rare
#pragma unroll
                for (int j = 0; j < RT; ++j)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[j][t][e] *= al[t];
            }
            // ---- scores of the next block, then sums of this one (a quarter of the latent channels for all 64 rows) with the softmax of the next between them; in this
            // order, which the compiler's own would give up for fewer registers: every product would wait for its operand
            bf16x8_t pf[NT], pl[NT], vf[2];
            auto read_v = [&](int j) { return la_turned(tile + vat[j % VB] + j / VB * (T::PERIOD * 16), 4 * PITCH); };
            auto read_p = [&](int t) { return *reinterpret_cast<const bf16x8_t*>(lds + T::P + which * T::PB + (t * 64 + lane) * 16); };
            __builtin_amdgcn_sched_barrier(0);
            if (has_rows) {
#pragma unroll
                for (int m = 0; m < NK; ++m) {
                    if (m + LA_AHEAD < NK) kf[(m + LA_AHEAD) % RK] = read_k(lds + get, m + LA_AHEAD);
                    else if (m + LA_AHEAD < NK + NT) pf[m + LA_AHEAD - NK] = read_p(m + LA_AHEAD - NK);
                    else if (m + LA_AHEAD == NK + NT) vf[0] = read_v(0);
                    __builtin_amdgcn_sched_barrier(0);
                    score(m);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
#pragma unroll
                for (int t = 0; t < NT; ++t) pf[t] = read_p(t);
                vf[0] = read_v(0);
            }
            static_assert(LA_AHEAD > 4, "probabilities and the first values are read with the last scores");
#pragma unroll
            for (int t = 0; t < NT; ++t) pl[t] = *reinterpret_cast<const bf16x8_t*>(lds + T::P + which * T::PB + T::PB / 2 + (t * 64 + lane) * 16);
#pragma unroll
            for (int j = 0; j < RT; ++j) {
                if (j + 1 < RT) vf[(j + 1) & 1] = read_v(j + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[j & 1], pf[t], acc[j][t], 0, 0, 0);
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[j & 1], pl[t], acc[j][t], 0, 0, 0);
                if (has_rows && (j * 5 / RT != (j + 1) * 5 / RT || RT < 5))        // five pieces over the RT steps (fewer steps than pieces: what is left at the end)
                    softmax(RT < 5 ? j : j * 5 / RT, (blk + 1) * LA_KEYS, which ^ 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (has_rows)
#pragma unroll
                for (int i = RT; i < 5; ++i) softmax(i, (blk + 1) * LA_KEYS, which ^ 1);
        }
        at = end;
        // ---- partial result of this part of the group
        const size_t slot = (size_t)w + g;
        l_run = la_sum4(l_run);
        if (has_rows && lq == 0) a.ml[slot * LA_ROWS + wave * 16 + l16] = make_float2(m_run, l_run);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (row0 + t * 16 + l16 >= rows) continue;
            float* const o = a.part + (slot * LA_ROWS + t * 16 + l16) * R + wave * (RT * 16) + lq * 4;
#pragma unroll
            for (int j = 0; j < RT; ++j) *reinterpret_cast<float4*>(o + j * 16) = make_float4(acc[j][t][0], acc[j][t][1], acc[j][t][2], acc[j][t][3]);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");               // the empty loads behind the last block and the stores: the next group counts from nothing
    }
#endif
}

// ---------------------------------------------------------------------------------------------------------------- values
// o[t, h] = W_uv[h] (sum over the parts).  A workgroup of eight waves has a head and `tokens` tokens (at most 16): it adds up the parts with their weights
// exp2(m - max), divides, and leaves the sums in LDS as two bf16 numbers each (16 of the float's 24 bits, so that this product rounds only its result);
// the waves take 16 value channels at a time.  2048 rows, r 512: 17 us for 38 MB of parts and W_uv for every four tokens; 256 rows 9 us, which is trips to memory.
template <int R>
__global__ __launch_bounds__(512, 4) void latent_values_kernel(const LatentArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int QUADS = R / 4, PARTS = 512 / QUADS, PITCH = R + 8;   // parts: lanes that share the parts of a token, or have tokens of their own
    __shared__ __attribute__((aligned(16))) bf16_t hi[16][PITCH], lo[16][PITCH];
    __shared__ __attribute__((aligned(16))) float4 sums[PARTS][QUADS];
    __shared__ float2 stats[16];                                       // of a token: reference, 1 / sum
    __shared__ size_t first[16];                                       // its first part's place
    __shared__ int count[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, lq = lane >> 4;
    const int h = blockIdx.x, t0 = blockIdx.y * a.tokens, tokens = min(a.tokens, a.B * a.M - t0);
    const int part = tid / QUADS, quad = tid - part * QUADS;
    const int total = a.table[a.groups], workgroups = min(a.workgroups, total);
    const int vt = (a.dv + 15) / 16;
    auto weights = [&](bf16x8_t (&wf)[R / 32], int v) {
        const bf16_t* const w = a.w_uv + ((size_t)h * a.dv + v * 16 + l16) * a.r;
#pragma unroll
        for (int ks = 0; ks < R / 32; ++ks) {
            uint4 x = make_uint4(0, 0, 0, 0);
            if (v * 16 + l16 < a.dv && ks * 32 + lq * 8 < a.r) x = *reinterpret_cast<const uint4*>(w + ks * 32 + lq * 8);
            wf[ks] = *reinterpret_cast<const bf16x8_t*>(&x);
        }
    };
    // ---- what the parts of each token weigh: 32 lanes a token go over its parts (workgroups that had some of its group's blocks), keeping a maximum
    // and a sum, and meet.  l == 0: no key was seen, zeros.
    if (tid < a.tokens * 32) {
        const int i = tid >> 5, t = t0 + i;
        if (i < tokens) {
            const int b = (int)fdiv((unsigned)t, a.d_M), row = (t - b * a.M) * a.heads + h, tile = row / LA_ROWS, g = b * a.tiles + tile;
            const int g0 = a.table[g], g1 = a.table[g + 1];
            const int w0 = g1 > g0 ? la_owner(g0, workgroups, total) : 0, n = g1 > g0 ? la_owner(g1 - 1, workgroups, total) - w0 + 1 : 0;
            const size_t at = ((size_t)g + w0) * LA_ROWS + (row - tile * LA_ROWS);
            float top = -INFINITY, l = 0.f;
            for (int p = tid & 31; p < n; p += 32) {
                const float2 v = a.ml[at + (size_t)p * LA_ROWS];
                const float m = fmaxf(top, v.x), base = m == -INFINITY ? 0.f : m;
                l = l * __builtin_amdgcn_exp2f(top - base) + v.y * __builtin_amdgcn_exp2f(v.x - base);
                top = m;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                const float mo = __shfl_xor(top, o), lo_ = __shfl_xor(l, o), m = fmaxf(top, mo), base = m == -INFINITY ? 0.f : m;
                l = l * __builtin_amdgcn_exp2f(top - base) + lo_ * __builtin_amdgcn_exp2f(mo - base);
                top = m;
            }
            if ((tid & 31) == 0) { stats[i] = make_float2(top == -INFINITY ? 0.f : top, l == 0.f ? 0.f : 1.0f / l); first[i] = at; count[i] = n; }
        }
    }
    __syncthreads();
    // the sums of token t0 + i over every `step`-th part from the first + `from` on
    auto merge = [&](int i, int from, int step) {
        float4 o = make_float4(0, 0, 0, 0);
        const float2 st = stats[i];
        const int n = count[i];
        const float2* const ml = a.ml + first[i];
        const float* const part_o = a.part + first[i] * R + quad * 4;
        for (int p0 = from; p0 < n; p0 += 4 * step) {                  // four parts requested at once (behind the last: that one again, without weight)
            float4 v[4];
            float f[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const size_t p = min(p0 + u * step, n - 1);
                f[u] = ml[p * LA_ROWS].x;
                v[u] = *reinterpret_cast<const float4*>(part_o + p * (LA_ROWS * R));
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float w = p0 + u * step < n ? __builtin_amdgcn_exp2f(f[u] - st.x) * st.y : 0.f;
                o.x = fmaf(w, v[u].x, o.x); o.y = fmaf(w, v[u].y, o.y); o.z = fmaf(w, v[u].z, o.z); o.w = fmaf(w, v[u].w, o.w);
            }
        }
        return o;
    };
    auto put = [&](int i, float4 o) {
        const unsigned h0 = f2bf2(o.x, o.y), h1 = f2bf2(o.z, o.w);
        auto rest = [](float v, float high) { return (__float_as_uint(high) & 0x7f800000u) == 0x7f800000u ? 0.f : v - high; };
        *reinterpret_cast<uint2*>(&hi[i][quad * 4]) = make_uint2(h0, h1);
        *reinterpret_cast<uint2*>(&lo[i][quad * 4]) = make_uint2(f2bf2(rest(o.x, lo16(h0)), rest(o.y, hi16(h0))), f2bf2(rest(o.z, lo16(h1)), rest(o.w, hi16(h1))));
    };
    // as many lane groups as tokens, or the groups deal a token's parts out among them
    const int share = a.tokens >= PARTS ? 1 : PARTS / a.tokens;
    if (share == 1) {
        if (part < PARTS)
            for (int i = part; i < tokens; i += PARTS) put(i, merge(i, 0, 1));
    } else {
        const int i = part / share, mine = part - i * share;
        const bool works = part < PARTS && i < tokens;
        float4 o = make_float4(0, 0, 0, 0);
        if (works) sums[part][quad] = o = merge(i, mine, share);
        __syncthreads();
        if (works && mine == 0) {
            for (int k = 1; k < share; ++k) { const float4 v = sums[part + k][quad]; o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w; }
            put(i, o);
        }
    }
    bf16x8_t wf[R / 32];
    if (wave < vt) weights(wf, wave);
    __syncthreads();
    const int src = l16 < tokens ? l16 : 0;                            // (tokens that do not exist: the first one's sums, not stored)
    for (int v = wave; v < vt; v += 8) {
        if (v != wave) weights(wf, v);
        f32x4_t acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
        for (int ks = 0; ks < R / 32; ++ks) {
            acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[ks], *reinterpret_cast<const bf16x8_t*>(&hi[src][ks * 32 + lq * 8]), acc[0], 0, 0, 0);
            acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[ks], *reinterpret_cast<const bf16x8_t*>(&lo[src][ks * 32 + lq * 8]), acc[1], 0, 0, 0);
            if (ks % 4 == 3) __builtin_amdgcn_sched_barrier(0);        // (all sums read at once would not leave room for a second workgroup on the CU)
        }
        const int c = v * 16 + lq * 4;
        if (l16 < tokens && c < a.dv)
            *reinterpret_cast<uint2*>(a.out + ((size_t)(t0 + l16) * a.heads + h) * a.dv + c) =
                make_uint2(f2bf2(acc[0][0] + acc[1][0], acc[0][1] + acc[1][1]), f2bf2(acc[0][2] + acc[1][2], acc[0][3] + acc[1][3]));
    }
#endif
}

template <int R, int DR, int NT> static int launch_absorbed(const LatentArgs& a, hipStream_t st) {
    using T = LaTile<R, DR, NT>;
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(&latent_absorbed_kernel<R, DR, NT>), hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS);
    if (attr != hipSuccess) return fail(FISE_ERR_HIP, "fise_latent_attention: cannot raise the dynamic LDS limit");
    const int tokens = a.B * a.M;
    // up to three workgroups a CU, which take several rounds of tokens where there are more
    const int cols = a.heads * (R / LQ_COLS), tiles = ceil_div(tokens, LQ_TOKENS), rounds = ceil_div(tiles, std::max(1, 3 * LA_CUS / cols));
    hipLaunchKernelGGL(latent_query_kernel, dim3((unsigned)cols + 1, (unsigned)ceil_div(tiles, rounds)), dim3(256), 0, st, a, R, DR, rounds);
    FISE_CHECK_LAUNCH("fise_latent_attention: queries");
    {
        const double pairs = (double)tokens * a.heads * a.n;
        ProfileScope prof(PROF_ATTENTION, 2.0 * pairs * (2 * a.r + a.dr), 2.0 * a.B * a.n * (a.r + a.dr), st);
        hipLaunchKernelGGL((latent_absorbed_kernel<R, DR, NT>), dim3((unsigned)a.workgroups), dim3(256), T::LDS, st, a);
    }
    FISE_CHECK_LAUNCH("fise_latent_attention: absorbed");
    {
        ProfileScope prof(PROF_ATTENTION_MERGE, 2.0 * tokens * a.heads * (double)a.r * a.dv, 2.0 * a.heads * (double)a.r * a.dv, st);
        hipLaunchKernelGGL(latent_values_kernel<R>, dim3((unsigned)a.heads, (unsigned)ceil_div(tokens, a.tokens)), dim3(512), 0, st, a);
    }
    FISE_CHECK_LAUNCH("fise_latent_attention: values");
    return FISE_OK;
}
template <int R, int DR> static int launch_absorbed(const LatentArgs& a, hipStream_t st) {
    return a.M * a.heads <= 16 ? launch_absorbed<R, DR, 1>(a, st) : a.M * a.heads <= 32 ? launch_absorbed<R, DR, 2>(a, st) : launch_absorbed<R, DR, 4>(a, st);
}
template <int R> static int launch_absorbed(const LatentArgs& a, hipStream_t st) { return a.dr ? launch_absorbed<R, 64>(a, st) : launch_absorbed<R, 0>(a, st); }

// What a launch's grid and 31 bits hold: blocks of keys of all tiles; of the expanded form tiles of queries and of keys x weights, too, 256 lanes each.
static bool absorbed_holds(const LatentShape& s) {
    const long long tiles = (long long)s.B * absorbed_tiles(s);
    return tiles < 1ll << 30 && tiles * ((s.n + LA_KEYS - 1) / LA_KEYS + 1) < 1ll << 31;
}
static bool expanded_holds(const LatentShape& s) {
    const double groups = (double)s.B * s.heads * expanded_tiles(s), makes = (double)s.B * (s.n / LX_KEYS + 1) * ((double)s.heads * (s.d + s.dv) / 128 + 2);
    return groups < 1 << 24 && makes < 1 << 24 && groups * (s.n / LX_BLOCK + 1) < 0x7fffffff;
}
// AUTO: the faster one of those that hold the call
static bool expands(int form, const LatentShape& s) {
    return form == FISE_LATENT_AUTO ? (latent_expands(s) ? expanded_holds(s) || !absorbed_holds(s) : !absorbed_holds(s)) : form == FISE_LATENT_EXPANDED;
}
static int latent_check(const char* fn, const fise_latent_attention_args* g, LatentShape& s) {
    if (!g || !g->q || !g->cache || !g->w_uk || !g->w_uv || !g->out) return fail(FISE_ERR_NULL, "%s: null pointer", fn);
    if (g->dtype != FISE_BF16) return fail(FISE_ERR_DTYPE, "%s: dtype %d (bf16 only)", fn, g->dtype);
    if (g->B < 1 || g->M < 0 || g->n_keys < 0 || g->cache_tokens < g->n_keys || g->heads < 1 || g->d < 1 || g->d > 160 || g->dv < 1 || g->dv > 160 || g->dr < 0 || g->dr > 64 ||
        g->r < 1 || g->r > 512 || g->form < FISE_LATENT_AUTO || g->form > FISE_LATENT_EXPANDED)
        return fail(FISE_ERR_SHAPE, "%s: B%d M%d keys%d of %lld heads%d d%d dr%d dv%d r%d form%d", fn, g->B, g->M, g->n_keys, (long long)g->cache_tokens, g->heads, g->d, g->dr, g->dv, g->r, g->form);
    if (g->d % 8 || g->dr % 8 || g->dv % 8 || g->r % 8) return fail(FISE_ERR_ALIGN, "%s: d %d, dr %d, dv %d and r %d must be multiples of 8", fn, g->d, g->dr, g->dv, g->r);
    for (const void* p : {g->q, g->cache, g->w_uk, g->w_uv, (const void*)g->out})
        if (!aligned16(p)) return fail(FISE_ERR_ALIGN, "%s: pointers must be 16-byte aligned", fn);
    if (!(g->scale > 0) || g->scale > 1e30f) return fail(FISE_ERR_SHAPE, "%s: scale %g", fn, g->scale);
    s = LatentShape{g->B, g->M, g->n_keys, g->heads, g->d, g->dr, g->dv, g->r, g->causal != 0};
    // limits of either form (tokens: the absorbed one's, a grid's second dimension, but what AUTO refuses should not depend on what it would choose); then of the one that runs
    if (g->n_keys > 1 << 26 || (long long)g->M * g->heads >= 1ll << 30 || (long long)g->B * g->M >= 1 << 20 || g->heads > 65535 || !(expands(g->form, s) ? expanded_holds(s) : absorbed_holds(s)))
        return fail(FISE_ERR_SHAPE, "%s: B%d M%d heads%d keys%d: too many rows, tiles or key blocks", fn, g->B, g->M, g->heads, g->n_keys);
    return FISE_OK;
}

}  // namespace fise

using namespace fise;

extern "C" size_t fise_latent_attention_workspace_bytes(const fise_latent_attention_args* g) {
    LatentShape s;
    if (latent_check("fise_latent_attention_workspace_bytes", g, s)) return 0;
    if (s.M == 0) return 256;
    return expands(g->form, s) ? expanded_layout(s).total : absorbed_layout(s).total;
}

extern "C" int fise_latent_attention(const fise_latent_attention_args* g, void* workspace, size_t workspace_bytes, void* stream) {
    const char* fn = "fise_latent_attention";
    LatentShape s;
    if (int e = latent_check(fn, g, s)) return e;
    if (s.M == 0) return FISE_OK;
    if (!workspace) return fail(FISE_ERR_NULL, "%s: null workspace", fn);
    if ((uintptr_t)workspace & 255) return fail(FISE_ERR_ALIGN, "%s: the workspace must be 256-byte aligned", fn);
    const bool expanded = expands(g->form, s);
    const size_t need = expanded ? expanded_layout(s).total : absorbed_layout(s).total;
    if (workspace_bytes < need) return fail(FISE_ERR_CAPACITY, "%s: workspace of %zu bytes, %zu needed", fn, workspace_bytes, need);
    unsigned char* const ws = (unsigned char*)workspace;
    LatentArgs a{};
    a.q = (const bf16_t*)g->q; a.cache = (const bf16_t*)g->cache; a.kv_len = g->kv_len; a.w_uk = (const bf16_t*)g->w_uk; a.w_uv = (const bf16_t*)g->w_uv; a.out = (bf16_t*)g->out;
    a.B = s.B; a.M = s.M; a.n = s.n; a.heads = s.heads; a.d = s.d; a.dr = s.dr; a.dv = s.dv; a.r = s.r; a.causal = s.causal; a.cache_tokens = g->cache_tokens;
    a.scale_log2e = g->scale * 1.4426950408889634f;
    a.d_heads = fast_div(s.heads); a.d_M = fast_div(s.M);
    const hipStream_t st = as_stream(stream);
    if (expanded) {
        const ExpandedLayout l = expanded_layout(s);
        a.n_pad = l.n_pad; a.k = (bf16_t*)(ws + l.k); a.v = (bf16_t*)(ws + l.v); a.flags = (unsigned*)(ws + l.flags);
        a.tiles = expanded_tiles(s); a.groups = (int)expanded_groups(s); a.whole = expanded_whole(s); a.workgroups = expanded_workgroups(s); a.d_tiles = fast_div(a.tiles);
        a.table = (int*)(ws + l.table); a.ml = (float2*)(ws + l.ml); a.part = (float*)(ws + l.part);
        return launch_expanded(a, expanded_tile(s), st);
    }
    const AbsorbedLayout l = absorbed_layout(s);
    a.tiles = absorbed_tiles(s); a.groups = s.B * a.tiles; a.workgroups = absorbed_workgroups(s); a.tokens = absorbed_tokens(s);
    a.table = (int*)(ws + l.table); a.qa = (bf16_t*)(ws + l.q); a.ml = (float2*)(ws + l.ml); a.part = (float*)(ws + l.part);
    a.d_tiles = fast_div(a.tiles);
    switch (latent_width(s.r)) {
    case 128: return launch_absorbed<128>(a, st);
    case 256: return launch_absorbed<256>(a, st);
    case 384: return launch_absorbed<384>(a, st);
    default: return launch_absorbed<512>(a, st);
    }
}
