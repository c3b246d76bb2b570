// What the two forms of attention over a cache of latent vectors share.  Internal.
#pragma once
#include "igemm.h"
#include "latent_choice.h"
#include "profile.h"

namespace fise {

struct LatentArgs {
    const bf16_t* q; const bf16_t* cache; const int* kv_len; const bf16_t* w_uk; const bf16_t* w_uv; bf16_t* out;
    int B, M, n, heads, d, dr, dv, r, causal; long long cache_tokens;
    float scale_log2e;
    int tiles, groups, workgroups;                       // tiles of rows or queries; of all elements (and heads); workgroups that share the line of key blocks
    int* table; float2* ml; float* part;                 // the line; of every part: reference and sum of a row, sums
    // absorbed
    int tokens; bf16_t* qa;                              // tokens of a workgroup of the third launch; queries behind W_uk
    // expanded
    int whole;                                           // a workgroup for every tile
    long long n_pad; bf16_t* k; bf16_t* v;               // keys of a head [B, heads, n_pad, 16 KD], values [B, heads * dv, n_pad]
    unsigned* flags;                                     // [B, value tiles, key tiles]: a byte for each wave that made the tile, not 0 if it holds a value that is not finite
    FastDiv d_heads, d_tiles, d_M;
};

// Keys of a batch element, and how many of them query m sees: all, or (causal) the query is the key at len - M + m and sees those up to itself.
__device__ __forceinline__ int la_len(const LatentArgs& a, int b) { return a.kv_len ? min(max(a.kv_len[b], 0), a.n) : a.n; }
__device__ __forceinline__ int la_limit(const LatentArgs& a, int len, int m) { return a.causal ? min(max(len - a.M + m + 1, 0), len) : len; }

// The line of key blocks: table[g] = blocks of all groups before g, by a workgroup of 256 lanes.  Workgroup w of G has blocks w T / G .. (w + 1) T / G of the T.
template <typename F> __device__ __forceinline__ void la_line(int* table, int groups, int* lds, F&& blocks) {
    const int tid = threadIdx.x, each = (groups + 255) / 256, g0 = min(tid * each, groups), g1 = min(g0 + each, groups);
    int s = 0;
    for (int g = g0; g < g1; ++g) s += blocks(g);
    lds[tid] = s;
    __syncthreads();
    for (int o = 1; o < 256; o <<= 1) {
        const int v = tid >= o ? lds[tid - o] : 0;
        __syncthreads();
        lds[tid] += v;
        __syncthreads();
    }
    int at = lds[tid] - s;
    for (int g = g0; g < g1; ++g) { table[g] = at; at += blocks(g); }
    if (tid == 255) table[groups] = lds[255];
}
// the workgroup that has block x: the largest w with w total / workgroups <= x
__device__ __forceinline__ int la_owner(int x, int workgroups, int total) { return (int)((((long long)x + 1) * workgroups - 1) / total); }
// last group that starts at or before block x: 64 entries at a time, one trip to memory for up to 64 groups, two for 4096
__device__ __forceinline__ int la_group(const int* table, int groups, int x) {
    int lo = 0;
    for (int n = groups; n > 1;) {
        const int step = (n + 63) >> 6, i = (int)(threadIdx.x & 63) * step;
        const int below = __popcll(__ballot(i < n && table[lo + min(i, n - 1)] <= x)) - 1;      // (the first is always)
        lo += below * step;
        n = min(step, n - below * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

__device__ __forceinline__ void la_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

#if defined(__HIP_DEVICE_COMPILE__)
// A raw buffer of `bytes` from a base that is the same for all lanes, in scalar registers whatever the compiler knows of it (see buf()).
__device__ __forceinline__ u32x4_t la_buffer(const void* p, int bytes) {
    const unsigned long long a = (unsigned long long)(size_t)p;
    return u32x4_t{(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)a), (unsigned)__builtin_amdgcn_readfirstlane((int)((a >> 32) & 0xffff)), (unsigned)__builtin_amdgcn_readfirstlane(bytes),
                   0x00020000u};
}
// Sixteen bytes a lane from there to LDS, the lanes side by side from `to` on; offsets that are not below the buffer's size bring zeros.  Written out because the
// compiler waits for every load of the builtin that is in flight in front of a turned read or a write of LDS; whoever reads what it brings waits by its count.
// (m0 is changed: nothing else in these kernels uses it.)
__device__ __forceinline__ void la_to_lds(u32x4_t from, unsigned off, unsigned to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(from), "s"(to) : "memory");
}
typedef short s16x4_t __attribute__((ext_vector_type(4)));
// Sixteen lanes read a block of 4 rows x 16 columns (lane i: four columns from 4 (i % 4) of row i / 4) and get it turned: lane i column i, all four rows.
// Two blocks are the operand of a 16x16x32 product whose summed index runs down the rows: row groups `at` and `at` + second.
__device__ __forceinline__ bf16x8_t la_turned(const unsigned char* at, int second) {
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FISE_AS3 s16x4_t*)(FISE_AS3 void*)at);
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((FISE_AS3 s16x4_t*)(FISE_AS3 void*)(at + second));
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}
// bf16 pairs whose values that are not finite are zeros
__device__ __forceinline__ uint4 la_finite(uint4 v) {
    auto clean = [](unsigned x) {
        if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
        if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
        return x;
    };
    return make_uint4(clean(v.x), clean(v.y), clean(v.z), clean(v.w));
}
// whether one of those values is not finite
__device__ __forceinline__ bool la_odd(uint4 v) {
    const uint4 f = la_finite(v);
    return ((v.x ^ f.x) | (v.y ^ f.y) | (v.z ^ f.z) | (v.w ^ f.w)) != 0;
}
// over the four lanes l, l + 16, l + 32, l + 48
__device__ __forceinline__ float la_max4(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}
__device__ __forceinline__ float la_sum4(float x) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}
#endif

int launch_expanded(const LatentArgs& a, int tile, hipStream_t st);

}  // namespace fise
