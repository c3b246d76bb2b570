// Products of few 8-bit rows with 8-bit weights, which stream the weights past the rows: what fp8.hip and experts.hip share.  Internal.
//
// The weights' bytes and the trips to memory bound it, not products: a workgroup has sixteen outputs (experts: of gate and of up), its waves share the columns block by block, a
// wave's loads are the lines of sixteen rows, and the waves' sums meet in LDS, added in their order.  Rows that are not in 8 bits yet are put there in registers: a lane has 32 columns of a
// block of its token, four lanes the block.  The codes go to the products as bf16, whose sums lose nothing (fp8_tile.h).
// One row, 1280 outputs of 320 columns: 5 us, a launch; 54 rows, 1283 of 5136: 11 us behind the 4 of the launch that puts them in 8 bits; 16 rows in 8 bits, 28672 of 8192: 59 us, 4.0 TB/s.
#pragma once
#include "fp8.h"

namespace fise {

enum { FP8_X_CODES = 0, FP8_X_BF16 = 1, FP8_X_F32 = 2 };

#if defined(__HIP_DEVICE_COMPILE__)
// A token's 32 columns of block kb in a lane, pieces lq and lq + 4 of sixteen, from values.  `row` is the row's offset in bytes, not below the buffer's size for rows that are not there.
template <int X> __device__ __forceinline__ void fp8_few_rows(__amdgpu_buffer_rsrc_t from, unsigned row, int kb, int lq, int K, Fp8Operand<true>& to, float& scale) {
    constexpr int OOB = 0x7ffffff0;
    i32x4_t code[2];
    {
        float v[2][16];
        unsigned top = 0;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int col = kb * FP8_BLOCK + lq * 16 + p * 64;
            if constexpr (X == FP8_X_BF16) {
                const int at = col < K ? (int)(row + (unsigned)col * 2u) : OOB;
                const u32x4_t a = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from, at, 0, 0)), b = __builtin_bit_cast(u32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from, at, 16, 0));
#pragma unroll
                for (int i = 0; i < 4; ++i) { v[p][2 * i] = lo16(a[i]); v[p][2 * i + 1] = hi16(a[i]); v[p][8 + 2 * i] = lo16(b[i]); v[p][9 + 2 * i] = hi16(b[i]); }
            } else {
                const int at = col < K ? (int)(row + (unsigned)col * 4u) : OOB;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x4_t a = __builtin_bit_cast(f32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from, at, 16 * j, 0));
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[p][4 * j + i] = a[i];
                }
            }
            top = max(top, fp8_largest<16>(v[p]));
        }
        top = max(top, (unsigned)__shfl_xor((int)top, 16));
        top = max(top, (unsigned)__shfl_xor((int)top, 32));
        const int e = fp8_exponent(top);
        const float inv = fp8_inverse(e);
        scale = fp8_power(e);
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) code[p][i] = (int)fp8_codes(v[p][4 * i], v[p][4 * i + 1], v[p][4 * i + 2], v[p][4 * i + 3], inv);
    }
    to.of(code[0], code[1]);
}
// Sixteen rows of weights and their scale: a lane's pieces of block kb.
struct Fp8FewWeights {
    i32x4_t lo, hi; float scale;
    __device__ __forceinline__ void ld(__amdgpu_buffer_rsrc_t from, unsigned row, const float* scales, int kb, int lq, int K) {
        constexpr int OOB = 0x7ffffff0;
        const int col = kb * FP8_BLOCK + lq * 16;
        lo = __builtin_bit_cast(i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from, col < K ? (int)(row + (unsigned)col) : OOB, 0, 0));
        hi = __builtin_bit_cast(i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from, col + 64 < K ? (int)(row + (unsigned)col + 64u) : OOB, 0, 0));
        scale = scales[kb];
    }
};
// The same of rows that are codes, with their scale.
struct Fp8FewCodes {
    i32x4_t lo, hi; float scale;
    __device__ __forceinline__ void ld(__amdgpu_buffer_rsrc_t from, unsigned row, const float* scales, long long at, bool there, int kb, int lq, int K) {
        constexpr int OOB = 0x7ffffff0;
        const int col = kb * FP8_BLOCK + lq * 16;
        lo = __builtin_bit_cast(i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from, col < K ? (int)(row + (unsigned)col) : OOB, 0, 0));
        hi = __builtin_bit_cast(i32x4_t, __builtin_amdgcn_raw_buffer_load_b128(from, col + 64 < K ? (int)(row + (unsigned)col + 64u) : OOB, 0, 0));
        scale = there ? scales[at] : 0.f;
    }
};
// where result (output n of sixteen, row m of a piece) is among the values of a piece, lane by lane, sixteen lanes 16 bytes off the banks' round
__device__ __forceinline__ int fp8_few_at(int n, int m) { return ((n >> 2) * 17 + m) * 4 + (n & 3); }
#endif

// A few tokens and their experts.
struct ExpertsFewArgs {
    const void* x; long long x_stride; unsigned x_bytes;               // [T, K]
    const int* ids; const float* weights;
    int T, k, E, K, I, N;
    const unsigned char* w_in; const float* w_in_scale; const unsigned char* w_out; const float* w_out_scale;
    float* h; unsigned h_bytes;                                        // [T k, I]
    const void* residual; long long residual_stride; void* y; long long y_stride; int y_f32;
};

constexpr int FP8_FEW_PIECE = 4 * 17 * 4;            // values of a piece in LDS
constexpr unsigned FP8_FEW_NO_ROW = 0x40000000u;   // behind every buffer of these kernels

}  // namespace fise
