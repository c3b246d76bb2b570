// Putting rows in 8 bits: what fp8.hip and experts.hip share.  Internal.
#pragma once
#include "fp8_tile.h"

namespace fise {

// Unit `id` of a row-major line of units of 8 columns, `units` (a multiple of 16) a row: sixteen lanes have a block of 128 columns.  Columns from K on are zeros, written up to
// `written` columns of a row.
template <typename T>
__device__ __forceinline__ void fp8_quantize_unit(const T* x, long long x_stride, int M, int K, int units, int written, unsigned char* codes, long long code_stride,
                                                  float* scale, long long scale_stride, long long id) {
    const long long row = id / units;
    const int col = (int)(id - row * units) * 8;
    float v[8];
    const bool in = row < M && col < K;
    if (in) fp8_load8(x + row * x_stride + col, v);
    else
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    const unsigned top = fp8_over<16>(fp8_largest<8>(v));
    if (row >= M) return;
    const int e = fp8_exponent(top);
    const float inv = fp8_inverse(e);
    if (col < written) *reinterpret_cast<u32x2_t*>(codes + row * code_stride + col) = u32x2_t{fp8_codes(v[0], v[1], v[2], v[3], inv), fp8_codes(v[4], v[5], v[6], v[7], inv)};
    if ((threadIdx.x & 15) == 0) scale[(col / FP8_BLOCK) * scale_stride + row] = fp8_power(e);
}

}  // namespace fise
