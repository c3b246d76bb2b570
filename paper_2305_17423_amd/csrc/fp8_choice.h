// Products in 8-bit floating point: which tile a call takes and what its workspace holds.  Plain C++: the CPU tests compile it too.
#pragma once
#include <algorithm>
#include <cstdint>

namespace fise {

enum { FP8_FORM_256 = 0, FP8_FORM_128 = 1, FP8_FORM_32 = 2, FP8_FORM_FEW = 3, FP8_FORM_64 = 4 };      // 256 x 256, 128 x 128, 32 tokens x 128 outputs; weights streamed past up to 64 rows

struct Fp8Choice {
    int form, bm, bn; int64_t m_tiles, n_tiles;
    int waves;                  // FEW: of a workgroup
    bool make_rows;             // x is put in 8 bits by a launch in front
};

// exact: products in bf16 (float results), whose operands leave no room for the largest tile
inline Fp8Choice fp8_choose(int64_t M, int64_t N, int64_t K, bool exact, bool codes) {
    Fp8Choice c{};
    auto set = [&](int form, int bm, int bn) { c.form = form; c.bm = bm; c.bn = bn; c.m_tiles = (M + bm - 1) / bm; c.n_tiles = (N + bn - 1) / bn; };
    c.make_rows = !codes && M > 0;
    // Few rows: streaming the weights past them is bound by the trips; more rows for many outputs read rows and turn codes into bf16 too often for that.  us, streamed and tiles:
    // 64 rows 4096 x 4096: 13.3 and 23.6, 8192 x 8192: 42 and 43.5, 10240 x 1280: 15.2 and 10.0, 28672 x 8192: 144 and 70; 32 rows 8192 x 8192: 27 and 38, 10240 x 1280: 9.9 and 8.6,
    // 28672 x 8192: 96 and 65; 16 rows 28672 x 8192: 59 and 63
    if (M <= 16 || (M <= 64 && N <= 8192)) {
        set(FP8_FORM_FEW, 64, 16);
        const int64_t blocks = (K + 127) / 128;
        c.waves = (int)std::min<int64_t>(16, blocks);
        // Each workgroup puts the rows in 8 bits for itself where that is one piece of sixteen rows a wave (16 rows, 1280 columns: 5.3 us, one launch); more is made once (54 rows of 5136
        // columns for 1283 outputs: 30 and 14.5 us)
        c.make_rows = !codes && M > 0 && !(M <= 16 && blocks <= 16);
        return c;
    }
    set(FP8_FORM_256, 256, 256);
    if (M <= 32) { set(FP8_FORM_32, 32, 128); return c; }
    if (M <= 64) { set(FP8_FORM_64, 64, 128); return c; }
    if (exact || c.m_tiles * c.n_tiles < 200) set(FP8_FORM_128, 128, 128);
    return c;
}

// rows that the call puts in 8 bits: codes of whole blocks, then the scales of each block
struct Fp8Space { int64_t stride, scale_off, bytes; };
inline Fp8Space fp8_space(int64_t M, int64_t K) {
    Fp8Space s{};
    const int64_t blocks = (K + 127) / 128;
    s.stride = blocks * 128;
    s.scale_off = (M * s.stride + 255) / 256 * 256;
    s.bytes = s.scale_off + (M * blocks * 4 + 255) / 256 * 256;
    return s;
}

// The experts' feed-forward: its form, tokens of a tile, an upper bound of the tiles, and the workspace.
// TOKENS: a workgroup has a pair, then a token's sum.  TILES: rows in 8 bits, tiles of an expert's rows through LDS.
enum { EXPERTS_TOKENS = 0, EXPERTS_TILES = 1 };
struct ExpertChoice {
    int form, bm, bm_in; int64_t m_tiles, m_tiles_in;                  // TILES: of the second product, of gate and up
    int waves_in, waves_out;    // of a workgroup (TOKENS)
    int64_t x_stride, x_scale_off, h_off, h_stride, h_scale_off, out_off, row_exp_off, table_off, place_off, table_in_off, bytes;
};
inline ExpertChoice expert_choose(int64_t T, int64_t K, int64_t I, int64_t N, int64_t E, int64_t k, int64_t x_row_bytes, int y_bytes) {
    ExpertChoice c{};
    const int64_t P = T * k, blocks_k = (K + 127) / 128, blocks_i = (I + 127) / 128;
    auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
    // Two launches instead of four, but each pair reads its expert's weights and each workgroup puts its token in 8 bits, a block of columns for sixteen channels at a time.  us, TOKENS and TILES:
    // one token, 2 of 16, 1280 x 640: 10.4 and 23.5; 8 of 128, 2048 x 768: 24 and 33; 8 of 64, 4096 x 1536: 51 and 53; four, 6 of 64, 2048 x 1408: 78 and 61
    const bool fits = T * x_row_bytes < (1 << 30) && P * I * 4 < (1 << 30);      // offsets of these kernels
    if (fits && T <= 4 && P * blocks_k * ((I + 15) / 16) <= 24576) {
        c.form = EXPERTS_TOKENS;
        c.waves_in = (int)std::min<int64_t>(16, blocks_k);
        c.waves_out = (int)std::min<int64_t>(16, blocks_i * k);
        c.bytes = up(P * I * 4);
        return c;
    }
    c.form = EXPERTS_TILES;
    // Gate and up have exact sums (fp8_tile.h) in every form, on 128 rows at most: what the 8-bit instruction drops of them moves codes of h that are next to a border, one in a thousand
    // (131072 pairs, 4096 x 1536: 1.75 ms instead of 3.3, but the result's error without residual 2.6e-3 instead of 1.7e-3, its rounding).  For the second product, behind which nothing is put in
    // 8 bits, bf16 results of many rows take that instruction, on tiles of 256 rows (1.0 ms, with exact sums on 128 rows 1.8); with fewer exact sums cost less (4096 tokens of 4 among 64,
    // 4096 x 1536: the call 864 us and 952).  Float results have exact sums at any size, as those of one product have
    c.bm = P >= 512 * E && y_bytes != 4 ? 256 : P >= 64 * E ? 128 : 32;
    c.bm_in = std::min(c.bm, 128);
    c.m_tiles = P / c.bm + std::min(E, P);
    c.m_tiles_in = P / c.bm_in + std::min(E, P);
    const Fp8Space x = fp8_space(T, K), h = fp8_space(P, I);
    c.x_stride = x.stride; c.x_scale_off = x.scale_off;
    c.h_off = x.bytes; c.h_stride = h.stride; c.h_scale_off = c.h_off + h.scale_off;
    c.out_off = c.h_off + h.bytes;
    c.row_exp_off = c.out_off + up(P * N * y_bytes);
    c.table_off = c.row_exp_off + (y_bytes == 4 ? 0 : up(P * ((N + 31) / 32)));
    c.place_off = c.table_off + up(c.m_tiles * 8);
    c.table_in_off = c.bm_in == c.bm ? c.table_off : c.place_off + up(P * 4);      // (one table where the tiles are the same)
    c.bytes = c.place_off + up(P * 4) + (c.bm_in == c.bm ? 0 : up(c.m_tiles_in * 8));
    return c;
}

}  // namespace fise
