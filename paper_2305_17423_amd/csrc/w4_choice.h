// How a product of few rows with 4-bit weights is laid over workgroups: plain C++, so that a host program can ask for the form of any size.  Internal.
#pragma once
#include <algorithm>

namespace fise {

// ---- packed weights: tiles of 16 rows (outputs) x 128 columns, 1 KB each: 16 bytes for every lane of a wave, lane = quarter * 16 + row.
// Word j of a lane holds columns 32 j + 8 quarter + (0..7) of the tile, the first in the lowest four bits: the operand of the j-th matrix
// instruction of the tile.  Behind the tiles, 256-byte aligned, the scales as bf16: [tile row][tile column][16 rows][128 / group] where a group is
// narrower than a tile, else [tile row][group][16 rows].
constexpr int W4_ROWS = 16, W4_COLS = 128, W4_TILE_BYTES = W4_ROWS * W4_COLS / 2;
inline bool w4_group_ok(int g) { return g >= 32 && g <= 256 && (g & (g - 1)) == 0; }
struct W4Layout { long long tiles_n, tiles_k, groups, scale_off, bytes; };
inline W4Layout w4_layout(int N, int K, int group) {
    W4Layout l;
    l.tiles_n = ((long long)N + W4_ROWS - 1) / W4_ROWS; l.tiles_k = ((long long)K + W4_COLS - 1) / W4_COLS;
    l.groups = ((long long)K + group - 1) / group;
    l.scale_off = l.tiles_n * l.tiles_k * W4_TILE_BYTES;                          // (a multiple of 1024)
    const long long per_row = group < W4_COLS ? l.tiles_k * (W4_COLS / group) : l.groups;
    l.bytes = l.scale_off + (l.tiles_n * per_row * W4_ROWS * 2 + 255) / 256 * 256;
    return l;
}

// ---- the launch.  A row of x is one row of the matrix instruction, or three where x is float or goes through SiLU (its value as the sum of three bf16
// numbers, which is exact); a workgroup takes up to 64 of those (one `slab`) and waves_n tiles of 16 outputs, each of them by waves_k waves that share its
// columns.  x passes through LDS in chunks of `chunk` tile columns.
struct W4Choice { int pieces, slab, slabs, mt, waves_n, waves_k, chunk, pitch, lds; };
constexpr int W4_LDS = 152 * 1024;
inline W4Choice w4_choose(int M, int N, int K, bool split) {
    W4Choice c;
    c.pieces = split ? 3 : 1;
    c.slab = std::min(M, 64 / c.pieces); c.slabs = (M + c.slab - 1) / c.slab;
    const int rows = c.slab * c.pieces;
    c.mt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const W4Layout l = w4_layout(N, K, 128);
    const int tk = (int)l.tiles_k;
    const long long tiles = l.tiles_n * c.slabs;
    c.waves_k = tiles < 512 ? 16 : tiles < 1024 ? 8 : 4;
    while (c.waves_k > 1 && c.waves_k / 2 >= tk) c.waves_k /= 2;
    c.waves_n = std::max(1, 8 / c.waves_k);
    const int waves = c.waves_n * c.waves_k;
    const int room = (waves > 8 ? W4_LDS : W4_LDS / 2);
    c.chunk = std::min<long long>(tk, (room / (2 * rows) - 8) / W4_COLS);
    c.pitch = c.chunk * W4_COLS + 8;
    c.lds = std::max(rows * c.pitch * 2, waves * c.mt * 1024);
    return c;
}

}  // namespace fise
