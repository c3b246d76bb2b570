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
// numbers, which is exact); a workgroup takes up to 64 of those (a `slab`): mt tiles of 16.
// Resident form: the workgroup's waves_k waves split the columns, kt tile columns each (x of those stays in registers, 64 of them at most, so kt * mt is at
// most 4), in `chunks` rounds where that does not cover all; every wave goes through the workgroup's tiles_n tiles of outputs, and what the waves have of
// an output meets in LDS.
// Staged form: more than 16 rows and several rounds, where the resident form would read x again for every few outputs (64 rows of 8192, 8192 outputs: 35 us, resident 63; 33 rows of 1280, 5120 outputs 8.2, 11.8): eight waves, of which waves_k share a tile of outputs, read x from
// LDS, four tile columns at a time.
struct W4Choice { int staged, pieces, slab, slabs, mt, kt, waves_k, chunks, tiles_n, groups_n, x_at, lds; };
constexpr int W4_LDS = 152 * 1024;
constexpr int W4_STAGE_COLS = 4 * W4_COLS, W4_STAGE_PITCH = W4_STAGE_COLS + 8, W4_STAGE_WAVES = 8;
inline W4Choice w4_choose(int M, int N, int K, bool split) {
    W4Choice c;
    c.pieces = split ? 3 : 1;
    const W4Layout l = w4_layout(N, K, 128);
    const int tk = (int)l.tiles_k;
    // slabs of the fewest row tiles that still leave at most one workgroup for every CU: fewer rows are less x to read for every one of them (27 rows, 1283 outputs, 5120
    // columns: two of 16 rows 8.4 us, one of 27 11.7); else, and with many outputs, as many rows as fit, so that weights are read once
    for (c.mt = 1;; c.mt *= 2) {
        c.slab = std::min(M, 16 * c.mt / c.pieces);
        c.slabs = (M + c.slab - 1) / c.slab;
        if (c.mt == 4 || c.slabs == 1 || l.tiles_n * c.slabs <= 256) break;
    }
    const int kt_max = 4 / c.mt, most = c.mt == 4 ? 8 : 16;                      // tile columns and waves
    c.kt = 1;
    while (c.kt < kt_max && (tk + c.kt - 1) / c.kt > most) c.kt *= 2;
    const int units = (tk + c.kt - 1) / c.kt;
    c.chunks = (units + most - 1) / most;
    c.waves_k = (units + c.chunks - 1) / c.chunks;
    c.x_at = 0;
    c.staged = c.mt > 1 && c.chunks > 1 && l.tiles_n * c.slabs > 256;
    if (c.staged) {
        c.waves_k = 4;
        while (c.waves_k > 1 && l.tiles_n * c.slabs * c.waves_k / W4_STAGE_WAVES > 256 * (c.mt == 2 ? 2 : 1)) c.waves_k /= 2;      // (that many are on the CUs at once)
        c.tiles_n = W4_STAGE_WAVES / c.waves_k;
        c.groups_n = (int)((l.tiles_n + c.tiles_n - 1) / c.tiles_n);
        c.chunks = (tk + 3) / 4;
        c.lds = 2 * c.mt * 16 * W4_STAGE_PITCH * 2;
        return c;
    }
    // as many workgroups as the CUs hold at once, but no more outputs a workgroup than LDS holds the parts of
    const long long at_once = 256 * (16 / c.waves_k);
    const int x_bytes = split ? 16 * (c.waves_k * W4_COLS + 8) * 2 : 0;          // x of a tile column of every wave, 16 rows at a time, on its way to registers
    const long long room = (W4_LDS - (c.chunks > 1 ? x_bytes : 0)) / (1024 * c.mt * c.waves_k);
    c.tiles_n = (int)std::max(1ll, std::min(room, (l.tiles_n * c.slabs + at_once - 1) / at_once));
    c.groups_n = (int)((l.tiles_n + c.tiles_n - 1) / c.tiles_n);
    const int parts = c.tiles_n * c.waves_k * c.mt * 1024;
    c.x_at = c.chunks > 1 ? parts : 0;                                           // one round: before there are parts
    c.lds = std::max(parts, c.x_at + x_bytes);
    return c;
}

}  // namespace fise
