// How attention over a cache of latent vectors is laid out and which form it takes: plain C++, so that a host program can ask for the form of any size.  Internal.
#pragma once
#include <algorithm>
#include <cstddef>

namespace fise {

constexpr int LA_ROWS = 64;           // rows (query, head) of a workgroup of the absorbed form
constexpr int LA_KEYS = 32;           // keys of a block
constexpr int LA_CUS = 256;

struct LatentShape { int B, M, n, heads, d, dr, dv, r; bool causal; };

// Widths the kernels are built for: the latent vector and the shared key are filled up with zeros on their way into LDS.
inline int latent_width(int r) { return r <= 128 ? 128 : r <= 256 ? 256 : r <= 384 ? 384 : 512; }
constexpr int latent_per_cu(int R) { return R <= 128 ? 3 : R <= 256 ? 2 : 1; }      // workgroups whose blocks of keys a CU's LDS holds
inline int latent_shared(int dr) { return dr ? 64 : 0; }

// ---- absorbed form.  Blocks of keys of all (batch element, tile of rows) groups stand in one line, which the workgroups share evenly: workgroup w has
// blocks w T / G .. (w + 1) T / G of T.  A workgroup's part of a group is a partial result in slot w + group, which no other pair has.
inline int absorbed_tiles(const LatentShape& s) { return (int)(((long long)s.M * s.heads + LA_ROWS - 1) / LA_ROWS); }
// As many workgroups as find room on the CUs at once, and two blocks each at least, as a partial result costs as much to write and read as a block of keys; one where its rows
// are few and short, 8 KB.  us, one and two blocks: 1000 keys, 8 rows of 128 (4 KB) 12.6, 13.4; 4096 keys, 16 rows of 512 (32 KB) 25.3, 23.7; 64 rows of 512 34.4, 30.4.  Four
// blocks: 14.5, 24.8, 30.1, but 37 instead of 27 where 128 rows have 300 keys.
inline int absorbed_workgroups(const LatentShape& s) {
    const long long blocks = (long long)s.B * absorbed_tiles(s) * ((s.n + LA_KEYS - 1) / LA_KEYS);
    const long long part = std::min<long long>(LA_ROWS, (long long)s.M * s.heads) * latent_width(s.r) * 4, each = part <= 8192 ? 1 : 2;
    return (int)std::max(1ll, std::min<long long>(latent_per_cu(latent_width(s.r)) * LA_CUS, (blocks + each - 1) / each));
}
struct AbsorbedLayout { size_t table, q, ml, part, total; };
inline AbsorbedLayout absorbed_layout(const LatentShape& s) {
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    const size_t R = latent_width(s.r), groups = (size_t)s.B * absorbed_tiles(s), slots = groups + absorbed_workgroups(s);
    AbsorbedLayout l;
    l.table = 0;
    l.q = l.table + up((groups + 1) * 4);
    l.ml = l.q + up((size_t)s.B * s.M * s.heads * (R + latent_shared(s.dr)) * 2);
    l.part = l.ml + up(slots * LA_ROWS * 8);
    l.total = l.part + up(slots * LA_ROWS * R * 4);
    return l;
}
// Tokens a workgroup of the last launch (merge, then the values' weights) takes: more read W_uv less often, as long as that leaves workgroups enough.  us of the whole call with
// 1, 4, 16: 128 rows 40.6, 47.7, 47.7; 1024 rows 77, 65, 68; 2048 rows 246, 224, 228; 16384 rows 410, 200, 158.
inline int absorbed_tokens(const LatentShape& s) {
    const long long tokens = (long long)s.B * s.M;
    return tokens * s.heads >= 16 * 2 * LA_CUS ? 16 : tokens * s.heads >= 4 * LA_CUS ? 4 : 1;
}

// ---- expanded form.  Keys of a head are rows [W_uk c | k_pe | 0] of 16 KD channels, values are transposed, as everywhere in the library; both for whole tiles of
// LX_KEYS keys.
constexpr int LX_QUERIES = 128, LX_BLOCK = 64, LX_KEYS = 128;
struct ExpandedTile { int KD, DB; };  // 16-channel steps of a key, 32-channel blocks of a value
constexpr ExpandedTile kExpandedTiles[] = {{4, 2}, {6, 2}, {8, 2}, {8, 4}, {12, 2}, {12, 4}, {14, 5}};
inline int expanded_tile(const LatentShape& s) {
    for (int i = 0;; ++i)
        if (16 * kExpandedTiles[i].KD >= s.d + s.dr && 32 * kExpandedTiles[i].DB >= s.dv) return i;      // (the last one holds the largest: 160 + 64, 160)
}
inline int expanded_tiles(const LatentShape& s) { return (s.M + LX_QUERIES - 1) / LX_QUERIES; }
// Tiles of queries (of an element and head) enough for all workgroups that the CUs hold at once (two each; one of the widest heads): one for each tile.  Fewer: the blocks of
// keys stand in one line too, and those workgroups share it evenly, three blocks each at least (192 queries on 1024 keys: with three 33 us, one and six 39); a cut tile costs its parts written and read again.  us, tiles and line:
// 512 causal tiles of 2 - 64 blocks 134, 154; 96 tiles of 64 blocks 80, 53; 32 of 64 blocks 108, 78 (the whole call).
constexpr int expanded_per_cu(int KD) { return KD <= 12 ? 2 : 1; }
inline long long expanded_groups(const LatentShape& s) { return (long long)s.B * s.heads * expanded_tiles(s); }
inline bool expanded_whole(const LatentShape& s) { return expanded_groups(s) >= expanded_per_cu(kExpandedTiles[expanded_tile(s)].KD) * LA_CUS; }
inline int expanded_workgroups(const LatentShape& s) {
    if (expanded_whole(s)) return (int)expanded_groups(s);
    const long long groups = expanded_groups(s), blocks = groups * ((s.n + LX_BLOCK - 1) / LX_BLOCK);
    const long long most = std::max(1ll, std::min<long long>(expanded_per_cu(kExpandedTiles[expanded_tile(s)].KD) * LA_CUS, (blocks + 2) / 3));
    // a whole number for each tile, if that leaves at most an eighth of them out: tiles of the same length then begin where a workgroup does
    // (96 tiles of 64 blocks on 480 workgroups 54 us, on 512 57; of 16 blocks 41, 48)
    return (int)(groups <= most && most / groups * groups * 8 >= most * 7 ? most / groups * groups : most);
}
inline long long latent_value_tiles(const LatentShape& s) { return ((long long)s.heads * s.dv + 127) / 128; }
// The line has of a head's tiles in turn the last and the first that are left, which together have as many keys as any other two where rows are causal: place i, and the place of a tile.
constexpr int expanded_line_tile(int i, int tiles) { return i & 1 ? i >> 1 : tiles - 1 - (i >> 1); }
constexpr int expanded_line_place(int tile, int tiles) { return tile >= tiles >> 1 ? 2 * (tiles - 1 - tile) : 2 * tile + 1; }
// A workgroup for every tile: which one workgroup w has, of `heads` heads (of all elements) with `tiles` tiles of queries each.  Consecutive workgroups go to the eight XCDs in turn;
// each XCD has whole heads where their number allows, and takes their tiles with most keys (causal rows: the last ones) first.  Where a CU holds two workgroups, the
// second ones of all CUs go the other way round, so that the two of a CU have about as many keys as any other two; what follows fills the room that comes free.  us, the other
// way round and not: 16 heads of 32 causal tiles 165, 170; of 33 170, 174; of 64 480, 500; 40 heads of 16 126, 125; 64 of 8 (d 40) 41, 41.
struct ExpandedPlace { int head, tile; };
constexpr ExpandedPlace expanded_place(int w, int heads, int tiles, int per_cu) {
    const bool split = heads % 8 == 0;
    const int here = split ? heads / 8 : heads, cus = split ? LA_CUS / 8 : LA_CUS, at = split ? w >> 3 : w;
    const int i = per_cu == 2 && at >= cus && at < 2 * cus ? 3 * cus - 1 - at : at, rank = i / here;
    return {(split ? (w & 7) * here : 0) + i - rank * here, tiles - 1 - rank};
}
struct ExpandedLayout { long long n_pad; size_t table, k, v, flags, ml, part, total; };
inline ExpandedLayout expanded_layout(const LatentShape& s) {
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    const ExpandedTile t = kExpandedTiles[expanded_tile(s)];
    const size_t groups = (size_t)expanded_groups(s), slots = expanded_whole(s) ? 0 : groups + expanded_workgroups(s);
    ExpandedLayout l;
    l.n_pad = ((long long)s.n + LX_KEYS - 1) / LX_KEYS * LX_KEYS;
    l.table = 0;
    l.k = l.table + up((groups + 1) * 4);
    l.v = l.k + up((size_t)s.B * s.heads * l.n_pad * t.KD * 32);
    l.flags = l.v + up((size_t)s.B * s.heads * s.dv * l.n_pad * 2);
    l.ml = l.flags + up((size_t)s.B * latent_value_tiles(s) * (l.n_pad / LX_KEYS) * 4);
    l.part = l.ml + up(slots * LX_QUERIES * 8);
    l.total = l.part + up(slots * LX_QUERIES * t.DB * 128);
    return l;
}

// ---- which form: the one with fewer operations (sums counted once; launches and joining are left out, so that near the border the other one can be a few percent faster).  us,
// absorbed and expanded, 4096 keys, 2 elements: 16 heads of 128 + 64, r 512: 64 queries 62, 80; 256 queries 135, 97; 4096 causal queries of one element 1102, 157.  8 heads of 40 + 32,
// r 128: 16 queries 20, 31; 64 queries 33, 33 - 35 (the rule takes the latter); 192 40, 39; 768 88, 54.
inline bool latent_expands(const LatentShape& s) {
    const double keys = (double)s.n, pairs = (double)s.M * s.heads * (s.causal && s.M > 1 ? keys - 0.5 * std::min<double>(s.M, keys) : keys);
    const double absorbed = pairs * (2.0 * latent_width(s.r) + latent_shared(s.dr)) + (double)s.M * s.heads * s.r * (s.d + s.dv);
    const ExpandedTile t = kExpandedTiles[expanded_tile(s)];
    const double expanded = pairs * (16 * t.KD + 32 * t.DB) + keys * s.heads * s.r * (s.d + s.dv);
    return expanded < absorbed;
}

}  // namespace fise
