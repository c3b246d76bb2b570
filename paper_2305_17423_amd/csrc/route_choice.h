// Launches of the routing of tokens to experts: lanes of a token, values of a lane, tokens of a workgroup, where the parts of the workspace begin.
// Plain C++: the CPU tests compile it too.
#pragma once
#include <cstdint>

namespace fise {

constexpr int ROUTE_MAX_EXPERTS = 1024, ROUTE_MAX_K = 64;
constexpr int ROUTE_SINGLE_TOKENS = 256, ROUTE_SINGLE_PAIRS = 4096;    // what one workgroup takes in one launch
constexpr int ROUTE_WAVES = 4, ROUTE_SINGLE_WAVES = 16;

struct RouteChoice {
    int lanes, values;          // of a token: lanes * values >= E, k and groups at most lanes
    int single;                 // one workgroup, one launch
    int waves;                  // of a workgroup
    int wave_tokens;            // of a wave, one after the other where they are more than 64 / lanes
    int chunks;                 // workgroups
    int64_t hist_off, total_off, bytes;                                // workspace: pairs, then chunks of each expert, then the experts' totals
};

inline RouteChoice route_choose(int64_t T, int E, int k, int groups, bool lists) {
    RouteChoice c{};
    if (E <= 64 && k <= 16 && groups <= 16) { c.lanes = 16; c.values = 4; }
    else if (E <= 256 && k <= 16 && groups <= 16) { c.lanes = 16; c.values = 16; }
    else { c.lanes = 64; c.values = 16; }
    const int at_once = 64 / c.lanes;
    c.single = T <= ROUTE_SINGLE_TOKENS && T * k <= ROUTE_SINGLE_PAIRS;
    c.waves = c.single ? ROUTE_SINGLE_WAVES : ROUTE_WAVES;
    if (c.single) {
        const int64_t rounds = (T + c.waves * at_once - 1) / (c.waves * at_once);
        c.wave_tokens = (int)(rounds > 0 ? rounds : 1) * at_once;
    } else c.wave_tokens = 12;      // (65536 tokens of 256 experts: 87 us, 91 with 16, 89 with 8)
    c.chunks = (int)((T + c.waves * c.wave_tokens - 1) / (c.waves * c.wave_tokens));
    if (lists && !c.single) {
        c.hist_off = (T * k * 4 + 255) / 256 * 256;
        c.total_off = c.hist_off + ((int64_t)E * c.chunks * 4 + 255) / 256 * 256;
        c.bytes = c.total_off + (E * 4 + 255) / 256 * 256;
    }
    return c;
}

}  // namespace fise
