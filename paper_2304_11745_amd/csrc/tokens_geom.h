// Host-side geometry of the operators of a decoding tenant that both their launchers and the executor need.
#pragma once
#include <stddef.h>
#include <algorithm>
#include "kernels.h"

namespace gacer {

// Attention over a cache, by the unsplit operator's shape (so that every decomposition adds in the same order): rows of a key/value head in
// tiles of `rows`, keys in `splits` parts of at least `split_min` tiles of 64 that a second kernel joins.
struct AttendGeom { int rows, waves, row_tiles, splits, split_min; };
inline AttendGeom attend_geom(const TokenArgs &a)
{
    AttendGeom g;
    const int64_t all = (int64_t)a.S * (a.heads / a.kv_heads);
    g.rows = all <= 8 ? 8 : all <= 16 ? 16 : all < 128 ? 32 : 128;
    g.waves = g.rows == 8 && a.dtype == DT_BF16 ? 8 : 4;
    g.row_tiles = (int)((all + g.rows - 1) / g.rows);
    const int64_t groups = (int64_t)a.batch * a.kv_heads * g.row_tiles;
    const int64_t most = std::min((int64_t)a.cache.max_pages << a.cache.page_shift, a.window > 0 ? (int64_t)a.window + a.S : (int64_t)1 << 40);
    const bool wide = g.rows == 128;
    const int want = wide ? 512 : 256, least = wide ? 256 : 1024;      // workgroups, keys of a split
    g.split_min = wide ? 4 : 8;
    g.splits = (int)std::min<int64_t>(std::min((want + groups - 1) / groups, std::max<int64_t>(1, most / least)), 128);
    return g;
}

// Floats of workspace that the unsplit operator needs.
inline size_t token_ws_floats(const TokenArgs &a)
{
    if (a.op == TK_CACHE_ATTENTION) {
        const AttendGeom g = attend_geom(a);
        if (g.splits > 1) return (size_t)a.batch * a.kv_heads * g.row_tiles * g.splits * g.rows * (a.D + 2);
    }
    return 0;
}

}  // namespace gacer
