// Host-side geometry of the operators of a decoding tenant that both their launchers and the executor need.
#pragma once
#include <stddef.h>
#include <algorithm>
#include "kernels.h"

namespace gacer {

// Attention over a cache, by the unsplit operator's shape (so that every decomposition adds in the same order): rows of a key/value head in
// tiles of `rows`, keys in `splits` parts of at least `split_min` tiles of 64 that a second kernel joins.  Measured, us (32 / 8 heads of 128
// features, bf16 unless said otherwise; lengths up to the stated ones):
//   rows    8 and not 16: one token of 16 sequences of 4096 keys 23 against 32, of one of 32768 19 against 25; 16 and not 32: four tokens of
//           them 33 against 45, 25 against 33.  32 and not 128: 24 rows (6 tokens), 32 sequences of 1024 keys 28 against 32, one of 32768 33
//           against 36, though 4 of 4096 31 against 23; 40 rows the other way, 48 against 37 and 45 against 42.  fp32 has three times
//           the matrix instructions, and a wave's share of them counts: 40 rows 81 against 88, but 80 rows 109 against 91.
//   waves   8 of a row tile of 8 share the keys of a tile and hide each other's loads; of 4: 64 sequences of 8192 keys 105 against 84, one of
//           131072 60 against 41.  With 16 rows or in fp32 the registers of 8 do not fit.
//   splits  workgroups as many as the units hold at a time of a kernel with few rows (twice: one sequence of 131072 keys 49 against 41, four
//           times 64), or with 128 (bf16 3 of 64 features, 2 of 128, fp32 2 and 1: 64 tokens of fp32 after 4 x 4096 keys 96 against 108
//           with two), each with 1024 keys or 256 at least.
// per_cu: workgroups that a unit holds, by the registers of their waves (4 waves: one workgroup of up to 512, two of 256, three of 168) and LDS.  8 waves of
// 155 to 251 registers are one workgroup; of the kernels of 4 waves and up to 32 rows those of 64 features and up to 16 rows stay within 256, the others have 317 to 512.
struct AttendGeom { int rows, waves, row_tiles, splits, split_min, per_cu; };
inline AttendGeom attend_geom(const TokenArgs &a)
{
    AttendGeom g;
    const int64_t all = (int64_t)a.S * (a.heads / a.kv_heads);
    g.rows = all <= 8 ? 8 : all <= 16 ? 16 : all <= (a.dtype == DT_BF16 ? 32 : 64) ? 32 : 128;
    g.waves = g.rows == 8 && a.dtype == DT_BF16 ? 8 : 4;
    g.row_tiles = (int)((all + g.rows - 1) / g.rows);
    const int64_t groups = (int64_t)a.batch * a.kv_heads * g.row_tiles;
    const int64_t most = std::min((int64_t)a.cache.max_pages << a.cache.page_shift, a.window > 0 ? (int64_t)a.window + a.S : (int64_t)1 << 40);
    const bool wide = g.rows == 128;
    g.per_cu = wide ? (a.D == 64 ? 2 : 1) + (a.dtype == DT_BF16 ? 1 : 0) : g.waves == 4 && a.D == 64 && g.rows <= 16 ? 2 : 1;
    const int want = 256 * (wide ? g.per_cu : 1), least = wide ? 256 : 1024;      // workgroups, keys of a split
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
