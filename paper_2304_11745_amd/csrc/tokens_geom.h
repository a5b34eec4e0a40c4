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

// Products of 8-bit rows, by the unsplit operator's shape (so that every decomposition adds in the same order): tiles of `features` of the result and
// `rows`, `slices` parts of the inner extent that a second kernel joins.  The choice with the least estimated time is taken: rounds of workgroups over the units,
// times blocks of 128 inner features in a slice, times what a block takes in this tile, and for a join its launch and its way through memory.
// Measured, us, the choice first (bf16; operands of three calls in turn, 75 to 350 MB, of which the last-level cache keeps a part):
//   4096 -> 6144: 1 row few 9.3, 64x32 in two slices 12.1; 32 rows few 12.1, 64x32 12.7; 64 rows 64x32 14.2, 64x64 15.2, in two 13.5; 128 rows 64x64 15.0, 128x128 34;
//   512 rows 128x128 31, 64x64 37, 256x128 50; 1024 rows 256x128 53, 128x128 70.  4096 -> 32000: 1 row 64x32 29, few 37.
//   14336 -> 4096: 1 row few in two 15.6, 64x32 in four 16.3, few whole 19.7; 32 rows 64x32 in four 16.5, few 20.5; 64 rows 64x64 in four 18.3, whole 44; 128 rows
//   128x128 in eight 27.5, 64x64 in two 28.5, whole 44; 512 rows 128x128 in two 69, 64x64 82; 2048 rows 256x128 206, 128x128 253.
//   gated, 4096 -> 14336: 1 row 256x32 in two 26.2, whole 32; 48 rows 256x64 in two 34.2, whole 35, 256x32 32; 128 rows 256x64 41, 256x128 51; 256 rows 256x128 64,
//   256x64 80.
// The constants below stand for these: a round's time less a launch of 4, over its blocks, is 0.32 for 64x32 (64 rows 4096 -> 6144), 0.34 for 64x64 (128), 0.84 for 128x128 (512), 1.53 for
// 256x128 (1024), and gated, 4096 -> 14336, 0.88 for 256x32 (48 rows), 1.16 for 256x64 (128), 1.88 for 256x128 (256); they differ from it by up to 15 %.  The choice is within 7 % of the
// best at the sizes above, and not the best at all of them (64 rows 4096 -> 6144, 48 gated rows).
// Numbers of slices between the powers of two gain nothing (64 rows 4096 -> 6144 14.9 and in three 15.1, gated 128 rows 5120 -> 5120 27.7 and 26.7, 333 rows
// 8192 -> 2048 25.0 and in five 25.5).
enum Fp8Tile { FP8_FEW, FP8_64x32, FP8_64x64, FP8_128x128, FP8_256x128, FP8_256x64, FP8_256x32 };      // rows of weights (a gated block: half gate, half up) x rows
enum { FP8_WS_MAX = 16 << 20 };                                                      // bytes of workspace, of the 32 MiB that all tenants share in gacer_run_static
struct Fp8Geom { Fp8Tile tile; int features, rows, slices, blocks_per_slice; };
// Tiles of a last round that are done in halves of their rows, by twice as many workgroups: where these are one round too.
inline int fp8_halves(int64_t tiles, int slices) { return slices == 1 && tiles > 256 && tiles % 256 <= 128 ? (int)(tiles % 256) : 0; }
inline Fp8Geom fp8_geom(const TokenArgs &a)
{
    const bool gated = a.op == TK_GATED_FP8;
    const int64_t rows = (int64_t)a.batch * a.S, blocks = (a.xq.features + FP8_BLOCK - 1) / FP8_BLOCK, N = a.features;
    struct Shape { Fp8Tile tile; int features, rows; double us; int held; double half; };      // us a block; workgroups that a unit works on at a time; us a block in halves
    static const Shape gemm[] = {{FP8_FEW, 32, 32, 0.0, 1, 0.0}, {FP8_64x32, 64, 32, 0.32, 2, 0.0}, {FP8_64x64, 64, 64, 0.37, 2, 0.0}, {FP8_128x128, 128, 128, 0.95, 1, 0.0}, {FP8_256x128, 256, 128, 1.5, 1, 1.1}};
    static const Shape block[] = {{FP8_256x32, 128, 32, 0.85, 1, 0.0}, {FP8_256x64, 128, 64, 1.05, 1, 0.0}, {FP8_256x128, 128, 128, 1.6, 1, 1.05}};
    Fp8Geom g = {};
    double least = 0.0;
    for (int i = 0; i < (gated ? 3 : 5); ++i) {
        const Shape &s = gated ? block[i] : gemm[i];
        const int64_t tiles = ((N + s.features - 1) / s.features) * ((rows + s.rows - 1) / s.rows);
        if (s.tile == FP8_FEW && rows > 32) continue;
        for (int slices = 1; slices <= 8; slices *= 2) {
            const int64_t per = (blocks + slices - 1) / slices, bytes = slices * rows * N * (gated ? 8 : 4);
            if ((slices > 1 && (per < 8 || bytes > FP8_WS_MAX)) || (s.tile == FP8_FEW && tiles * slices > 256)) break;
            double rounds = (double)(tiles * slices) / 256.0;
            if (s.held == 1) rounds = (double)((tiles * slices + 255) / 256);
            if (rounds < 1.0) rounds = 1.0;
            if (s.half > 0.0 && fp8_halves(tiles, slices)) rounds += s.half / s.us - 1.0;
            // few rows: a round of eight blocks, one a wave, longer by the rows that are read beside the weights
            const double us = s.tile == FP8_FEW ? (rows <= 8 ? 1.05 : rows <= 16 ? 1.45 : 1.85) * (double)((per + 7) / 8) : s.us * (double)per;
            const double all = rounds * us + (slices > 1 ? 3.5 + (double)bytes / 2.5e6 : 0.0);
            if (least == 0.0 || all < least) {
                least = all;
                g = {s.tile, s.features, s.rows, slices, (int)per};
            }
        }
    }
    return g;
}

// Floats of workspace that the unsplit operator needs.
inline size_t token_ws_floats(const TokenArgs &a)
{
    if (a.op == TK_CACHE_ATTENTION) {
        const AttendGeom g = attend_geom(a);
        if (g.splits > 1) return (size_t)a.batch * a.kv_heads * g.row_tiles * g.splits * g.rows * (a.D + 2);
    }
    if (a.op == TK_GEMM_FP8 || a.op == TK_GATED_FP8) {
        const Fp8Geom g = fp8_geom(a);
        if (g.slices > 1) return (size_t)g.slices * a.batch * a.S * a.features * (a.op == TK_GATED_FP8 ? 2 : 1);
    }
    return 0;
}

}  // namespace gacer
