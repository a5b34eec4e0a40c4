// Attention of new tokens over a paged 4-bit cache, on the matrix cores.
//
// The queries of one key/value head (heads/kv_heads heads x S tokens) are the rows of its products.  A wave takes 64 keys at a time: scores =
// rows x keys, lane = key, so that the scales of a key stand in the lane that scores it and each register is one row; the values' product
// has the same rows, lane = feature.  Codes enter the products as whole numbers k = c - BIAS (times a power of two), exact in bf16, and
// the scales are applied to the scores and to the softmax weights in fp32:
//   q.k_j = sum over groups g of  s_jg * (sum_d q_d k_jd) + (m_jg + BIAS s_jg) * sum_d q_d
//   out_d = sum_j (p_j s_jg) k_jd + sum_j p_j (m_jg + BIAS s_jg)
// so neither keys nor values are ever rounded.  In bf16 tenants k = 16 + c, which is a shift and a mask per pair of codes; fp32 tenants pay more
// instructions for k = c - 8, because sums of numbers that do not lie around zero lose what their differences need (attention over 1000 keys: relative
// error 6.8e-6 with 16 + c).  Operands that are not whole numbers are split into bf16 parts: queries of fp32 tenants into
// three, weights p_j s_jg into two (bf16 tenants: an error of at most 2^-15 against 2^-8 of the result's own rounding; one part would add as much as
// that) or three.  Where rows leave room in the products' 32, the parts are rows of one product.  Weights pass through a patch of LDS, from
// lane = key to the layout of an operand.
//
// The softmax keeps a reference per row that only moves when a score passes it by more than 2^8: weights are 2^(score - reference), sums are per
// lane and joined at the end.  Waves of a workgroup take parts of its keys and are joined in LDS; where there are too few workgroups
// the keys are also cut into splits, joined by a second kernel.
//
// Up to 8 rows the way from memory bounds it, and the 251 registers of a wave (two tiles of codes among them) that leave room for one workgroup in a
// unit: 64 sequences of up to 8192 keys, 8 kv heads of 128 features (one token, bf16, 308 MB of cache) 84 us = 3.7 TB/s, of which the loads alone take
// 65; one of 131072 keys (151 MB) 41 us = 3.7 TB/s, 5 of them the join.  With more rows the instructions that turn codes into operands
// and scores into weights bound it, and from 33 on (65 in fp32) the kernel for 128 rows takes over.
#include <hip/hip_runtime.h>
#include <limits.h>
#include <algorithm>
#include "cache_attention.h"
#include "tokens_geom.h"

namespace gacer {

// Two blocks of 32 keys and values as loaded: lane & 31 = key of its block (keys, scales) or feature (values), lane >> 5 = half of the group's
// features (keys) or of the block's keys (values)
template <int D> struct Tile {
    uint4 k[2][D / 64];
    uint2 v[2][D / 32];
    unsigned ks[2][D / 64], vs[2][D / 64];
    int page[2];
};

// sum over the 32 lanes of a half
template <int CTRL> __device__ __forceinline__ float add_lanes(float v) { return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true)); }
__device__ __forceinline__ float sum32(float v)
{
    v = add_lanes<0xB1>(v);                            // quad_perm 1,0,3,2
    v = add_lanes<0x4E>(v);                            // quad_perm 2,3,0,1
    v = add_lanes<0x141>(v);                           // mirrored within 8 lanes
    v = add_lanes<0x140>(v);                           // mirrored within 16
    return v + __shfl_xor(v, 16, 64);
}

template <typename T, int D, int ROWS, int NW> __global__ __launch_bounds__(NW * 64) void cache_attention_kernel(AttendArgs a)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int NG = D / 64, R4 = ROWS / 2, QP = F32 ? 3 : 1, PP = F32 ? 3 : 2, PROW = 128 + 16;    // bytes of a row of weights
    constexpr int STACK = 32 / ROWS < PP ? 32 / ROWS : PP, PM = (PP + STACK - 1) / STACK;              // parts in one product, products
    constexpr int QSTACK = 32 / ROWS < QP ? 32 / ROWS : QP, QM = (QP + QSTACK - 1) / QSTACK;
    constexpr float TIMES = F32 ? 16.f : 1.f, BIAS = F32 ? 8.f : -16.f;
    constexpr int PGROUP = PP * ROWS * PROW, PWAVE = NG * PGROUP;
    constexpr int JOIN = NW * ROWS * D * 4, BYTES = NW * PWAVE > JOIN ? NW * PWAVE : JOIN;
    __shared__ __align__(16) unsigned char lds[BYTES];
    __shared__ float2 ends[NW * ROWS];
    __shared__ float factor[NW * ROWS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    const int u = div_by((int)blockIdx.x, a.div_splits), sp = (int)blockIdx.x - u * a.splits, z = div_by(u, a.div_tiles), rt = u - z * a.row_tiles;
    const int zb = div_by(z, a.div_kv), g = z - zb * a.c.kv_heads, b = a.b_lo + zb;
    const int rows = a.S * a.per_kv, r0 = rt * ROWS;
    const Span span = span_of(a.c, b, a.S);
    const Range rg = range_of(a, span, r0, min(r0 + ROWS, rows));
    int lo = rg.lo, hi = rg.hi;
    if (a.splits > 1) {
        const int n = split_tiles(a, rg.hi - rg.lo);
        lo = rg.lo + sp * n;
        hi = min(rg.hi, lo + n);
        if (lo >= hi) return;
    }
    const int per = (hi - lo + NW - 1) / NW, w_lo = lo + wave * per, w_hi = min(hi, w_lo + per);

    const unsigned k_at = l32 * (D / 2) + half * 16, s_at = l32 * NG * 4, v_at = l32 * 16 + half * 8;
    int pages = -1, pages_at = INT_MIN / 2;            // lane i: page of block pages_at + i
    auto load = [&](int tile, Tile<D> &x) {
        const int blk = tile * 2;
        if (blk - pages_at >= 64 || blk < pages_at) {
            pages_at = blk;
            pages = page_of(a.c, b, min(blk + lane, 1 << 25) << 5);
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            x.page[m] = __builtin_amdgcn_readlane(pages, blk - pages_at + m);
            const int64_t row = page_row(a.c, max(x.page[m], 0), g) + (((blk + m) << 5) & ((1 << a.c.page_shift) - 1));
            const unsigned char *k = a.c.k_codes + row * (D / 2), *v = a.c.v_codes + row * (D / 2);
            const unsigned char *ks = (const unsigned char *)(a.c.k_scales + row * NG), *vs = (const unsigned char *)(a.c.v_scales + row * NG);
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                x.k[m][i] = *(const uint4 *)(k + k_at + i * 32);
                x.ks[m][i] = *(const unsigned *)(ks + s_at + i * 4);
                x.vs[m][i] = *(const unsigned *)(vs + s_at + i * 4);
            }
#pragma unroll
            for (int c = 0; c < D / 32; ++c) x.v[m][c] = *(const uint2 *)(v + v_at + c * 512);
        }
    };
    Tile<D> even, odd;
    if (w_lo < w_hi) load(w_lo, even);

    // queries: lane & 31 = row (and part: see STACK); features 64 g + 32 half + 8 j .. of step (g, j)
    bf16x8 q[QM][NG * 4];
    const unsigned sixteen = 0x41804180u;
#pragma unroll
    for (int n = 0; n < QM; ++n) {
        const int part = n * QSTACK + l32 / ROWS, r = r0 + (l32 & (ROWS - 1)), t = div_by(r, a.div_per_kv);
        const bool on = l32 < ROWS * QSTACK && part < QP && r < rows;
        const T *x = (const T *)a.x + ((int64_t)b * a.S + (on ? t : 0)) * (a.heads + 2 * a.c.kv_heads) * D + (g * a.per_kv + (on ? r - t * a.per_kv : 0)) * D + half * 32;
#pragma unroll
        for (int i = 0; i < NG * 4; ++i) {
            uint4 raw;
            if constexpr (F32) {
                float v[8];
                load8(x + (i >> 2) * 64 + (i & 3) * 8, v);
                unsigned w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    unsigned p[QP];
                    split_bf16<QP>(v[e], p);
                    w[e] = part == 0 ? p[0] : part == 1 ? p[1] : p[2];
                }
                raw = make_uint4(__builtin_amdgcn_perm(w[1], w[0], 0x07060302u), __builtin_amdgcn_perm(w[3], w[2], 0x07060302u),
                                 __builtin_amdgcn_perm(w[5], w[4], 0x07060302u), __builtin_amdgcn_perm(w[7], w[6], 0x07060302u));
            } else raw = *(const uint4 *)(x + (i >> 2) * 64 + (i & 3) * 8);
            q[n][i] = __builtin_bit_cast(bf16x8, on ? raw : make_uint4(0u, 0u, 0u, 0u));
        }
    }
    // a product's register of row e, parts added
    auto over_parts = [](const f32x16 &d, int e) {
        float v = d[e];
#pragma unroll
        for (int k = 1; k < QSTACK; ++k) v += d[e + k * R4];
        return v;
    };
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    float qs[NG][R4];                                  // sums of the queries over each group, in the registers of their rows
#pragma unroll
    for (int i = 0; i < NG; ++i) {
        f32x16 d = zero;
#pragma unroll
        for (int n = 0; n < QM; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) d = mfma(q[n][i * 4 + j], __builtin_bit_cast(bf16x8, make_uint4(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u)), d);
#pragma unroll
        for (int e = 0; e < R4; ++e) qs[i][e] = over_parts(d, e);
    }
    int at[R4];                                        // position of a register's row, -1: nothing to compute
#pragma unroll
    for (int e = 0; e < R4; ++e) {
        const int r = r0 + 8 * (e >> 2) + 4 * half + (e & 3), t = div_by(r, a.div_per_kv);
        at[e] = r < rows && t < span.count ? span.start + t : -1;
    }
    // every row sees all keys in [all_lo, all_hi)
    const int all_lo = a.window > 0 ? span.start + rg.t1 - a.window + 1 : 0, all_hi = span.start + rg.t0 + 1;

    float base[R4], l[R4], corr[NG][R4];               // base: the reference
    f32x16 o[D / 32];
#pragma unroll
    for (int e = 0; e < R4; ++e) {
        base[e] = NO_SCORE;
        l[e] = 0.f;
#pragma unroll
        for (int i = 0; i < NG; ++i) corr[i][e] = 0.f;
    }
#pragma unroll
    for (int c = 0; c < D / 32; ++c) o[c] = zero;
    unsigned char *pw = lds + wave * PWAVE;

    auto step = [&](const Tile<D> &x, int tile) {
        const int p0 = tile * 64;
        const bool edge = p0 < all_lo || p0 + 64 > all_hi || x.page[0] < 0 || x.page[1] < 0;
        float s[2][R4];
        bool over = false;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            float sc[NG], mm[NG];
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const float t = scale_of(x.ks[m][i]) * a.scale;
                sc[i] = t * TIMES;
                mm[i] = fmaf(BIAS, t, minimum_of(x.ks[m][i]) * a.scale);
            }
#pragma unroll
            for (int e = 0; e < R4; ++e) s[m][e] = 0.f;
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                f32x16 d = zero;
                const unsigned w[4] = {x.k[m][i].x, x.k[m][i].y, x.k[m][i].z, x.k[m][i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16x8 kj = F32 ? codes_around(w[j]) : codes_above(w[j], sixteen);
#pragma unroll
                    for (int n = 0; n < QM; ++n) d = mfma(q[n][i * 4 + j], kj, d);
                }
#pragma unroll
                for (int e = 0; e < R4; ++e) s[m][e] = fmaf(sc[i], over_parts(d, e), fmaf(mm[i], qs[i][e], s[m][e]));
            }
            if (edge) {
                int p = p0 + m * 32 + l32;
                in_branch(p);
#pragma unroll
                for (int e = 0; e < R4; ++e)
                    if (x.page[m] < 0 || p > at[e] || (a.window > 0 && p <= at[e] - a.window)) s[m][e] = -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < R4; ++e) over |= s[m][e] - base[e] > 8.f;
        }
        if (__any(over)) {                             // some score is far above its row's reference: the tile's largest becomes the reference
#pragma unroll
            for (int e = 0; e < R4; ++e) {
                in_branch(s[0][e]);
                float top = fmaxf(s[0][e], s[1][e]);
#pragma unroll
                for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k, 64));
                top = fmaxf(top, base[e]);
                const float f = __builtin_amdgcn_exp2f(base[e] - top);
                base[e] = top;
                l[e] *= f;
#pragma unroll
                for (int i = 0; i < NG; ++i) corr[i][e] *= f;
#pragma unroll
                for (int c = 0; c < D / 32; ++c)
#pragma unroll
                    for (int k = 0; k < STACK; ++k) o[c][e + k * R4] *= f;
            }
        }
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            float p[R4];
#pragma unroll
            for (int e = 0; e < R4; ++e) {
                p[e] = __builtin_amdgcn_exp2f(s[m][e] - base[e]);
                l[e] += p[e];
            }
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const float v = scale_of(x.vs[m][i]), sv = v * TIMES, mv = fmaf(BIAS, v, minimum_of(x.vs[m][i]));
                float ps[R4], pm[R4];
#pragma unroll
                for (int e = 0; e < R4; ++e) {
                    ps[e] = p[e] * sv;
                    pm[e] = p[e] * mv;
                }
                if (edge) {                            // whatever the scales of a key that is not seen hold
#pragma unroll
                    for (int e = 0; e < R4; ++e) {
                        in_branch(ps[e]);
                        if (s[m][e] == -INFINITY) ps[e] = pm[e] = 0.f;
                    }
                }
#pragma unroll
                for (int e = 0; e < R4; ++e) {
                    corr[i][e] += pm[e];
                    unsigned part[PP];
                    split_bf16<PP>(ps[e], part);
                    const int row = 8 * (e >> 2) + 4 * half + (e & 3);
#pragma unroll
                    for (int k = 0; k < PP; ++k) *(unsigned short *)(pw + i * PGROUP + (k * ROWS + row) * PROW + (m * 32 + l32) * 2) = (unsigned short)(part[k] >> 16);
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < NG; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {              // eight keys of each half of block j / 2
                bf16x8 pa[PM];
#pragma unroll
                for (int n = 0; n < PM; ++n) {         // rows beyond the parts: repeated where nothing reads their sums, zeros where a second product would add them
                    const bool real = n * 32 + l32 < PP * ROWS;
                    pa[n] = *(const bf16x8 *)(pw + i * PGROUP + (real ? n * 32 + l32 : l32 & (ROWS - 1)) * PROW + (j >> 1) * 64 + half * 32 + (j & 1) * 16);
                    if (PM > 1 && !real) pa[n] = __builtin_bit_cast(bf16x8, make_uint4(0u, 0u, 0u, 0u));
                }
#pragma unroll
                for (int c = 2 * i; c < 2 * i + 2; ++c) {
                    const unsigned w = j & 1 ? x.v[j >> 1][c].y : x.v[j >> 1][c].x;
                    const bf16x8 vj = F32 ? codes_around(w) : codes_above(w, sixteen);
#pragma unroll
                    for (int n = 0; n < PM; ++n) o[c] = mfma(pa[n], vj, o[c]);
                }
            }
        mfma_settle<DT_BF16>();
        __builtin_amdgcn_wave_barrier();
        asm volatile("" ::: "memory");
    };
    // The next tile is always loaded, at the end the last one again: where a load may or may not have been issued, the wait for an older one
    // waits for it too.
    for (int tile = w_lo; tile < w_hi; tile += 2) {
        load(min(tile + 1, w_hi - 1), odd);
        step(even, tile);
        if (tile + 1 >= w_hi) break;
        load(min(tile + 2, w_hi - 1), even);
        step(odd, tile + 1);
    }

    // the waves' results are joined in LDS, each relative to its own reference
#pragma unroll
    for (int e = 0; e < R4; ++e) {
        l[e] = sum32(l[e]);
#pragma unroll
        for (int i = 0; i < NG; ++i) corr[i][e] = sum32(corr[i][e]);
    }
    __syncthreads();                                   // every wave is done with its patch of weights
    float *mo = (float *)lds;
#pragma unroll
    for (int e = 0; e < R4; ++e) {
        const int row = 8 * (e >> 2) + 4 * half + (e & 3);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            float v = o[c][e] + corr[c / 2][e];
#pragma unroll
            for (int k = 1; k < STACK; ++k) v += o[c][e + k * R4];
            mo[(wave * ROWS + row) * D + c * 32 + l32] = v;
        }
        if (l32 == 0) ends[wave * ROWS + row] = make_float2(base[e], l[e]);
    }
    __syncthreads();
    float *part = a.ws + (a.splits > 1 ? ((((int64_t)b * a.c.kv_heads + g) * a.row_tiles + rt) * a.splits + sp) * (ROWS * (D + 2)) : 0);
    if (tid < ROWS) {                                  // a row: the largest reference, the waves' factors, the sum of the weights
        float top = NO_SCORE, sum = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) top = fmaxf(top, ends[w * ROWS + tid].x);
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = __builtin_amdgcn_exp2f(ends[w * ROWS + tid].x - top);
            sum = fmaf(f, ends[w * ROWS + tid].y, sum);
            factor[w * ROWS + tid] = f;
        }
        const int r = r0 + tid, t = div_by(r, a.div_per_kv);
        if (a.splits > 1) *(float2 *)(part + ROWS * D + tid * 2) = make_float2(top, sum);
        ends[tid] = make_float2(r < rows && t < span.count && sum != 0.f ? 1.f / sum : 0.f, 0.f);
    }
    __syncthreads();
    for (int i = tid * 4; i < ROWS * D; i += NW * 256) {
        const int row = i / D, d = i % D, r = r0 + row, t = div_by(r, a.div_per_kv);
        float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float f = factor[w * ROWS + row];
            const float4 x = *(const float4 *)(mo + (w * ROWS + row) * D + d);
            v[0] = fmaf(f, x.x, v[0]); v[1] = fmaf(f, x.y, v[1]); v[2] = fmaf(f, x.z, v[2]); v[3] = fmaf(f, x.w, v[3]);
        }
        if (a.splits > 1) store_vec4(part + i, v);
        else if (r < rows) {
            const float inv = ends[row].x;
            const bool none = inv == 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = none ? 0.f : v[e] * inv;
            store_vec4((T *)a.y + (((int64_t)b * a.S + t) * a.heads + g * a.per_kv + (r - t * a.per_kv)) * D + d, v);
        }
    }
}

// Joins the splits: D / 4 lanes to a row, and GROUPS of them where there are many splits, each over every GROUPS-th.  A split holds its rows'
// sums [rows][D], relative to their references, then [rows][reference, sum of the weights].
template <typename T, int D, int GROUPS> __global__ __launch_bounds__(256) void cache_attention_join_kernel(AttendArgs a, int outputs)
{
    constexpr int LANES = D / 4, ROWS = 256 / (LANES * GROUPS);                // rows of a workgroup
    __shared__ float4 acc_s[GROUPS > 1 ? 256 : 1];
    __shared__ float2 ml_s[GROUPS > 1 ? GROUPS : 1];
    const int tid = threadIdx.x, lane = tid % LANES, grp = tid / LANES % GROUPS;
    const int out = (int)blockIdx.x * ROWS + tid / (LANES * GROUPS);   // (sequence, token, head), counted from the first sequence of the call
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float top = NO_SCORE, sum = 0.f;
    auto add = [&](float m, float l, const float4 &v) {
        const float now = fmaxf(top, m), f0 = __builtin_amdgcn_exp2f(top - now), f1 = __builtin_amdgcn_exp2f(m - now);
        top = now;
        sum = fmaf(sum, f0, l * f1);
        acc = make_float4(fmaf(acc.x, f0, v.x * f1), fmaf(acc.y, f0, v.y * f1), fmaf(acc.z, f0, v.z * f1), fmaf(acc.w, f0, v.w * f1));
    };
    if (out < outputs) {
        const int bt = div_by(out, a.div_heads), h = out - bt * a.heads, g = div_by(h, a.div_per_kv), zb = div_by(bt, a.div_S), t = bt - zb * a.S, b = a.b_lo + zb;
        const int r = t * a.per_kv + (h - g * a.per_kv), rt = r / a.rows, row = r - rt * a.rows;
        const Span span = span_of(a.c, b, a.S);
        const Range rg = range_of(a, span, rt * a.rows, min(rt * a.rows + a.rows, a.S * a.per_kv));
        const int tiles = rg.hi - rg.lo, per = split_tiles(a, tiles), n = t < span.count && tiles > 0 ? (tiles + per - 1) / per : 0;
        const int64_t step = (int64_t)a.rows * (D + 2);
        const float *ws = a.ws + (((int64_t)b * a.c.kv_heads + g) * a.row_tiles + rt) * a.splits * step;
#pragma unroll 8
        for (int i = grp; i < n; i += GROUPS) {
            const float *x = ws + i * step;
            const float2 ml = *(const float2 *)(x + a.rows * D + row * 2);
            add(ml.x, ml.y, *(const float4 *)(x + row * D + lane * 4));
        }
    }
    if constexpr (GROUPS > 1) {
        acc_s[tid] = acc;
        if (lane == 0) ml_s[grp] = make_float2(top, sum);
        __syncthreads();
        if (grp) return;
#pragma unroll
        for (int i = 1; i < GROUPS; ++i) add(ml_s[i].x, ml_s[i].y, acc_s[i * LANES + lane]);
    }
    if (out >= outputs) return;
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
    const float v[4] = {acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
    store_vec4((T *)a.y + ((int64_t)out + (int64_t)a.b_lo * a.S * a.heads) * D + lane * 4, v);
}

// Whether the splits of a row are joined by several groups of lanes in a workgroup of their own, or one after another; by groups against one after another, us of
// the whole call (bf16, 128 features).  32 results after 131072 keys 41.3 against 43.9, 128 after 32768 25.2 against 28.6, 512 after 2 x 16384 32.7 against
// 35.0, 896 after 16384 34.4 against 37.2; about where the line is 2048 after 8192 35.3 against 34.6; 3584 after 4 x 4096 34.2 against 32.6, 4096 after
// 4096 36.6 against 35.0.  64 features: 1008 after 4 x 4096 18.5 against 19.2, 2160 of them 24.2 against 22.1.
static bool join_by_groups(const AttendArgs &b, int outputs) { return b.splits > 8 && outputs <= 2048; }

template <typename T, int D, int ROWS, int NW> static void attend(const AttendArgs &b, int grid, int outputs, hipStream_t s, int phase)
{
    if (phase != 2) {
        if constexpr (ROWS <= 32) GACER_LAUNCH((cache_attention_kernel<T, D, ROWS, NW>), dim3(grid), dim3(NW * 64), 0, s, b);
        else launch_cache_attention_wide(b, sizeof(T) == 4 ? DT_F32 : DT_BF16, D, grid, s);
    }
    if (b.splits > 1 && phase != 1) {
        if (join_by_groups(b, outputs)) GACER_LAUNCH((cache_attention_join_kernel<T, D, 1024 / D>), dim3((unsigned)outputs), dim3(256), 0, s, b, outputs);
        else GACER_LAUNCH((cache_attention_join_kernel<T, D, 1>), dim3((unsigned)((outputs + 1024 / D - 1) / (1024 / D))), dim3(256), 0, s, b, outputs);
    }
}

LaunchInfo launch_cache_attention(const TokenArgs &a, hipStream_t s, bool dry, int phase)
{
    const AttendGeom g = attend_geom(a);
    AttendArgs b;
    b.x = a.x; b.y = a.y; b.ws = a.ws; b.c = a.cache; b.b_lo = a.b_lo; b.S = a.S; b.heads = a.heads; b.per_kv = a.heads / a.kv_heads;
    b.window = a.window; b.rows = g.rows; b.row_tiles = g.row_tiles; b.splits = g.splits; b.split_min = g.split_min;
    b.scale = a.alpha * 1.4426950408889634f;
    b.groups = (a.b_hi - a.b_lo) * a.kv_heads; b.parts = b.groups * g.splits;
    divisor(b.per_kv, b.div_per_kv); divisor(a.kv_heads, b.div_kv); divisor(a.heads, b.div_heads); divisor(a.S, b.div_S);
    divisor(g.splits, b.div_splits); divisor(g.row_tiles, b.div_tiles); divisor(b.groups, b.div_groups); divisor(b.parts, b.div_parts);
    const int n = a.b_hi - a.b_lo, grid = n * a.kv_heads * g.row_tiles * g.splits;
    const int outputs = n * a.S * a.heads;
    LaunchInfo li;
    li.workgroups = phase == 2 ? (join_by_groups(b, outputs) ? outputs : (int)(((int64_t)outputs * a.D + 1023) / 1024)) : grid;
    li.threads = phase == 2 ? 256 : g.waves * 64;
    const bool f32 = a.dtype == DT_F32, grouped = join_by_groups(b, outputs);
    // up to 32 rows: the waves' patches of weights, or their results, and 12 bytes a row of them
    const int few = g.waves * g.rows * (std::max(a.D / 64 * (f32 ? 3 : 2) * (128 + 16), a.D * 4) + 12);
    li.lds_bytes = phase == 2 ? (grouped ? 4096 + 8192 / a.D : 0) : g.rows == 128 ? 2 * wide_tile_bytes(a.D, f32) : few;
    li.wg_per_cu = phase == 2 ? (!grouped ? 7 : a.D == 64 ? 4 : 6) : g.per_cu;
    li.kernel = phase == 2 ? "cache_attention_join" : a.dtype == DT_BF16 ? "cache_attention_bf16" : "cache_attention_f32";
    li.phases = g.splits > 1 ? 2 : 1;
    if (dry || !grid) return li;
#define ATTEND(TYPE, DIM, ROWS, NW) if (a.D == DIM && g.rows == ROWS && g.waves == NW) attend<TYPE, DIM, ROWS, NW>(b, grid, outputs, s, phase)
    if (a.dtype == DT_BF16) {
        ATTEND(unsigned short, 64, 8, 8); ATTEND(unsigned short, 64, 16, 4); ATTEND(unsigned short, 64, 32, 4); ATTEND(unsigned short, 64, 128, 4);
        ATTEND(unsigned short, 128, 8, 8); ATTEND(unsigned short, 128, 16, 4); ATTEND(unsigned short, 128, 32, 4); ATTEND(unsigned short, 128, 128, 4);
    } else {
        ATTEND(float, 64, 8, 4); ATTEND(float, 64, 16, 4); ATTEND(float, 64, 32, 4); ATTEND(float, 64, 128, 4);
        ATTEND(float, 128, 8, 4); ATTEND(float, 128, 16, 4); ATTEND(float, 128, 32, 4); ATTEND(float, 128, 128, 4);
    }
#undef ATTEND
    return li;
}

}  // namespace gacer
