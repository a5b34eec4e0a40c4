// Attention of many rows (prompts) over a paged 4-bit cache.
//
// A workgroup takes 128 rows (heads x tokens of one key/value head), 32 to a wave, and 64 keys at a time.  The codes are turned into bf16 once
// for all four waves and stand in LDS as the whole numbers c - 8 (the keys of bf16 tenants as 16 + c, which is half the work, and whose sums
// lose less than the rounding of the queries has): keys row by row, values feature by feature.  Scores are keys x rows (lane =
// row), so a row's weights stay in its lanes' registers and are the operand of the values' product, features x rows, as they are; the
// order of the keys within that product is the one in which a lane holds them, and the values are stored in it.  As in the kernel for
// few rows the scales are applied in fp32,
//   q.k_j = sum over groups g of  s_jg * (sum_d q_d (c_jd - z)) + (m_jg + z s_jg) * sum_d q_d             (z = 8 or -16)
//   out_d = sum_j w_jg (c_jd - 8) + sum_j w_jg (m_jg / s_jg + 8)                                        (w_jg = p_j s_jg)
// with the second sum of the scores as a further matrix instruction: the pair (s, m) of a key, two bf16 numbers, times the sums of the queries
// in three bf16 parts, and a one times the parts of minus the row's reference; that of the result likewise in bf16 tenants, the weights times
// m / s + 8 in two parts.  fp32 tenants have their queries and weights in three bf16 parts each, every part a matrix instruction, and add
// p_j (m + 8 s) as it is.  In bf16 tenants the weights w are rounded to bf16 once, and both sums take them rounded, so that what rounding
// does to a key is a factor, however far its values lie from its codes' middle: about as much as the result's own rounding adds, and a second part
// would be 16 more matrix instructions per 64 keys and two more operations per weight.
//
// Bound by the two waves of a SIMD that 254 registers allow: each runs scores, exponentials and products one after another, and vector
// instructions (52 % of the time), matrix instructions (32 %), LDS (35 %, 4 % more by conflicts of banks) and waits (35 % of the waves' time) fill each other's gaps only in part.  A
// prompt of 4096 tokens, 32 heads of 128 features over 8 (bf16): 233 us = 590 TFLOP/s, where a large product reaches 1377.  256 rows a workgroup, which
// halve the unpacking: 5 % faster there, but 98 us against 93 at 2048 tokens and 361 against 344 at 16 x 256 tokens after 4096 keys; two groups
// of waves that take turns at the matrix cores, a barrier after each turn: 17 % slower.
#include <hip/hip_runtime.h>
#include <limits.h>
#include "cache_attention.h"

namespace gacer {

template <typename T, int D> __global__ __launch_bounds__(256, sizeof(T) == 4 && D == 128 ? 1 : 2) void cache_attention_wide_kernel(AttendArgs a)
{
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int QP = F32 ? 3 : 1, PP = F32 ? 3 : 1, MP = 2;                  // bf16 parts of queries, weights, and of the minima (m + 8 s) / s
    constexpr float K_UNIT = F32 ? 16.f : 1.f, K_MIDDLE = F32 ? 8.f : -16.f;   // keys in LDS: (c - 8) / 16 or 16 + c; value of a step, of where they are zero
    constexpr int NG = D / 64, ROWS = 128, KROW = D * 2 + 16, VROW = 128 + 16, KROWS = 64 * KROW, VROWS = D * VROW;
    constexpr int EXT_K = 64 * 32, EXT_V = F32 ? NG * 64 * 4 : (MP * NG + 1) * VROW, BUF = wide_tile_bytes(D, F32);
    constexpr int ITEMS = 64 * D / 32;                 // 16-byte pieces of a tile's key codes, and of its value codes
    __shared__ __align__(16) unsigned char lds[2 * BUF];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, half = lane >> 5;
    // last rows first: they see the most keys; neighbours in the grid, which run on different XCDs, are different heads
    const int back = div_by((int)blockIdx.x, a.div_parts), part = (int)blockIdx.x - back * a.parts, rt = a.row_tiles - 1 - back;
    const int sp = div_by(part, a.div_groups), z = part - sp * a.groups, zb = div_by(z, a.div_kv), g = z - zb * a.c.kv_heads, b = a.b_lo + zb;
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
    const int r = r0 + wave * 32 + l32, t = div_by(r, a.div_per_kv), head = g * a.per_kv + (r - t * a.per_kv);
    const int at = r < rows && t < span.count ? span.start + t : -1;
    // what the wave's rows see: every row all of [all_lo, all_hi), none anything outside [any_lo, any_hi)
    const int w0 = r0 + wave * 32, w1 = min(w0 + 32, rows), t0 = div_by(w0, a.div_per_kv), t1 = min(div_by(max(w1 - 1, 0), a.div_per_kv), span.count - 1);
    const bool idle = w0 >= rows || t0 > t1;
    const int all_lo = a.window > 0 ? span.start + t1 - a.window + 1 : 0, all_hi = span.start + t0 + 1;
    const int any_lo = a.window > 0 ? span.start + t0 - a.window + 1 : 0, any_hi = span.start + t1 + 1;

    // -- a tile's codes and scales: loaded into registers, later turned into operands in LDS -------------------------------------------
    int pages = -1, pages_at = INT_MIN / 2;            // lane i: page of block pages_at + i
    uint4 kin, vin;
    unsigned sin[NG];
    int page_in[2], page_now[2];
    const bool k_mine = tid < ITEMS, v_mine = ITEMS == 256 || tid >= 256 - ITEMS, s_mine = tid < 128;
    const int ki = tid & (ITEMS - 1), kkey = ki / (D / 32), kpart = ki % (D / 32), vblk = ki / D, vd = ki % D, skey = tid & 63;
    auto load = [&](int tile) {
        const int blk = tile * 2;
        if (blk - pages_at >= 64 || blk < pages_at) {
            pages_at = blk;
            pages = page_of(a.c, b, min(blk + lane, 1 << 25) << 5);
        }
        int64_t row[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            page_in[m] = __builtin_amdgcn_readlane(pages, blk - pages_at + m);
            row[m] = page_row(a.c, max(page_in[m], 0), g) + (((blk + m) << 5) & ((1 << a.c.page_shift) - 1));
        }
        kin = *(const uint4 *)(a.c.k_codes + ((kkey >> 5 ? row[1] : row[0]) + (kkey & 31)) * (D / 2) + kpart * 16);
        vin = *(const uint4 *)(a.c.v_codes + (vblk ? row[1] : row[0]) * (D / 2) + vd * 16);
        const unsigned *sc = (tid & 64 ? a.c.v_scales : a.c.k_scales) + ((skey >> 5 ? row[1] : row[0]) + (skey & 31)) * NG;
#pragma unroll
        for (int i = 0; i < NG; ++i) sin[i] = sc[i];
    };
    auto unpack = [&](unsigned char *buf) {
        if (k_mine) {
            const unsigned w[4] = {kin.x, kin.y, kin.z, kin.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) *(bf16x8 *)(buf + kkey * KROW + kpart * 64 + i * 16) = F32 ? codes_around(w[i]) : codes_above(w[i], 0x41804180u);
        }
        if (v_mine) {                                  // of each 16 keys first those that half 0 of a wave holds: 0..3 and 8..11, then 4..7 and 12..15
            const unsigned w[4] = {vin.x, vin.y, vin.z, vin.w};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 p = __builtin_bit_cast(uint4, codes_around(w[2 * i])), q = __builtin_bit_cast(uint4, codes_around(w[2 * i + 1]));
                unsigned char *v = buf + KROWS + vd * VROW + (vblk * 2 + i) * 32;
                *(uint4 *)v = make_uint4(p.x, p.y, q.x, q.y);
                *(uint4 *)(v + 16) = make_uint4(p.z, p.w, q.z, q.w);
            }
        }
        if (s_mine) {
            float *scales = (float *)(buf + KROWS + VROWS + EXT_K + EXT_V);
            const int slot = (skey & 32) + (skey & 16) + ((skey >> 2) & 1) * 8 + ((skey >> 3) & 1) * 4 + (skey & 3);        // as the values' keys
            unsigned e[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const float sc = scale_of(sin[i]), m = minimum_of(sin[i]);
                if (tid < 64) {
                    scales[i * 64 + skey] = sc * K_UNIT * a.scale;
                    e[i] = sin[i];
                } else {
                    if constexpr (F32) {
                        scales[(NG + i) * 64 + skey] = sc * 16.f;
                        ((float *)(buf + KROWS + VROWS + EXT_K))[i * 64 + skey] = fmaf(8.f, sc, m);
                        continue;
                    }
                    // where the scale is nothing against the minimum, a small one: 15 of it are 2^-26 of the minimum
                    const float tiny = fabsf(m) * 0x1p-30f, unit = fabsf(sc) < tiny ? tiny : sc;
                    scales[(NG + i) * 64 + skey] = unit * 16.f;
                    unsigned part[MP];
                    split_bf16<MP>(unit == 0.f ? 0.f : fmaf(__fdiv_rn(m, unit), 0.0625f, 0.5f), part);       // in units of the codes' 16ths
#pragma unroll
                    for (int k = 0; k < MP; ++k) *(unsigned short *)(buf + KROWS + VROWS + EXT_K + (MP * i + k) * VROW + slot * 2) = (unsigned short)(part[k] >> 16);
                }
            }
            if (tid < 64) {                            // slots 0..7: the pairs of the groups, twice; 8..11: once more; 12..14: ones, for the reference
                unsigned char *x = buf + KROWS + VROWS + skey * 32;
                *(uint4 *)x = NG == 2 ? make_uint4(e[0], e[1], e[0], e[1]) : make_uint4(e[0], e[0], e[0], 0u);
                *(uint4 *)(x + 16) = make_uint4(NG == 2 ? e[0] : 0u, NG == 2 ? e[1] : 0u, 0x3F803F80u, 0x3F80u);
            }
        }
    };
    if (lo < hi) load(lo);
    if (!F32 && tid < 2 * VROW / 4) ((unsigned *)(lds + (tid >= VROW / 4) * BUF + KROWS + VROWS + EXT_K + MP * NG * VROW))[tid % (VROW / 4)] = 0u;

    // -- queries: lane & 31 = row; features 16 t + 8 half .. of step t, and the sums of each group as the operand of the pairs -----------
    bf16x8 q[QP][NG * 4], qx;
    {
        const bool on = r < rows;
        const T *x = (const T *)a.x + ((int64_t)b * a.S + (on ? t : 0)) * (a.heads + 2 * a.c.kv_heads) * D + (on ? head : 0) * D + half * 8;
        float sum[NG];
#pragma unroll
        for (int i = 0; i < NG; ++i) sum[i] = 0.f;
#pragma unroll
        for (int i = 0; i < NG * 4; ++i) {
            float v[8];
            load8(x + i * 16, v);
            unsigned part[8][QP];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (!on) v[e] = 0.f;
                sum[i / 4] += v[e];
                split_bf16<QP>(v[e], part[e]);
            }
#pragma unroll
            for (int k = 0; k < QP; ++k) q[k][i] = operand(part[0][k], part[1][k], part[2][k], part[3][k], part[4][k], part[5][k], part[6][k], part[7][k]);
        }
        unsigned pair[NG][3];                          // parts of (K_MIDDLE sum, sum) of each group, as they meet (scale, minimum)
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            const float all = (sum[i] + __shfl_xor(sum[i], 32, 64)) * a.scale;
            unsigned p8[3], p1[3];
            split_bf16<3>(K_MIDDLE * all, p8);
            split_bf16<3>(all, p1);
#pragma unroll
            for (int k = 0; k < 3; ++k) pair[i][k] = __builtin_amdgcn_perm(p1[k], p8[k], 0x07060302u);
        }
        const uint4 first = NG == 2 ? make_uint4(pair[0][0], pair[NG - 1][0], pair[0][1], pair[NG - 1][1]) : make_uint4(pair[0][0], pair[0][1], pair[0][2], 0u);
        const uint4 second = NG == 2 ? make_uint4(pair[0][2], pair[NG - 1][2], 0u, 0u) : make_uint4(0u, 0u, 0u, 0u);       // the reference is 0
        qx = __builtin_bit_cast(bf16x8, half ? second : first);
    }
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    f32x16 o[D / 32], small[F32 ? D / 32 : 1], corr[NG];                 // small: of the weights' second and third parts; corr: the minima's part of the result in bf16
#pragma unroll
    for (int c = 0; c < D / 32; ++c) o[c] = zero;
#pragma unroll
    for (int c = 0; c < (F32 ? D / 32 : 1); ++c) small[c] = zero;
#pragma unroll
    for (int i = 0; i < NG; ++i) corr[i] = zero;
    float base = 0.f, l = 0.f, cr[NG];             // cr: the minima's part of the result, of the lane's keys (fp32) or at the end
#pragma unroll
    for (int i = 0; i < NG; ++i) cr[i] = 0.f;

    // -- 32 keys of a tile: scores, weights, their product with the values ------------------------------------------------------------
    auto block = [&](const unsigned char *buf, int m, int p0, bool edge, bool gone) {
        f32x16 d[NG], x;
#pragma unroll
        for (int i = 0; i < NG; ++i) {
            d[i] = zero;
            bf16x8 k8[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) k8[j] = *(const bf16x8 *)(buf + (m * 32 + l32) * KROW + (i * 4 + j) * 32 + half * 16);
#pragma unroll
            for (int k = QP - 1; k >= 0; --k)          // the small parts first: their sums are rounded before they are large
#pragma unroll
                for (int j = 0; j < 4; ++j) d[i] = mfma(k8[j], q[k][i * 4 + j], d[i]);
        }
        x = mfma(*(const bf16x8 *)(buf + KROWS + VROWS + (m * 32 + l32) * 32 + half * 16), qx, zero);
        const float *scales = (const float *)(buf + KROWS + VROWS + EXT_K + EXT_V) + m * 32 + half * 4;
        float s[16], top = -INFINITY;                  // scores above the reference, which the extra product takes off: those that count are small when they are rounded
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float4 sc[NG];
#pragma unroll
            for (int i = 0; i < NG; ++i) sc[i] = *(const float4 *)(scales + i * 64 + k * 8);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float v = x[4 * k + e];
#pragma unroll
                for (int i = 0; i < NG; ++i) v = fmaf(e == 0 ? sc[i].x : e == 1 ? sc[i].y : e == 2 ? sc[i].z : sc[i].w, d[i][4 * k + e], v);
                s[4 * k + e] = v;
            }
        }
        if (edge) {
            int q0 = p0 + 4 * half;
            in_branch(q0);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int p = q0 + 8 * (e >> 2) + (e & 3);
                if (gone || p > at || (a.window > 0 && p <= at - a.window)) s[e] = -INFINITY;
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s[e]);
        if (__any(top > 8.f || (l == 0.f && top > -INFINITY))) {      // the largest score so far becomes the reference, and the first one
            in_branch(top);
            const bool first = l + __shfl_xor(l, 32, 64) == 0.f;
            top = fmaxf(top, __shfl_xor(top, 32, 64));
            const float up = top == -INFINITY ? 0.f : first ? top : fmaxf(top, 0.f), f = first ? 1.f : __builtin_amdgcn_exp2f(-up);
            base += up;
            unsigned part[3];
            split_bf16<3>(-base, part);
            base = -(__uint_as_float(part[0] & 0xFFFF0000u) + __uint_as_float(part[1] & 0xFFFF0000u) + __uint_as_float(part[2] & 0xFFFF0000u));
            if (half) {
                uint4 u = __builtin_bit_cast(uint4, qx);
                u.z = __builtin_amdgcn_perm(part[1], part[0], 0x07060302u);
                u.w = part[2] >> 16;
                qx = __builtin_bit_cast(bf16x8, u);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] -= up;
            l *= f;
#pragma unroll
            for (int i = 0; i < NG; ++i) cr[i] *= f;
#pragma unroll
            for (int i = 0; i < (F32 ? 0 : NG); ++i) {      // the two rows of a group's sums that are looked at
                corr[i][2 * i] *= f;
                corr[i][2 * i + 1] *= f;
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    o[c][e] *= f;
                    if constexpr (F32) small[c][e] *= f;
                }
            }
        }
        float p[16], sum[8];
#pragma unroll
        for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f(s[e]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = p[e] + p[e + 8];
        l += ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));      // one at a time a thousand keys cost l 1e-6
#pragma unroll
        for (int k = 0; k < 2; ++k) {                  // 16 keys
            bf16x8 w[NG][PP];                          // the weights times the groups' scales
#pragma unroll
            for (int i = 0; i < NG; ++i) {
                const float4 s0 = *(const float4 *)(scales + (NG + i) * 64 + k * 16), s1 = *(const float4 *)(scales + (NG + i) * 64 + k * 16 + 8);
                float v[8] = {p[8 * k] * s0.x, p[8 * k + 1] * s0.y, p[8 * k + 2] * s0.z, p[8 * k + 3] * s0.w,
                              p[8 * k + 4] * s1.x, p[8 * k + 5] * s1.y, p[8 * k + 6] * s1.z, p[8 * k + 7] * s1.w};
                if (edge) {                            // whatever the scales of a key that is not seen hold
#pragma unroll
                    for (int e = 0; e < 8; ++e) in_branch(v[e]);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (s[8 * k + e] == -INFINITY) v[e] = 0.f;
                }
                operands<PP>(v, w[i]);
            }
            const int at_key = (m * 2 + k) * 32 + half * 16;
            if constexpr (F32) {
                const float *mm = (const float *)(buf + KROWS + VROWS + EXT_K) + m * 32 + half * 4 + k * 16;
#pragma unroll
                for (int i = 0; i < NG; ++i) {
                    const float4 m0 = *(const float4 *)(mm + i * 64), m1 = *(const float4 *)(mm + i * 64 + 8);
                    float v[8] = {p[8 * k] * m0.x, p[8 * k + 1] * m0.y, p[8 * k + 2] * m0.z, p[8 * k + 3] * m0.w,
                                  p[8 * k + 4] * m1.x, p[8 * k + 5] * m1.y, p[8 * k + 6] * m1.z, p[8 * k + 7] * m1.w};
                    if (edge) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) in_branch(v[e]);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (s[8 * k + e] == -INFINITY) v[e] = 0.f;
                    }
                    cr[i] += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
                }
            } else {
#pragma unroll
                for (int i = 0; i < NG; ++i) {             // the minima of a group meet the weights of that group, in sums of their own: the other group's may be NaN
                    bf16x8 mx = *(const bf16x8 *)(buf + KROWS + VROWS + EXT_K + (l32 / MP == i ? l32 : MP * NG) * VROW + at_key);
                    if (edge) {                            // the same for them: an operand that holds no NaN
                        uint4 u = __builtin_bit_cast(uint4, mx);
                        unsigned *e = (unsigned *)&u;
                        asm volatile("" : "+v"(e[0]));
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if ((e[j] & 0x7F80u) == 0x7F80u) e[j] &= 0xFFFF0000u;
                            if ((e[j] & 0x7F800000u) == 0x7F800000u) e[j] &= 0xFFFFu;
                        }
                        mx = __builtin_bit_cast(bf16x8, u);
                    }
                    corr[i] = mfma(mx, w[i][0], corr[i]);
                }
            }
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                const bf16x8 v8 = *(const bf16x8 *)(buf + KROWS + (c * 32 + l32) * VROW + at_key);
#pragma unroll
                for (int n = 0; n < PP; ++n) {
                    if (F32 && n) small[F32 ? c : 0] = mfma(v8, w[c / 2][n], small[F32 ? c : 0]);
                    else o[c] = mfma(v8, w[c / 2][n], o[c]);
                }
            }
        }
        mfma_settle<DT_BF16>();
    };
    for (int tile = lo; tile < hi; ++tile) {
        unsigned char *buf = lds + ((tile - lo) & 1) * BUF;
        unpack(buf);
        page_now[0] = page_in[0];
        page_now[1] = page_in[1];
        __syncthreads();
        load(min(tile + 1, hi - 1));
        if (idle) continue;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int p0 = tile * 64 + m * 32;
            if (p0 >= any_hi || p0 + 32 <= any_lo) continue;
            const bool gone = page_now[m] < 0;
            block(buf, m, p0, gone || p0 < all_lo || p0 + 32 > all_hi, gone);
        }
    }

    if constexpr (F32) {
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[c][e] += small[c][e];
    }
    l += __shfl_xor(l, 32, 64);
#pragma unroll
    for (int i = 0; i < NG; ++i) {
        if constexpr (F32) cr[i] += __shfl_xor(cr[i], 32, 64);
        else {                                         // rows 2 i and 2 i + 1 of the product, in half 0
            const float v = corr[i][2 * i] + corr[i][2 * i + 1], other = __shfl_xor(v, 32, 64);
            cr[i] = half ? other : v;
        }
    }
    if (r >= rows) return;
    if (a.splits > 1) {
        float *ws = a.ws + ((((int64_t)b * a.c.kv_heads + g) * a.row_tiles + rt) * a.splits + sp) * (ROWS * (D + 2));
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = o[c][4 * k + e] + cr[c / 2];
                store_vec4(ws + (r - r0) * D + c * 32 + k * 8 + half * 4, v);
            }
        if (!half) *(float2 *)(ws + ROWS * D + (r - r0) * 2) = make_float2(l != 0.f ? base : NO_SCORE, l);
        return;
    }
    const bool seen = at >= 0 && l != 0.f;
    const float inv = 1.f / l;
    T *y = (T *)a.y + (((int64_t)b * a.S + t) * a.heads + head) * D + half * 4;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = seen ? (o[c][4 * k + e] + cr[c / 2]) * inv : 0.f;
            store_vec4(y + c * 32 + k * 8, v);
        }
}

void launch_cache_attention_wide(const AttendArgs &b, int dtype, int D, int grid, hipStream_t s)
{
    if (dtype == DT_BF16 && D == 64) GACER_LAUNCH((cache_attention_wide_kernel<unsigned short, 64>), dim3(grid), dim3(256), 0, s, b);
    else if (dtype == DT_BF16) GACER_LAUNCH((cache_attention_wide_kernel<unsigned short, 128>), dim3(grid), dim3(256), 0, s, b);
    else if (D == 64) GACER_LAUNCH((cache_attention_wide_kernel<float, 64>), dim3(grid), dim3(256), 0, s, b);
    else GACER_LAUNCH((cache_attention_wide_kernel<float, 128>), dim3(grid), dim3(256), 0, s, b);
}

}  // namespace gacer
