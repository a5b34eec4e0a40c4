// What the attention kernels over a 4-bit cache share: their arguments, the range of keys of some rows, codes as operands of matrix instructions.
#pragma once
#include "cache_util.h"
#include "gemm_util.h"
#include "kernels.h"

namespace gacer {

struct AttendArgs {
    const void *x;
    void *y;
    float *ws;
    CacheView c;
    int b_lo, S, heads, per_kv, window, rows, row_tiles, splits, split_min;      // rows: of a row tile; split_min: fewest tiles of 64 keys in a split
    float scale;               // alpha * log2(e)
    // set by the launcher, see divisor(): heads per kv head, kv heads, heads, tokens, splits, row tiles, (sequence, kv head) pairs, those times splits
    unsigned div_per_kv[2], div_kv[2], div_heads[2], div_S[2], div_splits[2], div_tiles[2], div_groups[2], div_parts[2];
    int groups, parts;
};

// the tiles of each split of n tiles
__device__ __forceinline__ int split_tiles(const AttendArgs &a, int n) { return max(a.split_min, (n + a.splits - 1) / a.splits); }

// The tiles of 64 keys that rows [r0, r1) of a sequence see, and the first and last of its tokens among them (t1 < t0: none)
struct Range { int t0, t1, lo, hi; };
__device__ __forceinline__ Range range_of(const AttendArgs &a, const Span &s, int r0, int r1)
{
    Range g;
    g.t0 = div_by(r0, a.div_per_kv);
    g.t1 = min(div_by(r1 - 1, a.div_per_kv), s.count - 1);
    g.lo = g.hi = 0;
    if (g.t1 >= g.t0) {
        const int first = a.window > 0 ? max(0, s.start + g.t0 - a.window + 1) : 0;
        const int last = min(s.start + g.t1, (a.c.max_pages << a.c.page_shift) - 1);
        g.lo = first >> 6;
        g.hi = max(g.lo, (last >> 6) + 1);
    }
    return g;
}

// eight codes of a word as the bf16 numbers 16 + c
__device__ __forceinline__ unsigned and_or(unsigned a, unsigned mask, unsigned bits)
{
    unsigned r;                                        // one instruction; from plain operators the compiler makes two, each with a literal
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "s"(mask), "v"(bits));
    return r;
}
__device__ __forceinline__ bf16x8 codes_above(unsigned w, unsigned sixteen)
{
    constexpr unsigned MASK = 0x00780078u;
    return __builtin_bit_cast(bf16x8, make_uint4(and_or(w << 3, MASK, sixteen), and_or(w >> 1, MASK, sixteen), and_or(w >> 5, MASK, sixteen), and_or(w >> 9, MASK, sixteen)));
}
// and as (c - 8) / 16: the hardware's conversion of a signed 4-bit number
__device__ __forceinline__ bf16x8 codes_around(unsigned w)
{
    const unsigned x = w ^ 0x88888888u;
    unsigned r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned lo = __float_as_uint(__builtin_amdgcn_cvt_off_f32_i4((int)(x >> (4 * i)))), hi = __float_as_uint(__builtin_amdgcn_cvt_off_f32_i4((int)(x >> (4 * i + 16))));
        r[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
    }
    return __builtin_bit_cast(bf16x8, make_uint4(r[0], r[1], r[2], r[3]));
}

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

// v as a sum of PARTS numbers whose upper 16 bits are bf16, each the largest that does not pass it, but for the second of two, which is rounded: errors
// that all lie on one side add up over the keys (weights of 131072 keys: an error of 8.5e-3 of the result, which is small against each of its terms).
// Three hold all of v.
template <int PARTS> __device__ __forceinline__ void split_bf16(float v, unsigned *p)
{
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        p[i] = __float_as_uint(v);
        if (PARTS == 2 && i == 1) p[i] += 0x8000u;
        v -= __uint_as_float(p[i] & 0xFFFF0000u);
    }
}

// eight numbers whose upper 16 bits are bf16, as an operand
__device__ __forceinline__ bf16x8 operand(unsigned a, unsigned b, unsigned c, unsigned d, unsigned e, unsigned f, unsigned g, unsigned h)
{
    return __builtin_bit_cast(bf16x8, make_uint4(__builtin_amdgcn_perm(b, a, 0x07060302u), __builtin_amdgcn_perm(d, c, 0x07060302u),
                                                 __builtin_amdgcn_perm(f, e, 0x07060302u), __builtin_amdgcn_perm(h, g, 0x07060302u)));
}
// eight numbers as PARTS operands, one: rounded
template <int PARTS> __device__ __forceinline__ void operands(const float *v, bf16x8 *out)
{
    if constexpr (PARTS == 1) {
        out[0] = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])));
    } else {
        unsigned p[8][PARTS];
#pragma unroll
        for (int e = 0; e < 8; ++e) split_bf16<PARTS>(v[e], p[e]);
#pragma unroll
        for (int k = 0; k < PARTS; ++k) out[k] = operand(p[0][k], p[1][k], p[2][k], p[3][k], p[4][k], p[5][k], p[6][k], p[7][k]);
    }
}

// the reference of a row that has seen no key yet; scores lie above it
static constexpr float NO_SCORE = -1e38f;

// Keeps the (wave-uniform) branch around it a branch: as selects, every tile would pay for what only the first and the last need.
template <typename V> __device__ __forceinline__ void in_branch(V &v) { asm volatile("" : "+v"(v)); }

// Bytes of LDS that a tile of 64 unpacked keys and values takes in the kernel for 128 rows: rows of keys and of features (16 bytes apart more
// than they are long, so that their starts fall on all banks), the keys' further operand, the minima (bf16 tenants: in
// two parts, and a row of zeros), the scales
constexpr int wide_tile_bytes(int D, bool f32) { return 64 * (2 * D + 16) + D * 144 + 64 * 32 + (f32 ? D / 64 * 256 : (D / 64 * 2 + 1) * 144) + D / 64 * 512; }

void launch_cache_attention_wide(const AttendArgs &b, int dtype, int D, int grid, hipStream_t s);      // rows of 128

}  // namespace gacer
