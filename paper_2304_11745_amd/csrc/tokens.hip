// Operators of a decoding tenant that stream over tokens: norm and rotation of queries and keys, writing a 4-bit cache and reading it back.
#include <hip/hip_runtime.h>
#include <algorithm>
#include "cache_util.h"
#include "device_util.h"
#include "kernels.h"
#include "tokens_geom.h"

namespace gacer {

static LaunchInfo info(const char *name, int64_t workgroups, int lds)
{
    LaunchInfo li;
    li.workgroups = (int)workgroups; li.threads = 256; li.lds_bytes = lds; li.wg_per_cu = 8; li.kernel = name; li.phases = 1;
    return li;
}

// ---- RMS norm and rotation ---------------------------------------------------------------------------------------------------------
// y = x * rsqrt(mean(x^2) + eps) * gamma for every query and key head, then (a, b) -> (a c - b s, b c + a s) for its pairs.
//
// A head is held by LPH lanes, eight features each: two runs of four, which are the two halves of the lane's pairs (i, i + R/2), so that
// the rotation needs no other lane; beyond the rotated features, and for interleaved pairs, the two runs are neighbours.  Cosine and sine
// depend on the token and the lane alone and are loaded once for all heads that a workgroup takes; the token's positions come through the scalar
// cache.  Every element is read and written once: bound by the way to memory and back (3 x 4111 tokens of 28 + 4 + 4 heads of 128 features, bf16, 227
// MB: 52 us = 4.4 TB/s, vector instructions busy 73 % of it; fp32, 457 MB, 84 us = 5.5 TB/s).  A lane takes three heads; two take
// 64 us, four 55 (few models' heads fill them), one 113 against 80 at 16384 tokens of 32 + 8 + 8 heads, and no faster for a single token (5 us, a launch).
// In fp32 the loads of all three are in flight together; in bf16 they are converted where they are loaded, under the same condition, and each head's
// loads are waited for before the next one's are issued.
struct RopeArgs {
    const void *x;
    void *y;
    const float *gamma_q, *gamma_k, *table;
    const int *positions;
    float eps, inv_d;
    int D, R, interleaved, axes, s1, s2, n_positions;
    int width, heads, normed, all;      // elements per token; query heads; query and key heads; heads to write (values too unless in place)
    int t_lo;                           // first token
};

__device__ __forceinline__ void load4(const float *p, float *v)
{
    const float4 a = *(const float4 *)p;
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
}
__device__ __forceinline__ void load4(const unsigned short *p, float *v)
{
    const uint2 a = *(const uint2 *)p;
    v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xFFFF0000u);
    v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xFFFF0000u);
}
__device__ __forceinline__ void store4(float *p, const float *v) { *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store4(unsigned short *p, const float *v) { *(uint2 *)p = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])); }

template <typename T, int LPH, int IT> __global__ __launch_bounds__(256) void qknorm_rope_kernel(RopeArgs a)
{
    constexpr int SLOTS = 256 / LPH;
    const int tid = threadIdx.x, sub = tid % LPH, slot = tid / LPH;
    const int64_t token = a.t_lo + (int64_t)blockIdx.x;
    const int h0 = (int)blockIdx.y * (SLOTS * IT) + slot;
    const T *x = (const T *)a.x + token * a.width;
    T *y = (T *)a.y + token * a.width;
    const bool on = sub * 8 < a.D, turned = sub * 8 < a.R, halves = turned && !a.interleaved;
    const int f0 = halves ? sub * 4 : sub * 8, f1 = halves ? a.R / 2 + sub * 4 : sub * 8 + 4;

    float v[IT][8];
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int h = h0 + i * SLOTS;
        if (on && h < a.all) {
            load4(x + h * a.D + f0, v[i]);
            load4(x + h * a.D + f1, v[i] + 4);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        }
    }
    int pos[3] = {0, 0, 0};                            // the token's position on each axis (a missing one is not looked at)
    if (a.R > 0) {                                     // without rotated features there are no positions
#pragma unroll
        for (int i = 0; i < 3; ++i) pos[i] = fixed_int(a.positions, token * a.axes + min(i, a.axes - 1));
    }
    float c[4], s[4];
    if (turned) {
        const int pair = sub * 4, half = a.R / 2;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int at = pair + e < a.s1 ? pos[0] : pair + e < a.s2 ? pos[1] : pos[2];
            const bool known = (unsigned)at < (unsigned)a.n_positions;
            const float2 cs = *(const float2 *)(a.table + ((int64_t)(known ? at : 0) * half + pair + e) * 2);
            c[e] = known ? cs.x : NAN;
            s[e] = known ? cs.y : NAN;
        }
    }
    float gq[8], gk[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) gq[e] = gk[e] = 1.f;
    if (on && a.gamma_q) { load4(a.gamma_q + f0, gq); load4(a.gamma_q + f1, gq + 4); }
    if (on && a.gamma_k) { load4(a.gamma_k + f0, gk); load4(a.gamma_k + f1, gk + 4); }
#pragma unroll
    for (int i = 0; i < IT; ++i) {
        const int h = h0 + i * SLOTS;
        if (__builtin_amdgcn_readfirstlane(h) >= a.all) break;         // none of the wave's heads
        const bool query = h < a.heads;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fmaf(v[i][e], v[i][e], sum);
#pragma unroll
        for (int o = LPH / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        if (!on || h >= a.all) continue;
        if (h < a.normed) {
            if (query ? a.gamma_q != nullptr : a.gamma_k != nullptr) {
                const float r = rsqrtf(fmaf(sum, a.inv_d, a.eps));
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = v[i][e] * r * (query ? gq[e] : gk[e]);
            }
            if (turned) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = a.interleaved ? v[i][2 * e] : v[i][e], q = a.interleaved ? v[i][2 * e + 1] : v[i][e + 4];
                    const float lo = p * c[e] - q * s[e], hi = q * c[e] + p * s[e];
                    if (a.interleaved) { v[i][2 * e] = lo; v[i][2 * e + 1] = hi; }
                    else { v[i][e] = lo; v[i][e + 4] = hi; }
                }
            }
        }
        store4(y + h * a.D + f0, v[i]);
        store4(y + h * a.D + f1, v[i] + 4);
    }
}

static constexpr int HEADS_AT_A_TIME = 3;

template <typename T, int LPH> static void rope_launch(RopeArgs b, int64_t tokens, hipStream_t s)
{
    const int heads = 256 / LPH * HEADS_AT_A_TIME;
    for (int64_t at = 0; at < tokens; at += 1 << 22, b.t_lo += 1 << 22) {        // a grid holds fewer than 2^32 threads
        const unsigned n = (unsigned)std::min<int64_t>(tokens - at, 1 << 22);
        GACER_LAUNCH((qknorm_rope_kernel<T, LPH, HEADS_AT_A_TIME>), dim3(n, (b.all + heads - 1) / heads), dim3(256), 0, s, b);
    }
}

LaunchInfo launch_qknorm_rope(const TokenArgs &a, hipStream_t s, bool dry)
{
    RopeArgs b;
    b.x = a.x; b.y = a.y; b.gamma_q = a.gamma_q; b.gamma_k = a.gamma_k; b.table = a.table; b.positions = a.positions;
    b.eps = a.eps; b.inv_d = 1.f / (float)a.D;
    b.D = a.D; b.R = a.R; b.interleaved = a.interleaved; b.axes = a.axes; b.n_positions = a.n_positions;
    b.s1 = a.axes > 1 ? a.sections[0] : a.R; b.s2 = a.axes > 2 ? a.sections[0] + a.sections[1] : a.R;
    b.width = (a.heads + 2 * a.kv_heads) * a.D;
    b.heads = a.heads; b.normed = a.heads + a.kv_heads; b.all = b.normed + (a.x == a.y ? 0 : a.kv_heads);
    b.t_lo = a.b_lo * a.S;
    const int64_t tokens = (int64_t)(a.b_hi - a.b_lo) * a.S;
    int lph = 1;
    while (lph * 8 < a.D) lph *= 2;
    const int heads = 256 / lph * HEADS_AT_A_TIME;
    LaunchInfo li = info(a.dtype == DT_BF16 ? "qknorm_rope_bf16" : "qknorm_rope_f32", tokens * ((b.all + heads - 1) / heads), 0);
    if (dry || !tokens) return li;
#define ROPE(L)                                                                              \
    case L:                                                                                  \
        if (a.dtype == DT_BF16) rope_launch<unsigned short, L>(b, tokens, s);           \
        else rope_launch<float, L>(b, tokens, s);                                       \
        break
    switch (lph) {
        ROPE(1); ROPE(2); ROPE(4); ROPE(8); ROPE(16); ROPE(32); ROPE(64);
    }
#undef ROPE
    return li;
}

// ---- into the cache and out of it --------------------------------------------------------------------------------------------------
// A workgroup owns one block of 32 cache positions of one kv head (a block never crosses a page).  Writing: half of its waves quantise
// keys, half values, eight features of a token per lane; a group's minimum and maximum go over the eight lanes that hold it.  Key codes
// are one word per lane as they stand.  Of the values a wave takes eight tokens at a time, 64 features of each, and the eight lanes that
// hold the same features transpose their 8 x 8 codes in three exchanges; where a word also has codes of tokens outside the call, those stay.
// Nothing goes through LDS but the exchanges.  6 prompts of up to 5001 tokens, 8 kv heads of 128 features (bf16, 154 MB) 44 us = 3.5 TB/s; by divisions and
// with the transposition by LDS atomics 65.  Vector instructions, 18 for an element, are busy 70 % of that; the rest are waits: in bf16 a lane's loads, one for
// each pass, are converted where they are loaded and so follow one another (in fp32 they are in flight together).
// Reading is a copy that widens: value codes go through LDS to become rows of a token again.  The same prompts 25 us; 8 x 8192 tokens
// (327 MB) 67 us = 4.9 TB/s, what a large copy reaches.
struct CacheArgs {
    const void *x;
    void *y;
    CacheView c;
    int b_lo, S, blocks, width, k_off;  // blocks: of 32 positions, per sequence and kv head; k_off: first key feature of a token
};

struct Block { int b, head, p0; Span span; };
__device__ __forceinline__ Block block_of(const CacheArgs &a)
{
    Block k;
    const int z = (int)blockIdx.x / a.blocks;
    k.b = a.b_lo + z / a.c.kv_heads;
    k.head = z % a.c.kv_heads;
    k.span = span_of(a.c, k.b, a.S);
    k.p0 = (k.span.start / 32 + (int)blockIdx.x % a.blocks) * 32;
    return k;
}

// Over the eight lanes of a group: with the neighbour, the other pair, the other four (in reverse).  One instruction each, after the two wait states that
// such a move asks for behind the instruction that wrote its source; from builtins the compiler makes three.
#define GROUP_STEP(op, v, move) asm("s_nop 1\n\t" op "_dpp %0, %1, %1 " move " row_mask:0xf bank_mask:0xf" : "=v"(v) : "v"(v))
__device__ __forceinline__ float group_min(float v)
{
    GROUP_STEP("v_min_f32", v, "quad_perm:[1,0,3,2]");
    GROUP_STEP("v_min_f32", v, "quad_perm:[2,3,0,1]");
    GROUP_STEP("v_min_f32", v, "row_half_mirror");
    return v;
}
__device__ __forceinline__ float group_max(float v)
{
    GROUP_STEP("v_max_f32", v, "quad_perm:[1,0,3,2]");
    GROUP_STEP("v_max_f32", v, "quad_perm:[2,3,0,1]");
    GROUP_STEP("v_max_f32", v, "row_half_mirror");
    return v;
}
#undef GROUP_STEP

// d / s, correctly rounded, for an s of few significant bits (8 at most) and `inverse` within some units of 1 / s: the remainder of the first guess is exact, and the
// quotient is either half way between two numbers or further from there than 2^-9 of their distance, while the second guess errs by 2^-21 of it.
__device__ __forceinline__ float divided(float d, float s, float inverse)
{
    const float q = __fmul_rn(d, inverse);
    return __fmaf_rn(__fmaf_rn(-q, s, d), inverse, q);
}

// eight values of one lane -> their code word; `pair` receives scale and minimum of the group of eight lanes (a minimum of zero without a
// sign: which of two zeros a minimum returns is not defined)
__device__ __forceinline__ unsigned quantise(const float *v, unsigned &pair)
{
    float lo = v[0], hi = v[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
        lo = __builtin_elementwise_minimum(lo, v[e]);  // NaN if there is any
        hi = fmaxf(hi, v[e]);
    }
    lo = group_min(lo == lo ? lo : -INFINITY);
    hi = group_max(hi);
    const unsigned short low = to_bf16(lo), step = to_bf16(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f));
    const float m = ld_f32(&low, 0) + 0.f, s = ld_f32(&step, 0);
    if (!(fabsf(s) < INFINITY && fabsf(m) < INFINITY)) {
        pair = 0x7FC0u;
        return 0u;
    }
    pair = (unsigned)step | __float_as_uint(m);
    if (!(s > 0.f)) return 0u;
    float q[8];
    if (__any(!(s > 0x1p-100f && s < 0x1p100f))) {     // 1 / s or a remainder may not be a number of full precision
        asm volatile("");                              // a branch: both sides would cost more than the divisions alone
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = __fdiv_rn(__fsub_rn(v[e], m), s);
    } else {
        const float inverse = __builtin_amdgcn_rcpf(s);
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = divided(__fsub_rn(v[e], m), s, inverse);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = __builtin_amdgcn_fmed3f(rintf(q[e]), 0.f, 15.f);
    // elements of even and of odd index: sums of codes times powers of 16, whole numbers
    const float even = fmaf(fmaf(fmaf(q[6], 16.f, q[4]), 16.f, q[2]), 16.f, q[0]), odd = fmaf(fmaf(fmaf(q[7], 16.f, q[5]), 16.f, q[3]), 16.f, q[1]);
    return (unsigned)even | (unsigned)odd << 16;
}

// Lane 8 t + s of a wave has the codes of token t, features 8 s ..; lane f receives those of feature f, tokens 0..7.  Three exchanges, one for each
// bit of the index: halves of a word, then of its bytes, then of its halves' bytes (the order of code_shift()).
__device__ __forceinline__ unsigned transpose_codes(unsigned w)
{
    const int lane = threadIdx.x & 63;
    auto exchange = [&](int across, unsigned mask, int shift) {
        const unsigned o = (unsigned)__shfl_xor((int)w, across, 64);
        w = lane & across ? (w & ~mask) | (o & ~mask) >> shift : (w & mask) | (o & mask) << shift;
    };
    exchange(8, 0x0000FFFFu, 16);
    exchange(16, 0x0F0F0F0Fu, 4);
    exchange(32, 0x00FF00FFu, 8);
    return (unsigned)__shfl((int)w, (lane & 7) * 8 + (lane >> 3), 64);       // in the order of the features: neighbours store neighbours
}

template <typename T, int D> __global__ __launch_bounds__(256) void cache_write_kernel(CacheArgs a)
{
    constexpr int LPT = D / 8, PER = 128 / LPT, PASSES = 32 / PER, NG = D / CACHE_GROUP;     // lanes per token, tokens per pass of a half
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6 & 1;
    const bool values = __builtin_amdgcn_readfirstlane(tid >> 7);
    const Block k = block_of(a);
    const int lo = max(k.p0, k.span.start), hi = min(k.p0 + 32, k.span.start + k.span.count);
    if (lo >= hi) return;
    const int page = page_of(a.c, k.b, k.p0);
    if (page < 0) return;
    const int64_t first = page_row(a.c, page, k.head) + (k.p0 & ((1 << a.c.page_shift) - 1));
    // the lane's features 8 sub .. and tokens: keys row by row, values eight tokens of 64 features a wave
    const int sub = !values ? tid & (LPT - 1) : D == 128 ? wave * 8 + (lane & 7) : lane & 7;
    const int row = !values ? (tid & 127) / LPT : (D == 128 ? 0 : wave * PASSES * 8) + (lane >> 3), next = values ? 8 : PER;
    const T *x = (const T *)a.x + ((int64_t)k.b * a.S - k.span.start) * a.width + a.k_off + (values * a.c.kv_heads + k.head) * D + sub * 8;
    float v[PASSES][8];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int p = k.p0 + i * next + row;
        if (p >= lo && p < hi) load8(x + (int64_t)p * a.width, v[i]);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        }
    }
    unsigned words[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int t = i * next + row, p = k.p0 + t;
        unsigned pair;
        words[i] = quantise(v[i], pair);
        if (p < lo || p >= hi) continue;
        if (!values) ((unsigned *)a.c.k_codes)[(first + t) * LPT + sub] = words[i];
        if (sub % 8 == 0) (values ? a.c.v_scales : a.c.k_scales)[(first + t) * NG + sub / 8] = pair;
    }
    if (!values) return;
    unsigned *out = (unsigned *)a.c.v_codes + first * LPT + ((sub & ~7) * 8 + lane) * 4;       // the feature's four words of eight tokens
    const int w0 = D == 128 ? 0 : wave * PASSES;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) words[i] = transpose_codes(words[i]);
    if (lo == k.p0 && hi == k.p0 + 32) {
        if constexpr (PASSES == 4) *(uint4 *)out = make_uint4(words[0], words[1], words[2], words[3]);
        else *(uint2 *)(out + w0) = make_uint2(words[0], words[1]);
        return;
    }
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int q0 = k.p0 + (w0 + i) * 8;
        if (q0 >= hi || q0 + 8 <= lo) continue;
        unsigned mine = 0u;                            // of the word's codes those that the call writes
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (q0 + e >= lo && q0 + e < hi) mine |= 15u << code_shift(e);
        unsigned w = words[i];
        if (mine != ~0u) w = (w & mine) | (out[w0 + i] & ~mine);
        out[w0 + i] = w;
    }
}

template <typename T, int D> __global__ __launch_bounds__(256) void cache_read_kernel(CacheArgs a)
{
    constexpr int LPT = D / 8, PER = 256 / LPT, PASSES = 32 / PER, NG = D / CACHE_GROUP;
    __shared__ __align__(8) unsigned char codes[32][D + 8];      // value codes, a row per token
    const int tid = threadIdx.x, sub = tid & (LPT - 1), row = tid / LPT;
    const Block k = block_of(a);
    const int page = k.p0 < k.span.start + k.span.count ? page_of(a.c, k.b, k.p0) : -1;
    const int64_t first = page < 0 ? 0 : page_row(a.c, page, k.head) + (k.p0 & ((1 << a.c.page_shift) - 1));
    if (page >= 0) {
        const unsigned *w = (const unsigned *)a.c.v_codes + first * LPT;
        for (int i = tid; i < D * 4; i += 256) {
            const unsigned word = w[i];
#pragma unroll
            for (int e = 0; e < 8; ++e) codes[(i & 3) * 8 + e][i >> 2] = (unsigned char)((word >> code_shift(e)) & 15u);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int t = i * PER + row, p = k.p0 + t;
        if (p < k.span.start || p >= k.span.start + a.S) continue;
        T *y = (T *)a.y + ((int64_t)k.b * a.S + (p - k.span.start)) * a.width + k.head * D + sub * 8;
        float kv[8], vv[8];
        if (page >= 0 && p < k.span.start + k.span.count) {
            const unsigned word = ((const unsigned *)a.c.k_codes)[(first + t) * LPT + sub];
            const unsigned kp = a.c.k_scales[(first + t) * NG + sub / 8], vp = a.c.v_scales[(first + t) * NG + sub / 8];
            const uint2 c8 = *(const uint2 *)&codes[t][sub * 8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                kv[e] = fmaf((float)((word >> code_shift(e)) & 15u), scale_of(kp), minimum_of(kp));
                vv[e] = fmaf((float)(((e < 4 ? c8.x : c8.y) >> (e & 3) * 8) & 255u), scale_of(vp), minimum_of(vp));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) kv[e] = vv[e] = 0.f;
        }
        store8(y, kv);
        store8(y + a.c.kv_heads * D, vv);
    }
}

static CacheArgs cache_args(const TokenArgs &a, bool read)
{
    CacheArgs b;
    b.x = a.x; b.y = a.y; b.c = a.cache; b.b_lo = a.b_lo; b.S = a.S;
    b.blocks = (a.S + 30) / 32 + 1;                    // blocks that S positions from anywhere on can touch
    b.width = (read ? 2 : a.heads / a.kv_heads + 2) * a.kv_heads * a.D;
    b.k_off = a.heads * a.D;
    return b;
}

LaunchInfo launch_cache_write(const TokenArgs &a, hipStream_t s, bool dry)
{
    const CacheArgs b = cache_args(a, false);
    LaunchInfo li = info(a.dtype == DT_BF16 ? "cache_write_bf16" : "cache_write_f32", (int64_t)(a.b_hi - a.b_lo) * a.kv_heads * b.blocks, 0);
    if (dry || !li.workgroups) return li;
    const dim3 grid(li.workgroups), block(256);
    if (a.dtype == DT_BF16 && a.D == 64) GACER_LAUNCH((cache_write_kernel<unsigned short, 64>), grid, block, 0, s, b);
    else if (a.dtype == DT_BF16) GACER_LAUNCH((cache_write_kernel<unsigned short, 128>), grid, block, 0, s, b);
    else if (a.D == 64) GACER_LAUNCH((cache_write_kernel<float, 64>), grid, block, 0, s, b);
    else GACER_LAUNCH((cache_write_kernel<float, 128>), grid, block, 0, s, b);
    return li;
}

LaunchInfo launch_cache_read(const TokenArgs &a, hipStream_t s, bool dry)
{
    const CacheArgs b = cache_args(a, true);
    LaunchInfo li = info(a.dtype == DT_BF16 ? "cache_read_bf16" : "cache_read_f32", (int64_t)(a.b_hi - a.b_lo) * a.kv_heads * b.blocks, 32 * (a.D + 8));
    if (dry || !li.workgroups) return li;
    const dim3 grid(li.workgroups), block(256);
    if (a.dtype == DT_BF16 && a.D == 64) GACER_LAUNCH((cache_read_kernel<unsigned short, 64>), grid, block, 0, s, b);
    else if (a.dtype == DT_BF16) GACER_LAUNCH((cache_read_kernel<unsigned short, 128>), grid, block, 0, s, b);
    else if (a.D == 64) GACER_LAUNCH((cache_read_kernel<float, 64>), grid, block, 0, s, b);
    else GACER_LAUNCH((cache_read_kernel<float, 128>), grid, block, 0, s, b);
    return li;
}

LaunchInfo launch_tokens(const TokenArgs &a, hipStream_t s, bool dry, int phase)
{
    switch (a.op) {
    case TK_QKNORM_ROPE: return launch_qknorm_rope(a, s, dry);
    case TK_CACHE_WRITE: return launch_cache_write(a, s, dry);
    case TK_CACHE_READ: return launch_cache_read(a, s, dry);
    case TK_CACHE_ATTENTION: return launch_cache_attention(a, s, dry, phase);
    default: return launch_sample(a, s, dry, phase);
    }
}

}  // namespace gacer
