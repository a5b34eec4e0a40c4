// Products of 8-bit rows with 8-bit weights: y[r][o] = act(sum_b sx[r][b] sw[o/128][b] sum_{k in b} x[r][k] w[o][k] + bias[o] + res[r][o]), and the gated block.
//
// Codes are widened to bf16, which holds each of them exactly, and multiplied by the bf16 matrix instruction, whose products and sums are those of 32 bits.
// The 8-bit matrix instructions would be twice as fast, but they line up the eight products of a group by the largest of them and drop what lies 2^-12
// and more below it: an error of 1.5e-5 of the result on bell-shaped rows of 128 (4.8e-5 with an outlier), where this way it is 1e-8.
#include <hip/hip_runtime.h>
#include <algorithm>
#include "fp8.h"
#include "tokens_geom.h"

namespace gacer {

// The end of a product of features f0.. of a row: bias, residual, activation, one rounding.
template <typename T> __device__ __forceinline__ void finish(const Fp8Args &a, int64_t row, int f, float v)
{
    if (a.bias) v += a.bias[f];
    if (a.res) v += ld_f32((const T *)a.res, row * a.N + f);
    st_f32((T *)a.y, row * a.N + f, activate8(v, a.act));
}

// One workgroup of eight waves per tile of 32 rows and 32 features (gated: 16 gate and 16 up features); the waves take the tile's blocks of 128 inner
// features in turn and their sums are added in order.  Operands come straight from memory: lane l holds feature (row) l % 32, and of every
// 32 inner features the 16 codes of half l / 32.
template <typename T, bool GATED> __global__ __launch_bounds__(512) void fp8_few_kernel(Fp8Args a)
{
    constexpr int W = 8, FT = GATED ? 16 : 32;
    __shared__ float red[W][16][65];
    const int tid = threadIdx.x, l = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r = l & 31, half = l >> 5;
    int id = blockIdx.x;
    const int slice = id % a.slices; id /= a.slices;
    const int f0 = (id % a.f_tiles) * FT, r0 = a.r_lo + (id / a.f_tiles) * 32;
    const int row = min(r0 + r, a.r_hi - 1);            // rows and features beyond the end repeat the last one; their results are not stored
    const unsigned char *x = a.x + (int64_t)row * a.K;
    const unsigned char *w = GATED ? (r < 16 ? a.w : a.w2) + (int64_t)min(f0 + (r & 15), a.N - 1) * a.K : a.w + (int64_t)min(f0 + r, a.N - 1) * a.K;
    const float *ws = a.ws + (int64_t)(f0 / FP8_BLOCK) * a.KB, *ws2 = GATED ? a.ws2 + (int64_t)(f0 / FP8_BLOCK) * a.KB : nullptr;
    const int lo = slice * a.per_slice, hi = min(lo + a.per_slice, a.KB);

    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[i] = 0.f;
    for (int kb = lo + wave; kb < hi; kb += W) {
        uint4 xv[4], wv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int k = kb * FP8_BLOCK + 32 * j + 16 * half, at = min(k, a.K - 16);
            wv[j] = *(const uint4 *)(w + at);
            xv[j] = *(const uint4 *)(x + at);
            if (k >= a.K) xv[j] = make_uint4(0, 0, 0, 0);       // behind the end
        }
        const float sx = a.xs[(int64_t)kb * a.rows + row], s = sx * ws[kb], s2 = GATED ? sx * ws2[kb] : s;
        f32x16 p;
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(wv[j].x, wv[j].y), widen(xv[j].x, xv[j].y), p, 0, 0, 0);
            p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(wv[j].z, wv[j].w), widen(xv[j].z, xv[j].w), p, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[i] = fmaf(p[i], GATED && i >= 8 ? s2 : s, acc[i]);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) red[wave][i][l] = acc[i];
    __syncthreads();
    // accumulator i of lane l: feature 8 (i / 4) + 4 (l / 32) + i % 4 of the tile, row l % 32
    auto sum = [&](int f, int row) {
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) v += red[i][(f >> 3) * 4 + (f & 3)][row + 32 * ((f >> 2) & 1)];
        return v;
    };
    const int n = min(32, a.r_hi - r0);
    for (int e = tid; e < FT * n; e += 512) {
        const int f = e % FT, m = e / FT;
        if (f0 + f >= a.N) continue;
        const float v = sum(f, m), u = GATED ? sum(f + 16, m) : 0.f;
        const int64_t at = r0 + m;
        if (a.part) {
            float *p = a.part + ((int64_t)slice * a.rows + at) * a.N * (GATED ? 2 : 1) + f0 + f;
            p[0] = v;
            if (GATED) p[a.N] = u;
        } else if (GATED) st_f32((T *)a.y, at * a.N + f0 + f, activate8(v, a.act) * u);
        else finish<T>(a, at, f0 + f, v);
    }
}

// Adds the slices in order and ends the product: a wave per row and block of 128 features, two neighbouring features a lane.
template <typename T, bool GATED> __global__ __launch_bounds__(256) void fp8_join_kernel(Fp8Args a)
{
    const int l = threadIdx.x & 63, blocks = (a.N + FP8_BLOCK - 1) / FP8_BLOCK;
    const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), row = a.r_lo + id / blocks;
    if (row >= a.r_hi) return;
    const int block = (int)(id % blocks), f = block * FP8_BLOCK + 2 * l;
    const int64_t width = (int64_t)a.N * (GATED ? 2 : 1), step = a.rows * width;
    float v[2] = {0.f, 0.f}, u[2] = {0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        if (f + e >= a.N) continue;
        const float *p = a.part + row * width + f + e;
        for (int i = 0; i < a.slices; ++i) {
            v[e] += p[i * step];
            if (GATED) u[e] += p[i * step + a.N];
        }
    }
    if (!GATED) {
#pragma unroll
        for (int e = 0; e < 2; ++e) if (f + e < a.N) finish<T>(a, row, f + e, v[e]);
        return;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) v[e] = activate8(v[e], a.act) * u[e];
    if (!a.yq) {
#pragma unroll
        for (int e = 0; e < 2; ++e) if (f + e < a.N) st_f32((T *)a.y, row * a.N + f + e, v[e]);
        return;
    }
    unsigned most = max(f < a.N ? magnitude(v[0]) : 0u, f + 1 < a.N ? magnitude(v[1]) : 0u);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) most = max(most, (unsigned)__shfl_xor((int)most, d));
    const float2 s = scale_of_block(most);
    const unsigned c = s.y == 0.f ? 0u : to_codes(v[0], v[1], 0.f, 0.f, s.y);
    if (f < a.N) *(unsigned short *)(a.yq + row * a.N + f) = (unsigned short)c;      // a.N is even here
    if (l == 0) a.ys[(int64_t)block * a.rows + row] = s.x;
}

LaunchInfo launch_gemm_fp8(const TokenArgs &a, hipStream_t s, bool dry, int phase)
{
    const Fp8Geom g = fp8_geom(a);
    const bool gated = a.op == TK_GATED_FP8;
    Fp8Args b;
    b.x = a.xq.codes; b.xs = a.xq.scales; b.w = a.w.codes; b.ws = a.w.scales; b.w2 = a.w2.codes; b.ws2 = a.w2.scales;
    b.bias = a.bias; b.res = a.res; b.y = a.y; b.yq = a.yq.codes; b.ys = a.yq.scales; b.part = g.join ? a.ws : nullptr;
    b.K = a.xq.features; b.KB = (b.K + FP8_BLOCK - 1) / FP8_BLOCK; b.N = a.features; b.rows = a.batch * a.S; b.act = a.act;
    b.r_lo = a.b_lo * a.S; b.r_hi = a.b_hi * a.S;
    b.f_tiles = (b.N + g.features - 1) / g.features; b.r_tiles = (b.r_hi - b.r_lo + 31) / 32; b.slices = g.slices; b.per_slice = g.blocks_per_slice;
    const int64_t units = (int64_t)(b.r_hi - b.r_lo) * ((b.N + FP8_BLOCK - 1) / FP8_BLOCK);
    LaunchInfo li;
    li.workgroups = phase == 2 ? (int)((units + 3) / 4) : (int)((int64_t)b.f_tiles * b.r_tiles * b.slices);
    li.threads = phase == 2 ? 256 : 512; li.lds_bytes = phase == 2 ? 0 : 8 * 16 * 65 * 4; li.wg_per_cu = phase == 2 ? 8 : 4; li.phases = g.join ? 2 : 1;
    li.kernel = phase == 2 ? "fp8_join" : gated ? "gated_fp8" : "gemm_fp8";
    if (dry || b.r_hi <= b.r_lo) return li;
#define BOTH(T, GATED)                                                                                                               \
    do {                                                                                                                             \
        if (phase != 2) GACER_LAUNCH((fp8_few_kernel<T, GATED>), dim3((unsigned)((int64_t)b.f_tiles * b.r_tiles * b.slices)), dim3(512), 0, s, b); \
        if (g.join && phase != 1) GACER_LAUNCH((fp8_join_kernel<T, GATED>), dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, b); \
    } while (0)
    if (a.dtype == DT_BF16) { if (gated) BOTH(unsigned short, true); else BOTH(unsigned short, false); }
    else { if (gated) BOTH(float, true); else BOTH(float, false); }
#undef BOTH
    return li;
}

}  // namespace gacer
