// Residual, RMS norm and 8-bit rows: h = x + res, y = h * rsqrt(mean(h^2) + eps) * gamma, then e4m3 codes with a scale for each row and block of 128 features.
//
// Every element is read and written once, the row in between in registers: bound by the way to memory.  4101 rows of 4096 features, bf16, with residual (118 MB):
// 25.3 us = 4.7 TB/s; codes alone of 8192 rows of 8192 (203 MB) 39.4 us = 5.1 TB/s, what a large copy reaches; 1018 rows of 5008 in fp32 8.3 us, one row 5.3, of which a
// launch in a stream of launches is 4.  With the loads under conditions, each waited for where it stood, they took 47, 54 and 16 us.
#include <hip/hip_runtime.h>
#include <algorithm>
#include "fp8.h"

namespace gacer {

struct NormArgs {
    const void *x, *res;
    const float *gamma;
    void *y;
    unsigned char *codes;
    float *scales;
    float eps, inv_c;
    int C, norm, rows;                 // rows: of the whole operator (stride of the scales)
    int r_lo, r_hi;
};

// Eight features as they lie in memory, behind a row's end zeros.  WHOLE: rows of a multiple of eight features, aligned vectors; otherwise one by one.
template <typename T, bool WHOLE> struct Run;
template <> struct Run<unsigned short, true> {
    uint4 v;
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t row, int f) { v = buf_load16(row, f * 2); }
    __device__ __forceinline__ float get(int e) const
    {
        const unsigned w = e / 2 == 0 ? v.x : e / 2 == 1 ? v.y : e / 2 == 2 ? v.z : v.w;
        return __uint_as_float(e % 2 ? w & 0xFFFF0000u : w << 16);
    }
};
template <> struct Run<float, true> {
    uint4 a, b;
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t row, int f) { a = buf_load16(row, f * 4); b = buf_load16(row, f * 4 + 16); }
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(e == 0 ? a.x : e == 1 ? a.y : e == 2 ? a.z : e == 3 ? a.w : e == 4 ? b.x : e == 5 ? b.y : e == 6 ? b.z : b.w); }
};
template <typename T> struct Run<T, false> {
    T v[8];
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t row, int f)
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = buf_load1<T>(row, (f + e) * (int)sizeof(T));
    }
    __device__ __forceinline__ float get(int e) const { return ld_f32(&v[e], 0); }
};
template <typename T, bool WHOLE> __device__ __forceinline__ void store(T *row, int f, int C, const float *v)
{
    if constexpr (WHOLE) {
        if (f < C) store8(row + f, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) if (f + e < C) st_f32(row, f + e, v[e]);
    }
}

// A row is held by LANES threads in registers, R runs of eight features each; 16 neighbouring lanes hold a block of 128.  All loads of a row are issued, through
// descriptors that answer zeros behind the row, before the first is converted: under a condition each would be waited for where it stands.
// LONG: a row that the registers do not fit goes through them in pieces of LANES * R * 8 features, with a norm twice; the second time it comes from the caches.
template <typename T, int LANES, int R, bool WHOLE, bool LONG> __global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rmsnorm_fp8_kernel(NormArgs a)
{
    constexpr int THREADS = LANES < 256 ? 256 : LANES, PER = THREADS / LANES, PIECE = LANES * R * 8;
    __shared__ float sums[LANES > 64 ? LANES / 64 : 1];
    const int tid = threadIdx.x, lane = tid % LANES;
    const __amdgpu_buffer_rsrc_t gr = make_rsrc(a.gamma, a.gamma ? a.C * 4 : 0);
    for (int64_t row = a.r_lo + (int64_t)blockIdx.x * PER + tid / LANES; row < a.r_hi; row += (int64_t)gridDim.x * PER) {
        const __amdgpu_buffer_rsrc_t xr = make_rsrc((const T *)a.x + row * a.C, a.C * (int64_t)sizeof(T));
        float h[R][8];
        auto fetch = [&](int from) {
            Run<T, WHOLE> x[R], r[R];
#pragma unroll
            for (int i = 0; i < R; ++i) x[i].load(xr, from + (i * LANES + lane) * 8);
            if (a.res) {
                const __amdgpu_buffer_rsrc_t rr = make_rsrc((const T *)a.res + row * a.C, a.C * (int64_t)sizeof(T));
#pragma unroll
                for (int i = 0; i < R; ++i) r[i].load(rr, from + (i * LANES + lane) * 8);
            }
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) h[i][e] = x[i].get(e);
            if (a.res) {
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) h[i][e] += r[i].get(e);
            }
        };
        auto keep = [&](int from) {                        // in the tenant's type
#pragma unroll
            for (int i = 0; i < R; ++i) store<T, WHOLE>((T *)a.y + row * a.C, from + (i * LANES + lane) * 8, a.C, h[i]);
        };
        Run<float, WHOLE> g[R];
        auto fetch_gamma = [&](int from) {
            if (!a.gamma) return;
#pragma unroll
            for (int i = 0; i < R; ++i) g[i].load(gr, from + (i * LANES + lane) * 8);
        };
        float sum = 0.f;
        auto squares = [&] {
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(h[i][e], h[i][e], sum);
        };
        float by = 1.f;
        auto factor = [&] {
#pragma unroll
            for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
            if constexpr (LANES > 64) {
                if (tid % 64 == 0) sums[tid / 64] = sum;
                __syncthreads();
                sum = 0.f;
#pragma unroll
                for (int i = 0; i < LANES / 64; ++i) sum += sums[i];
                if (gridDim.x * PER < a.r_hi - a.r_lo) __syncthreads();      // another row follows
            }
            by = rsqrtf(sum * a.inv_c + a.eps);
        };
        auto leave = [&](int from) {
            if (a.norm) {
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) h[i][e] = h[i][e] * by * (a.gamma ? g[i].get(e) : 1.f);
            }
            if (!a.codes) {
                keep(from);
                return;
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {                  // codes: rows of a multiple of 16 features
                const int f = from + (i * LANES + lane) * 8;
                unsigned most = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) most = max(most, magnitude(h[i][e]));
#pragma unroll
                for (int d = 1; d < 16; d *= 2) most = max(most, (unsigned)__shfl_xor((int)most, d));
                const float2 s = scale_of_block(most);
                uint2 c = make_uint2(to_codes(h[i][0], h[i][1], h[i][2], h[i][3], s.y), to_codes(h[i][4], h[i][5], h[i][6], h[i][7], s.y));
                if (s.y == 0.f) c = make_uint2(0, 0);
                if (f < a.C) {
                    *(uint2 *)(a.codes + row * a.C + f) = c;
                    if (lane % 16 == 0) a.scales[(int64_t)(f / FP8_BLOCK) * a.rows + row] = s.x;
                }
            }
        };
        if constexpr (!LONG) {
            fetch(0);
            if (a.codes && a.y) keep(0);
            if (a.norm) {
                fetch_gamma(0);
                squares();
                factor();
            }
            leave(0);
        } else {
            if (a.norm) {
                for (int from = 0; from < a.C; from += PIECE) {
                    fetch(from);
                    squares();
                }
                factor();
            }
            for (int from = 0; from < a.C; from += PIECE) {
                fetch(from);
                if (a.norm) fetch_gamma(from);
                if (a.codes && a.y) keep(from);
                leave(from);
            }
        }
    }
}

template <typename T, int LANES, int R, bool LONG> static void norm(const NormArgs &a, int grid, hipStream_t s)
{
    const dim3 g(grid), b(LANES < 256 ? 256 : LANES);
    if (a.C % 8 == 0) GACER_LAUNCH((rmsnorm_fp8_kernel<T, LANES, R, true, LONG>), g, b, 0, s, a);
    else GACER_LAUNCH((rmsnorm_fp8_kernel<T, LANES, R, false, LONG>), g, b, 0, s, a);
}

LaunchInfo launch_rmsnorm_fp8(const TokenArgs &a, hipStream_t s, bool dry)
{
    NormArgs n;
    n.x = a.x; n.res = a.res; n.gamma = a.gamma; n.y = a.y; n.codes = a.yq.codes; n.scales = a.yq.scales;
    n.eps = a.eps; n.C = a.features; n.inv_c = 1.f / (float)a.features; n.norm = a.norm; n.rows = a.batch * a.S;
    n.r_lo = a.b_lo * a.S; n.r_hi = a.b_hi * a.S;
    // lanes of a row: a wave up to 1024 features, four up to 8192, else sixteen.  Measured, us with 64 / 256 / 1024 lanes, codes and sum with residual, buffers of 1.5 GB in
    // turn, so that the last-level cache holds none (the same ones again take up to 25 % less): bf16 8192 rows of 512 9.2 / 14.4 / 43, of 1024 14.9 / 17.5 / 45, of 1536
    // 21.1 / 21.2 / 46, 4101 of 4096 30.4 / 26.3 / 30.5, 2048 of 8192 - / 27.6 / 26.8, of 12288 - / 44 / 41, 1000 of 16384 - / 30.4 / 29.5; fp32 8192 of 1024 25.1 / 26.7 / 62, of
    // 1536 35.4 / 32.9 / 66, 4101 of 4096 51 / 44.5 / 50, 2048 of 8192 - / 45.7 / 44.2, of 12288 - / 68 / 75, 1000 of 16384 - / 49.4 / 48.0.  Beyond 16384 features in pieces, us whole (in
    // registers and, from 65536 on, scratch memory) / in pieces: bf16 500 rows of 65536 113 / 68, one row 32 / 14, 500 of 32768 30 / 35, 2000 of 32768 99 / 117; fp32 200 / 120, 54 / 21,
    // 48 / 60, 172 / 216; a product's inner extent of that size is rare, and one kernel does them all.
    const int runs = (a.features + 7) / 8, lanes = runs <= 128 ? 64 : runs <= 1024 ? 256 : 1024;
    const int per = lanes == 64 ? 4 : 1, each = (runs + lanes - 1) / lanes;
    // workgroups that a unit holds, by the registers of (64, 1), (64, 2), (256, 1), (256, 2), (256, 4) and wider
    static const int held[2][2][6] = {{{8, 6, 8, 5, 3, 1}, {8, 7, 8, 7, 4, 1}}, {{8, 4, 8, 4, 2, 1}, {8, 8, 8, 7, 4, 1}}};
    LaunchInfo li;
    li.workgroups = (int)std::min<int64_t>(((int64_t)(n.r_hi - n.r_lo) + per - 1) / per, 1 << 20);
    li.threads = std::max(256, lanes); li.lds_bytes = lanes == 64 ? 0 : lanes / 16; li.phases = 1;
    li.wg_per_cu = held[a.dtype == DT_BF16][a.features % 8 == 0][lanes == 64 ? each - 1 : lanes == 256 ? (each > 2 ? 4 : each + 1) : 5];
    li.kernel = a.dtype == DT_BF16 ? "rmsnorm_fp8_bf16" : "rmsnorm_fp8_f32";
    if (dry || !li.workgroups) return li;
#define NORM(LANES, R, LONG) if (lanes == LANES && (LONG ? each > R : each > R / 2 && each <= R)) { if (a.dtype == DT_BF16) norm<unsigned short, LANES, R, LONG>(n, li.workgroups, s); else norm<float, LANES, R, LONG>(n, li.workgroups, s); }
    NORM(64, 1, false) NORM(64, 2, false) NORM(256, 1, false) NORM(256, 2, false) NORM(256, 4, false) NORM(1024, 2, false) NORM(1024, 2, true)
#undef NORM
    return li;
}

}  // namespace gacer
