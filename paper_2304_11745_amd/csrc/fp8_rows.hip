// Residual, RMS norm and 8-bit rows: h = x + res, y = h * rsqrt(mean(h^2) + eps) * gamma, then e4m3 codes with a scale for each row and block of 128 features.
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

// eight values from p on, of which `n` are there
template <bool WHOLE> __device__ __forceinline__ void load8(const float *p, int n, float *v)
{
    if constexpr (WHOLE) {
        if (n >= 8) {
            load8(p, v);
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? p[e] : 0.f;
}
template <bool WHOLE> __device__ __forceinline__ void load8(const unsigned short *p, int n, float *v)
{
    if constexpr (WHOLE) {
        if (n >= 8) {
            load8(p, v);
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? ld_f32(p, e) : 0.f;
}
template <bool WHOLE> __device__ __forceinline__ void store8(float *p, int n, const float *v)
{
    if (WHOLE && n >= 8) {
        store8(p, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < n) p[e] = v[e];
}
template <bool WHOLE> __device__ __forceinline__ void store8(unsigned short *p, int n, const float *v)
{
    if (WHOLE && n >= 8) {
        store8(p, v);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) if (e < n) p[e] = to_bf16(v[e]);
}

// A row is held by LANES threads in registers, R runs of eight features each; 16 neighbouring lanes hold a block of 128.  WHOLE: rows of a
// multiple of eight features, whose runs are aligned vectors.
template <typename T, int LANES, int R, bool WHOLE> __global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rmsnorm_fp8_kernel(NormArgs a)
{
    constexpr int THREADS = LANES < 256 ? 256 : LANES, PER = THREADS / LANES;
    __shared__ float sums[LANES > 64 ? LANES / 64 : 1];
    const int tid = threadIdx.x, lane = tid % LANES;
    for (int64_t row = a.r_lo + (int64_t)blockIdx.x * PER + tid / LANES; row < a.r_hi; row += (int64_t)gridDim.x * PER) {
        const T *x = (const T *)a.x + row * a.C, *res = a.res ? (const T *)a.res + row * a.C : nullptr;
        float h[R][8];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int f = (i * LANES + lane) * 8;
            load8<WHOLE>(x + f, a.C - f, h[i]);
        }
        if (res) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int f = (i * LANES + lane) * 8;
                float r[8];
                load8<WHOLE>(res + f, a.C - f, r);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[i][e] += r[e];
            }
        }
        if (a.codes && a.y) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int f = (i * LANES + lane) * 8;
                store8<WHOLE>((T *)a.y + row * a.C + f, a.C - f, h[i]);
            }
        }
        if (a.norm) {
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(h[i][e], h[i][e], sum);
#pragma unroll
            for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
            if constexpr (LANES > 64) {
                if (tid % 64 == 0) sums[tid / 64] = sum;
                __syncthreads();
                sum = 0.f;
#pragma unroll
                for (int i = 0; i < LANES / 64; ++i) sum += sums[i];
                __syncthreads();
            }
            const float by = 1.f / sqrtf(sum * a.inv_c + a.eps);
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int f = (i * LANES + lane) * 8;
                float g[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
                if (a.gamma) load8<false>(a.gamma + f, a.C - f, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[i][e] = h[i][e] * by * g[e];
            }
        }
        if (!a.codes) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int f = (i * LANES + lane) * 8;
                store8<WHOLE>((T *)a.y + row * a.C + f, a.C - f, h[i]);
            }
            continue;
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int f = (i * LANES + lane) * 8;
            unsigned most = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, f + e < a.C ? magnitude(h[i][e]) : 0u);
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
    }
}

template <typename T, int LANES, int R> static void norm(const NormArgs &a, int grid, hipStream_t s)
{
    const dim3 g(grid), b(LANES < 256 ? 256 : LANES);
    if (a.C % 8 == 0) GACER_LAUNCH((rmsnorm_fp8_kernel<T, LANES, R, true>), g, b, 0, s, a);
    else GACER_LAUNCH((rmsnorm_fp8_kernel<T, LANES, R, false>), g, b, 0, s, a);
}

LaunchInfo launch_rmsnorm_fp8(const TokenArgs &a, hipStream_t s, bool dry)
{
    NormArgs n;
    n.x = a.x; n.res = a.res; n.gamma = a.gamma; n.y = a.y; n.codes = a.yq.codes; n.scales = a.yq.scales;
    n.eps = a.eps; n.C = a.features; n.inv_c = 1.f / (float)a.features; n.norm = a.norm; n.rows = a.batch * a.S;
    n.r_lo = a.b_lo * a.S; n.r_hi = a.b_hi * a.S;
    const int runs = (a.features + 7) / 8, lanes = runs <= 128 ? 64 : runs <= 2048 ? 256 : 1024;
    const int per = lanes == 64 ? 4 : 1, each = (runs + lanes - 1) / lanes;
    LaunchInfo li;
    li.workgroups = (int)std::min<int64_t>(((int64_t)(n.r_hi - n.r_lo) + per - 1) / per, 1 << 20);
    li.threads = std::max(256, lanes); li.lds_bytes = 0; li.wg_per_cu = 1; li.phases = 1;
    li.kernel = a.dtype == DT_BF16 ? "rmsnorm_fp8_bf16" : "rmsnorm_fp8_f32";
    if (dry || !li.workgroups) return li;
#define NORM(LANES, R) if (lanes == LANES && each > R / 2 && each <= R) { if (a.dtype == DT_BF16) norm<unsigned short, LANES, R>(n, li.workgroups, s); else norm<float, LANES, R>(n, li.workgroups, s); }
    NORM(64, 1) NORM(64, 2) NORM(256, 1) NORM(256, 2) NORM(256, 4) NORM(256, 8) NORM(1024, 4) NORM(1024, 8)
#undef NORM
    return li;
}

}  // namespace gacer
