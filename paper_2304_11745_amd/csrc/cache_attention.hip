// Attention of new tokens over a paged 4-bit cache.  One wave per query row: a lane scores one key at a time with the queries in LDS, the
// running maximum and sum of the softmax are per wave, and each lane keeps D / 64 features of the result.
#include <hip/hip_runtime.h>
#include "cache_util.h"
#include "kernels.h"
#include "tokens_geom.h"

namespace gacer {

struct AttendArgs {
    const void *x;
    void *y;
    CacheView c;
    int b_lo, S, heads, per_kv, window;
    float alpha;
};

template <typename T, int D> __global__ __launch_bounds__(64) void cache_attention_rows_kernel(AttendArgs a)
{
    constexpr int NG = D / CACHE_GROUP;
    __shared__ float q[D], p[64];
    __shared__ int at[64];
    const int lane = threadIdx.x, h = blockIdx.x % a.heads, g = h / a.per_kv;
    const int64_t row = (int64_t)blockIdx.x / a.heads;
    const int b = a.b_lo + (int)(row / a.S), t = (int)(row % a.S);
    const Span span = span_of(a.c, b, a.S);
    const T *x = (const T *)a.x + ((int64_t)b * a.S + t) * (a.heads + 2 * a.c.kv_heads) * D + h * D;
    T *y = (T *)a.y + (((int64_t)b * a.S + t) * a.heads + h) * D;
    for (int i = lane; i < D; i += 64) q[i] = ld_f32(x, i);
    const int pos = span.start + t, first = a.window > 0 ? max(0, pos - a.window + 1) : 0;
    float acc[NG] = {}, m = -INFINITY, l = 0.f;
    for (int j0 = first & ~63; t < span.count && j0 <= pos; j0 += 64) {
        __syncthreads();
        const int j = j0 + lane, page = j >= first && j <= pos ? page_of(a.c, b, j) : -1;
        const int64_t r = page < 0 ? 0 : page_row(a.c, page, g) + (j & ((1 << a.c.page_shift) - 1));
        float s = -INFINITY;
        if (page >= 0) {
            s = 0.f;
            for (int w = 0; w < D / 8; ++w) {
                const unsigned word = ((const unsigned *)a.c.k_codes)[r * (D / 8) + w], kp = a.c.k_scales[r * NG + w / 8];
                for (int e = 0; e < 8; ++e) s = fmaf(q[w * 8 + e], fmaf((float)((word >> code_shift(e)) & 15u), scale_of(kp), minimum_of(kp)), s);
            }
            s *= a.alpha;
        }
        float top = s;
        for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
        const float now = fmaxf(m, top);
        if (now == -INFINITY) continue;
        const float scale = expf(m - now), e = expf(s - now);
        float sum = e;
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        l = l * scale + sum;
        m = now;
        p[lane] = e;
        at[lane] = page < 0 ? -1 : page;
        __syncthreads();
        for (int i = 0; i < NG; ++i) acc[i] *= scale;
        for (int k = 0; k < 64; ++k) {
            if (at[k] < 0) continue;
            const int64_t base = page_row(a.c, at[k], g), o = (j0 + k) & ((1 << a.c.page_shift) - 1);
            for (int i = 0; i < NG; ++i) {
                const unsigned word = ((const unsigned *)a.c.v_codes)[(base + (o & ~31)) * (D / 8) + (i * 64 + lane) * 4 + ((o & 31) >> 3)];
                const unsigned vp = a.c.v_scales[(base + o) * NG + i];
                acc[i] = fmaf(p[k], fmaf((float)((word >> code_shift(o & 7)) & 15u), scale_of(vp), minimum_of(vp)), acc[i]);
            }
        }
    }
    for (int i = 0; i < NG; ++i) st_f32(y, i * 64 + lane, l > 0.f ? acc[i] / l : 0.f);
}

LaunchInfo launch_cache_attention(const TokenArgs &a, hipStream_t s, bool dry, int)
{
    AttendArgs b;
    b.x = a.x; b.y = a.y; b.c = a.cache; b.b_lo = a.b_lo; b.S = a.S; b.heads = a.heads; b.per_kv = a.heads / a.kv_heads;
    b.window = a.window; b.alpha = a.alpha;
    LaunchInfo li;
    li.workgroups = (a.b_hi - a.b_lo) * a.S * a.heads;
    li.threads = 64; li.lds_bytes = 1024; li.wg_per_cu = 32; li.kernel = a.dtype == DT_BF16 ? "cache_attention_bf16" : "cache_attention_f32"; li.phases = 1;
    if (dry || !li.workgroups) return li;
    const dim3 grid(li.workgroups), block(64);
    if (a.dtype == DT_BF16 && a.D == 64) GACER_LAUNCH((cache_attention_rows_kernel<unsigned short, 64>), grid, block, 0, s, b);
    else if (a.dtype == DT_BF16) GACER_LAUNCH((cache_attention_rows_kernel<unsigned short, 128>), grid, block, 0, s, b);
    else if (a.D == 64) GACER_LAUNCH((cache_attention_rows_kernel<float, 64>), grid, block, 0, s, b);
    else GACER_LAUNCH((cache_attention_rows_kernel<float, 128>), grid, block, 0, s, b);
    return li;
}

}  // namespace gacer
