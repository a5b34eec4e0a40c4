// Sampling: one token per row of logits (gacer_sampling in include/gacer.h has the definition).
//
// A workgroup owns a row.  Weights are whole numbers, so every sum is exact and the same in any order.  The entries that the filters keep are
// a prefix of the order "larger first, equal ones by index", described by a key (the logit's bits in an order of unsigned
// numbers) and a number of entries with that key; both top-k (by count) and top-p (by weight) find it digit by digit, eight bits of the key at
// a time, from a histogram in LDS.  The draw halves in on its index by sums over ranges.
#include <hip/hip_runtime.h>
#include "device_util.h"
#include "kernels.h"

namespace gacer {

typedef unsigned long long u64;

struct SampleArgs {
    const void *x;
    int64_t row_lo;
    int V;
    const float *u, *temperature, *top_p, *min_p;
    const int *top_k;
    int *tokens;
    float *logp;
};

// numbers in an order of unsigned integers: -inf and NaN lowest, both zeros alike
__device__ __forceinline__ unsigned key_of(float x)
{
    if (x != x) x = -INFINITY;
    const unsigned b = __float_as_uint(x + 0.f);
    return b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xFFFFFFFFu)); }

template <typename T> struct Row {
    static constexpr int THREADS = 1024, WAVES = THREADS / 64;
    const T *x;
    int V;
    float top, temperature;
    u64 *shared;               // WAVES + 1

    __device__ unsigned key(int i) const { return key_of(ld_f32(x, i)); }
    __device__ float part(unsigned k) const
    {
        const float v = value_of(k);
        return v == top ? 1.f : expf(__fdiv_rn(__fsub_rn(v, top), temperature));
    }
    static __device__ u64 weight(float part) { return (u64)(part * 2147483648.f); }
    __device__ u64 sum(u64 v)
    {
        for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
        __syncthreads();
        if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = v;
        __syncthreads();
        u64 s = 0;
        for (int w = 0; w < WAVES; ++w) s += shared[w];
        return s;
    }
    // The first index at which the sum of f over 0..i exceeds `goal` (goal < sum of all).
    template <typename F> __device__ int locate(u64 goal, F f)
    {
        int lo = 0, hi = V;
        const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
        while (hi - lo > 64) {
            const int per = ((hi - lo + WAVES - 1) / WAVES + 63) & ~63;
            const int a = min(hi, lo + wave * per), b = min(hi, a + per);
            u64 v = 0;
            for (int i = a + lane; i < b; i += 64) v += f(i);
            for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
            __syncthreads();
            if (lane == 0) shared[wave] = v;
            __syncthreads();
            int w = 0;
            while (w < WAVES - 1 && shared[w] <= goal) goal -= shared[w++];
            const int end = hi;
            lo = min(end, lo + w * per);
            hi = min(end, lo + per);
        }
        u64 v = lo + lane < hi ? f(lo + lane) : 0;
        for (int o = 1; o < 64; o <<= 1) {
            const u64 n = __shfl_up(v, o, 64);
            if (lane >= o) v += n;
        }
        return lo + __popcll(__ballot(v <= goal && lo + lane < hi));
    }
};

template <typename T> __global__ __launch_bounds__(1024) void sample_kernel(SampleArgs a)
{
    __shared__ u64 shared[Row<T>::WAVES + 1], bins[256];
    __shared__ unsigned topmost;
    const int tid = threadIdx.x;
    const int64_t r = a.row_lo + blockIdx.x;
    Row<T> row = {(const T *)a.x + r * a.V, a.V, 0.f, 1.f, shared};
    if (tid == 0) topmost = 0u;
    __syncthreads();
    unsigned best = 0u;
    for (int i = tid; i < a.V; i += 1024) best = max(best, row.key(i));
    atomicMax(&topmost, best);
    __syncthreads();
    const unsigned none = key_of(-INFINITY), peak = topmost;
    if (peak <= none) {
        if (tid == 0) {
            a.tokens[r] = -1;
            if (a.logp) a.logp[r] = -INFINITY;
        }
        return;
    }
    row.top = value_of(peak);
    row.temperature = a.temperature ? a.temperature[r] : 1.f;
    const float top_p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f;
    int top_k = a.top_k ? a.top_k[r] : 0;
    if (!(row.temperature > 0.f) || !(top_p > 0.f) || !(min_p <= 1.f)) top_k = 1;
    if (top_k <= 0 || top_k > a.V) top_k = a.V;

    // kept: keys above `cut`, and the first `ties` entries (by index, up to `last`) with that key
    unsigned cut = 0u;
    int last = a.V;
    for (int pass = 0; pass < 2; ++pass) {
        const bool by_weight = pass == 1;
        if (by_weight ? !(top_p < 1.f) || top_k == 1 : top_k == a.V) continue;
        auto measure = [&](int i, unsigned k) -> u64 {
            if (!by_weight) return 1;
            return k > cut || (k == cut && i <= last) ? Row<T>::weight(row.part(k)) : 0;
        };
        double reach = (double)top_k;
        if (by_weight) {
            u64 v = 0;
            for (int i = tid; i < a.V; i += 1024) v += measure(i, row.key(i));
            reach = (double)top_p * (double)row.sum(v);
        }
        u64 before = 0;                              // measure of the keys above the digits found so far
        unsigned prefix = 0u;
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            if (tid < 256) bins[tid] = 0;
            __syncthreads();
            for (int i = tid; i < a.V; i += 1024) {
                const unsigned k = row.key(i);
                if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) {
                    const u64 m = measure(i, k);
                    if (m) atomicAdd(&bins[(k >> shift) & 255u], m);
                }
            }
            __syncthreads();
            int digit = 255;
            for (; digit > 0 && (double)(before + bins[digit]) < reach; --digit) before += bins[digit];
            prefix |= (unsigned)digit << shift;
        }
        // entries of this very key that the prefix still takes, one by one
        const u64 each = by_weight ? Row<T>::weight(row.part(prefix)) : 1;
        u64 ties = 1;
        if (each) {
            const double more = reach - (double)before;
            ties = (u64)(more / (double)each);
            while ((double)(before + ties * each) < reach) ++ties;
            while (ties > 1 && (double)(before + (ties - 1) * each) >= reach) --ties;
        }
        u64 equal = 0;
        const unsigned old_cut = cut;
        const int old_last = last;
        auto same = [&](int i) -> u64 { return row.key(i) == prefix && (prefix > old_cut || i <= old_last); };
        for (int i = tid; i < a.V; i += 1024) equal += same(i);
        equal = row.sum(equal);
        last = ties < equal ? row.locate(ties - 1, same) : (prefix > old_cut ? a.V : old_last);
        cut = prefix;
    }
    auto kept = [&](int i) -> u64 {
        const unsigned k = row.key(i);
        if (k < cut || (k == cut && i > last) || k <= none) return 0;
        const float part = row.part(k);
        return part >= min_p || top_k == 1 ? Row<T>::weight(part) : 0;
    };
    u64 total = 0;
    for (int i = tid; i < a.V; i += 1024) total += kept(i);
    total = row.sum(total);
    const double goal = floor((double)a.u[r] * (double)total);
    const u64 g = goal > 0. ? (goal >= (double)total ? total - 1 : (u64)goal) : 0;
    const int token = row.locate(g, kept);
    if (tid == 0) {
        a.tokens[r] = token;
        if (a.logp) {
            const float v = value_of(row.key(token));
            a.logp[r] = (v == row.top ? 0.f : __fdiv_rn(__fsub_rn(v, row.top), row.temperature)) - logf((float)total * 0x1p-31f);
        }
    }
}

LaunchInfo launch_sample(const TokenArgs &a, hipStream_t s, bool dry, int)
{
    SampleArgs b;
    b.x = a.x; b.row_lo = (int64_t)a.b_lo * a.S; b.V = a.vocab; b.u = a.u; b.temperature = a.temperature; b.top_p = a.top_p; b.min_p = a.min_p;
    b.top_k = a.top_k; b.tokens = a.tokens; b.logp = a.logp;
    LaunchInfo li;
    li.workgroups = (a.b_hi - a.b_lo) * a.S;
    li.threads = 1024; li.lds_bytes = 2304; li.wg_per_cu = 2; li.kernel = a.dtype == DT_BF16 ? "sample_bf16" : "sample_f32"; li.phases = 1;
    if (dry || !li.workgroups) return li;
    if (a.dtype == DT_BF16) GACER_LAUNCH(sample_kernel<unsigned short>, dim3(li.workgroups), dim3(1024), 0, s, b);
    else GACER_LAUNCH(sample_kernel<float>, dim3(li.workgroups), dim3(1024), 0, s, b);
    return li;
}

}  // namespace gacer
