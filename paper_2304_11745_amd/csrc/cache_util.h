// Device helpers of the operators on a paged 4-bit cache (gacer_cache in include/gacer.h has the layout).
#pragma once
#include "device_util.h"
#include "kernels.h"

namespace gacer {

// A sequence's part of a call: `start` tokens before it, `count` new ones; out of range on the device: none.
struct Span { int start, count; };
// an integer that nothing writes while the kernel runs: where the index is uniform it comes through the scalar cache
__device__ __forceinline__ int fixed_int(const int *p, int64_t i) { return ((const __attribute__((address_space(4))) int *)(uintptr_t)p)[i]; }
__device__ __forceinline__ Span span_of(const CacheView &c, int b, int S)
{
    Span s = {fixed_int(c.start, b), S};
    if (c.count) s.count = max(0, min(fixed_int(c.count, b), S));
    if (s.start < 0 || s.start > c.max_pages << c.page_shift) s = {0, 0};
    return s;
}

// Page of position p of sequence b, -1 where there is none; p >= 0.
__device__ __forceinline__ int page_of(const CacheView &c, int b, int p)
{
    const int i = p >> c.page_shift;
    if (i >= c.max_pages) return -1;
    const int page = c.page_table[(int64_t)b * c.max_pages + i];
    return (unsigned)page < (unsigned)c.n_pages ? page : -1;
}

// First token row of a page's kv head: rows are D / 2 bytes of codes and D / 64 words of scales, for keys and for values alike.
__device__ __forceinline__ int64_t page_row(const CacheView &c, int page, int kv_head) { return ((int64_t)page * c.kv_heads + kv_head) << c.page_shift; }

// Bit at which element e of a code word starts: elements 2i and 2i + 1 stand in the two halves, so that one shift and one mask give
// both at the same place of a pair of 16-bit numbers.
__device__ __forceinline__ constexpr int code_shift(int e) { return (e >> 1) * 4 + (e & 1) * 16; }

__device__ __forceinline__ float scale_of(unsigned pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float minimum_of(unsigned pair) { return __uint_as_float(pair & 0xFFFF0000u); }

// eight consecutive elements as floats, and back (16-byte aligned)
__device__ __forceinline__ void load8(const float *p, float *v)
{
    const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const unsigned short *p, float *v)
{
    Vec<unsigned short, 8> x;
    x.raw = *(const uint4 *)p;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x.get(i);
}
__device__ __forceinline__ void store8(float *p, const float *v)
{
    *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
    *(float4 *)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(unsigned short *p, const float *v)
{
    Vec<unsigned short, 8> x;
    x.pack(v);
    *(uint4 *)p = x.raw;
}

}  // namespace gacer
