// What the operators on 8-bit rows share: codes to operands and back, activations, the end of a product.
#pragma once
#include "device_util.h"

namespace gacer {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

static constexpr float FP8_LEAST = 0x1p-60f, FP8_LARGEST = 448.f;

// Eight e4m3 codes as bf16, which holds each of them exactly.
__device__ __forceinline__ bf16x8 widen(unsigned lo, unsigned hi)
{
    uint4 v;
    v.x = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
    v.y = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
    v.z = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
    v.w = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
    return __builtin_bit_cast(bf16x8, v);
}

// Four values times `inv` as e4m3 codes, rounded to nearest even.
__device__ __forceinline__ unsigned to_codes(float a, float b, float c, float d, float inv)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, w, true);
}

// A block's scale and the factor of its values, from the largest magnitude as bits (whole numbers keep a NaN the largest): (NaN, 0) where that is no number.
__device__ __forceinline__ float2 scale_of_block(unsigned most)
{
    const float m = __builtin_fmaxf(__uint_as_float(most), FP8_LEAST);
    return most >= 0x7F800000u ? make_float2(__uint_as_float(0x7FC00000u), 0.f) : make_float2(m / FP8_LARGEST, FP8_LARGEST / m);
}
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// The activations of products, `act` uniform.  A row or block that is no number has to stay none: the bounds of ReLU and the hard activations are comparisons, which
// keep a NaN (the maximum and the median that activate() takes return a bound for it) and give the same bits for every number.
__device__ __forceinline__ float between(float v, float most) { return v <= 0.f ? 0.f : v >= most ? most : v; }
__device__ __forceinline__ float activate8(float v, int act)
{
    if (act == ACT_RELU) return v <= 0.f ? 0.f : v;
    if (act == ACT_RELU6) return between(v, 6.f);
    if (act == ACT_HSWISH || act == ACT_HSIGMOID) {
        const float s = __fmul_rn(between(__fadd_rn(v, 3.f), 6.f), 0.16666667163372039794921875f);
        return act == ACT_HSWISH ? __fmul_rn(v, s) : s;
    }
    if (act == ACT_SILU) return v / (1.f + __expf(-v));
    if (act == ACT_GELU_TANH) return v / (1.f + __expf(-1.5957691216057308f * (v + 0.044715f * v * v * v)));
    return activate(v, act);
}

__device__ __forceinline__ void store4(float *p, const float *v) { *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store4(unsigned short *p, const float *v) { *(uint2 *)p = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])); }

__device__ __forceinline__ void store8(float *p, const float *v) { store4(p, v); store4(p + 4, v + 4); }
__device__ __forceinline__ void store8(unsigned short *p, const float *v) { *(uint4 *)p = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])); }
__device__ __forceinline__ void load8(const float *p, float *v)
{
    const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
__device__ __forceinline__ void load8(const unsigned short *p, float *v)
{
    const Vec<unsigned short, 8> r = ld_vec<unsigned short, 8>(p, 0);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = r.get(e);
}

// N values at once: one (uniform) branch for all of them.
template <int N, int ACT> __device__ __forceinline__ void activate8_all(float *v)
{
#pragma unroll
    for (int q = 0; q < N; ++q) v[q] = activate8(v[q], ACT);
}
template <int N> __device__ __forceinline__ void activate8_n(float *v, int act)
{
    if (act == ACT_NONE) return;
    if (act == ACT_SILU) activate8_all<N, ACT_SILU>(v);
    else if (act == ACT_GELU_TANH) activate8_all<N, ACT_GELU_TANH>(v);
    else if (act == ACT_GELU) activate8_all<N, ACT_GELU>(v);
    else if (act == ACT_RELU) activate8_all<N, ACT_RELU>(v);
    else if (act == ACT_RELU6) activate8_all<N, ACT_RELU6>(v);
    else if (act == ACT_HSWISH) activate8_all<N, ACT_HSWISH>(v);
    else activate8_all<N, ACT_HSIGMOID>(v);
}

// The two scales of a block's sums.  Their product does for both, but where it leaves the range or loses bits below 2^-126: there it would turn sums of 0 into NaN and
// small results into rough ones, and the scales are taken one after the other, the larger first.  (A product below 2^-150, or of a scale of 0, is 0.)  Which way a row
// goes is up to its own scales, so that it has the same bits whichever rows lie beside it.
static constexpr int CLASS_ODD = 0x294;                      // bits of the class instruction: infinite or subnormal, either sign
__device__ __forceinline__ float2 factors(float a, float b)
{
    if (!__builtin_amdgcn_classf(a * b, CLASS_ODD)) return make_float2(1.f, a * b);
    return __builtin_fabsf(a) > __builtin_fabsf(b) ? make_float2(a, b) : make_float2(b, a);
}
// Lanes whose product is such a one (the builtin beneath a ballot would become a number a lane first, then a mask again).
__device__ __forceinline__ uint64_t odd_lanes(float product)
{
    uint64_t lanes;
    asm("v_cmp_class_f32_e64 %0, %1, %2" : "=s"(lanes) : "v"(product), "s"(CLASS_ODD));
    return lanes;
}

// Arguments of the products (see gacer_fp8_gemm, gacer_fp8_gated)
struct Fp8Args {
    const unsigned char *x, *w, *w2;
    const float *xs, *ws, *ws2;
    const float *bias;
    const void *res;
    void *y;
    unsigned char *yq;
    float *ys, *part;
    int K, KB, N, rows, r_lo, r_hi, act;     // KB: blocks of K; rows: of the whole operator; r_lo..r_hi: of this launch
    int f_tiles, r_tiles, slices, per_slice; // tiles of this launch; slices of K of per_slice blocks
    int whole;                               // tiles that are not done in halves
};

}  // namespace gacer
