// What the attention operators over a paged cache share: how fp32 numbers go into the matrix cores, and small helpers.
#pragma once
#include "spd_device.h"

namespace spda {
using namespace spdd;

constexpr float SLACK = 3.f;                     // a row's reference is raised when a probability would pass 2^3: seldom after the first turns
constexpr float FAR = 0x1p20f;                   // scores (base 2) from which on an exponent is formed from the rounded score

typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef unsigned long long u64;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// exp2(a - b) with exp2(-inf - anything) = 0, also where b is -inf (nothing seen yet).
__device__ __forceinline__ float exp2_below(float a, float b) { return __builtin_amdgcn_exp2f(a - (b == -INFINITY ? 0.f : b)); }

// PARTS: numbers of the cache's type that stand for one fp32 number.
// Probabilities are exp2(score - reference + P_BITS) P_SCALE.  fp16: at most 2^15 then, and two fp16 numbers hold them to 2^-37 of the reference (sixty
// thousand keys may be off by 2^-21 of the sum together); values of at most 2^16 stay far below fp32's end.  (The exponent of some twelve is off by 2^-21: a
// factor behind the exponential would be one instruction of ten per key.  Values that are subnormal fp16 numbers lose bits in the matrix cores, 2^-37 at most.)
// The other types have fp32's range, and values up to its end: scaled down, 2^21 keys of them add up to no infinity, and what small values lose is fp32's
// gradual underflow, 2^-126 at most (measured: 4e-7 of values of 2^-100, 3e-6 of 2^-106).
template <typename KT> struct Type;
template <> struct Type<half_t> { static constexpr int PARTS = 2; static constexpr float P_BITS = 12.f, P_SCALE = 1.f; };
template <> struct Type<bf16_t> { static constexpr int PARTS = 3; static constexpr float P_BITS = 0.f, P_SCALE = 0x1p-24f; };
template <> struct Type<float> { static constexpr int PARTS = 1; static constexpr float P_BITS = 0.f, P_SCALE = 0x1p-24f; };

// Two fp32 numbers as pairs of the cache's type, most significant part first.  Every part is rounded to nearest and what it leaves has a sign, so two fp16 numbers
// hold 24 bits and three bf16 numbers all of them; and where a sum is so large that small parts are lost in it, they are lost to either side.  (Cut off,
// sixty thousand small weights beside a large one added up to 4e-5 less than they are over a bf16 cache.)
typedef float f32x2v __attribute__((ext_vector_type(2)));
template <typename KT> __device__ __forceinline__ void parts_of(float x, float y, uint32_t (&out)[Type<KT>::PARTS]);
template <> __device__ __forceinline__ void parts_of<half_t>(float x, float y, uint32_t (&out)[2]) {
    typedef _Float16 pair __attribute__((ext_vector_type(2)));
    out[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2v{x, y}), pair));
    float rx, ry;                                // x - hi, y - hi, in one instruction each (as two they are a sixth of a turn's vector instructions)
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(rx) : "v"(out[0]), "v"(x));
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(ry) : "v"(out[0]), "v"(y));
    out[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2v{rx, ry}), pair));
}
template <> __device__ __forceinline__ void parts_of<bf16_t>(float x, float y, uint32_t (&out)[3]) {
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        out[p] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2v{x, y}), pair));
        x -= __uint_as_float(out[p] << 16);
        y -= __uint_as_float(out[p] & 0xFFFF0000u);
    }
}
// The same for queries, which in bf16 may be as large as fp32's largest number: rounded, that would be an infinity.  Three times eight bits cut off are
// all of them.
template <typename KT> __device__ __forceinline__ void query_parts(float x, float y, uint32_t (&out)[Type<KT>::PARTS]) {
    if constexpr (Type<KT>::PARTS == 2) parts_of<KT>(x, y, out);
    else {
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
            out[p] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            x -= __uint_as_float(a & 0xFFFF0000u);
            y -= __uint_as_float(b & 0xFFFF0000u);
        }
    }
}

// The power of two that takes a row whose largest value is `top` to the upper end of fp16's range, and its inverse.
__device__ __forceinline__ void scaling(float top, float &up, float &down) {
    int ex = 15;
    if (top > 0.f && top < INFINITY) (void)frexpf(top, &ex);
    ex = max(ex, -100);
    up = ldexpf(1.f, 15 - ex);
    down = ldexpf(1.f, ex - 15);
}

// n / d for n < 2^31 (d's inverse by the host: one multiplication; a division by a number that is not known takes some forty
// instructions, and a block of a short call has little else to do).
__device__ __forceinline__ int over(int n, const Divisor &d) { return (int)(__umulhi(2u * (uint32_t)n, d.mul) >> d.shift); }

__device__ __forceinline__ void to_lds16(const char *from, char *to) {
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
#endif
}

// With l = ceil(log2 d): ceil(2^(31 + l) / d) exceeds the exact inverse by less than one part in 2^31.
inline Divisor divisor(int d) {
    int l = 0;
    while ((1u << l) < (unsigned)d) ++l;
    return Divisor{(uint32_t)(((1ull << (31 + l)) + d - 1) / d), l};
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace spda
