// Device helpers of the microscaled 4-bit kernels.
//
// Format: a row of K values is padded with zeros to Kp, a multiple of 128, and cut into blocks of 32.  A value is an
// E2M1 code (sign, two exponent bits, one mantissa bit), two in a byte, the lower index in the low half; a block has
// one scale byte s that stands for 2^(s - 127), 255 for "not a number".
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "mbu_internal.h"
#include "mfma_common.h"

namespace mbu {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

// The matrix instruction on 16 x 128 by 128 x 16 codes.  Lane l holds 32 codes and one scale byte (number J of the
// word) of row l % 16 of either operand; which of the four blocks of the instruction's 128 inputs these are is free, as
// long as both operands agree.  Lane l gets the outputs [4 (l / 16) + 0..3] of operand a's rows, operand b's row l % 16.
template <int J> __device__ __forceinline__ v4f mx4_mfma(v4i a, uint32_t sa, v4i b, uint32_t sb, v4f c)
{
    const v8i a8 = {a.x, a.y, a.z, a.w, 0, 0, 0, 0};
    const v8i b8 = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, J, (int)sa, J, (int)sb);
}

// Scale byte of a block whose largest magnitude has these float32 bits: floor(log2(magnitude)) - 2, so that the largest
// element lands in [4, 8) and is rounded to 4 or 6; 2^-127 where that is too small (a block of zeros among them);
// 255 for an infinity or NaN.
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t top)
{
    const uint32_t e = top >> 23;
    return e == 255u ? 255u : max(e, 2u) - 2u;
}

// Eight values -> eight codes and the largest magnitude, as float32 bits, for the three input types.  A value of the
// 16-bit types stays packed: magnitudes compare like unsigned numbers, NaN above infinity above all others, and the
// conversion takes them as they are (exact scaling by a power of two, nearest even, saturating at 6).
template <typename T> struct Mx4In;
template <> struct Mx4In<float> {
    static constexpr int CHUNK = 4;          // values of a 16-byte load
    uint32_t v[8];
    __device__ __forceinline__ void set(int i, float x) { v[i] = __float_as_uint(x); }
    __device__ __forceinline__ void set_chunk(int c, uint4 x)
    {
        v[4 * c] = x.x; v[4 * c + 1] = x.y; v[4 * c + 2] = x.z; v[4 * c + 3] = x.w;
    }
    __device__ __forceinline__ uint32_t top() const
    {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, v[i] & 0x7fffffffu);
        return t;
    }
    __device__ __forceinline__ uint32_t codes(float scale) const
    {
        uint32_t q = 0;
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v[0]), __uint_as_float(v[1]), scale, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v[2]), __uint_as_float(v[3]), scale, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v[4]), __uint_as_float(v[5]), scale, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, __uint_as_float(v[6]), __uint_as_float(v[7]), scale, 3);
        return q;
    }
};
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b)
{
    typedef unsigned short v2us __attribute__((ext_vector_type(2)));
    const v2us r = __builtin_elementwise_max(__builtin_bit_cast(v2us, a), __builtin_bit_cast(v2us, b));
    return __builtin_bit_cast(uint32_t, r);
}
template <> struct Mx4In<__bf16> {
    static constexpr int CHUNK = 8;
    uint32_t v[4];
    __device__ __forceinline__ void set(int i, __bf16 x)
    {
        const uint32_t u = __builtin_bit_cast(unsigned short, x);
        v[i >> 1] = (i & 1) ? (v[i >> 1] & 0xffffu) | (u << 16) : u;
    }
    __device__ __forceinline__ void set_chunk(int, uint4 x) { v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; }
    __device__ __forceinline__ uint32_t top() const
    {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) t = max_halves(t, v[i] & 0x7fff7fffu);
        return max(t & 0xffff0000u, t << 16);
    }
    __device__ __forceinline__ uint32_t codes(float scale) const
    {
        uint32_t q = 0;
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(v2bf, v[0]), scale, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(v2bf, v[1]), scale, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(v2bf, v[2]), scale, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(q, __builtin_bit_cast(v2bf, v[3]), scale, 3);
        return q;
    }
};
template <> struct Mx4In<_Float16> {
    static constexpr int CHUNK = 8;
    uint32_t v[4];
    __device__ __forceinline__ void set(int i, _Float16 x)
    {
        const uint32_t u = __builtin_bit_cast(unsigned short, x);
        v[i >> 1] = (i & 1) ? (v[i >> 1] & 0xffffu) | (u << 16) : u;
    }
    __device__ __forceinline__ void set_chunk(int, uint4 x) { v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; }
    __device__ __forceinline__ uint32_t top() const
    {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) t = max_halves(t, v[i] & 0x7fff7fffu);
        const unsigned short h = (unsigned short)max(t & 0xffffu, t >> 16);
        return __float_as_uint((float)__builtin_bit_cast(_Float16, h));      // exact
    }
    __device__ __forceinline__ uint32_t codes(float scale) const
    {
        uint32_t q = 0;
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, __builtin_bit_cast(v2h, v[0]), scale, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, __builtin_bit_cast(v2h, v[1]), scale, 1);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, __builtin_bit_cast(v2h, v[2]), scale, 2);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(q, __builtin_bit_cast(v2h, v[3]), scale, 3);
        return q;
    }
};
// 16 bytes of a row of floats, aligned to their type only (the hardware takes any address)
template <typename T> __device__ __forceinline__ uint4 load_floats(const T *p)
{
    uint4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
// the first `n` values of a chunk of eight, zeros behind them
template <typename T> __device__ __forceinline__ Mx4In<T> load_some(const T *p, int n)
{
    Mx4In<T> in;
#pragma unroll
    for (int i = 0; i < 8; ++i) in.set(i, i < n ? p[i] : (T)0.0f);
    return in;
}
template <typename T> __device__ __forceinline__ Mx4In<T> load_eight(const T *p)
{
    Mx4In<T> in;
#pragma unroll
    for (int c = 0; c < 8 / Mx4In<T>::CHUNK; ++c) in.set_chunk(c, load_floats(p + c * Mx4In<T>::CHUNK));
    return in;
}
template <typename T> __device__ __forceinline__ Mx4In<T> zero_eight()
{
    Mx4In<T> in;
#pragma unroll
    for (int c = 0; c < 8 / Mx4In<T>::CHUNK; ++c) in.set_chunk(c, make_uint4(0, 0, 0, 0));
    return in;
}

// the conversions read the exponent field of the scale alone: 2^-127, whose float32 form is a subnormal, is 0 here
__device__ __forceinline__ float mx4_scale_float(uint32_t s) { return __uint_as_float(s << 23); }

// The 16 scale bytes of a row's 512 inputs -> the four that lane group g multiplies with, byte j for instruction j:
// bytes g, 4 + g, 8 + g, 12 + g
__device__ __forceinline__ uint32_t mx4_scales_of(v4i s, int g)
{
    const uint32_t pick = 0x0400u + 0x0101u * (uint32_t)g;          // byte g of the second word, byte g of the first
    const uint32_t lo = __builtin_amdgcn_perm((uint32_t)s.y, (uint32_t)s.x, pick);
    const uint32_t hi = __builtin_amdgcn_perm((uint32_t)s.w, (uint32_t)s.z, pick);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
}
// ... of a row that has `left` scale bytes left (a multiple of four; what follows belongs to another row)
__device__ __forceinline__ v4i mx4_row_end(v4i s, int left)
{
    return (v4i){left > 0 ? s.x : 0, left > 4 ? s.y : 0, left > 8 ? s.z : 0, left > 12 ? s.w : 0};
}

// Masked-binary weights: two bits a weight, 16 in a word.  Nibble q holds weight q in bits 3 (sign) and 1 (kept) and
// weight q + 8 in bits 2 and 0, so that a mask makes eight codes of either half: -1 is 0b1010, +1 is 0b0010.
__device__ __forceinline__ v4i expand_masked(uint32_t w0, uint32_t w1)
{
    v4i r;
    r.x = (int)(w0 & 0xaaaaaaaau);
    r.y = (int)((w0 << 1) & 0xaaaaaaaau);
    r.z = (int)(w1 & 0xaaaaaaaau);
    r.w = (int)((w1 << 1) & 0xaaaaaaaau);
    return r;
}

// the type that a template argument of mbu_float_type stands for
template <int CODE> struct Mx4Type { using T = uint8_t; };
template <> struct Mx4Type<MBU_FLOAT32> { using T = float; };
template <> struct Mx4Type<MBU_FLOAT16> { using T = _Float16; };
template <> struct Mx4Type<MBU_BFLOAT16> { using T = __bf16; };

// The one rounding of a product: from the float32 sum to the output's type, to nearest even.
__device__ __forceinline__ void mx4_store(float *p, float v) { *p = v; }
__device__ __forceinline__ void mx4_store(__bf16 *p, float v) { *p = (__bf16)v; }
__device__ __forceinline__ void mx4_store(_Float16 *p, float v) { *p = (_Float16)v; }
// four values of 2 bytes
typedef int v2i __attribute__((ext_vector_type(2)));
template <typename T> __device__ __forceinline__ v2i mx4_pack4(v4f v)
{
    typedef T v4t __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(v2i, (v4t){(T)v.x, (T)v.y, (T)v.z, (T)v.w});
}

}  // namespace mbu
