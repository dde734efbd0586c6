// Pieces of eight neighbouring numbers in memory, in fp32, bf16 or fp16, at any alignment of their type, and the e8m0 scales.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace spinner {

// 16 bytes that are aligned only as their numbers are: the hardware takes such addresses in one access
struct __attribute__((packed, aligned(2))) Bytes16 { unsigned w[4]; };
struct __attribute__((packed, aligned(4))) Words4 { unsigned w[4]; };
struct __attribute__((packed, aligned(2))) Bytes8 { unsigned w[2]; };

template <typename T> struct Piece;

template <> struct Piece<float> {
    struct Raw { Words4 lo, hi; };
    static __device__ __forceinline__ Raw fetch(const float* p)
    {
        typedef unsigned Four __attribute__((ext_vector_type(4), aligned(4)));
        const Four a = __builtin_nontemporal_load(reinterpret_cast<const Four*>(p)), b = __builtin_nontemporal_load(reinterpret_cast<const Four*>(p) + 1);
        return {{{a[0], a[1], a[2], a[3]}}, {{b[0], b[1], b[2], b[3]}}};
    }
    static __device__ __forceinline__ void widen(const Raw& r, float* v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = __uint_as_float(r.lo.w[i]);
            v[4 + i] = __uint_as_float(r.hi.w[i]);
        }
    }
    static __device__ __forceinline__ void store(float* p, const float* v)
    {
        Raw r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            r.lo.w[i] = __float_as_uint(v[i]);
            r.hi.w[i] = __float_as_uint(v[4 + i]);
        }
        reinterpret_cast<Words4*>(p)[0] = r.lo;
        reinterpret_cast<Words4*>(p)[1] = r.hi;
    }
};

template <typename T> struct Piece16 {
    typedef T Pair __attribute__((ext_vector_type(2)));
    typedef Bytes16 Raw;
    static __device__ __forceinline__ Raw fetch(const T* p)
    {
        typedef unsigned Four __attribute__((ext_vector_type(4), aligned(2)));
        const Four a = __builtin_nontemporal_load(reinterpret_cast<const Four*>(p));
        return {{a[0], a[1], a[2], a[3]}};
    }
    static __device__ __forceinline__ void widen(const Raw& r, float* v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Pair t = __builtin_bit_cast(Pair, r.w[i]);
            v[2 * i] = (float)t[0];
            v[2 * i + 1] = (float)t[1];
        }
    }
    // to nearest even: the one rounding of a result
    static __device__ __forceinline__ unsigned narrow(float a, float b)
    {
        const Pair t = {(T)a, (T)b};
        return __builtin_bit_cast(unsigned, t);
    }
    static __device__ __forceinline__ void store(T* p, const float* v)
    {
        Bytes16 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = narrow(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<Bytes16*>(p) = r;
    }
};
template <> struct Piece<__bf16> : Piece16<__bf16> {};
template <> struct Piece<_Float16> : Piece16<_Float16> {};

// 2^(byte - 127); 2^-127 is a subnormal number
__device__ __forceinline__ float exponent_value(int byte)
{
    return __uint_as_float(byte ? (unsigned)byte << 23 : 0x00400000u);
}

}  // namespace spinner
