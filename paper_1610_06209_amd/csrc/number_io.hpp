// Pieces of 16 bytes of numbers in memory, in fp32, bf16 or fp16, at any alignment of their type, and the e8m0 scales.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace spinner {

// 16 bytes that are aligned only as their numbers are: the hardware takes such addresses in one access
struct __attribute__((packed, aligned(2))) Bytes16 { unsigned w[4]; };
struct __attribute__((packed, aligned(4))) Words4 { unsigned w[4]; };

// 16 bytes from an address of the alignment of T, which will not be asked for again
typedef unsigned Quad __attribute__((ext_vector_type(4)));
template <int BYTES> struct LooseQuad;
template <> struct LooseQuad<2> { typedef unsigned type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct LooseQuad<4> { typedef unsigned type __attribute__((ext_vector_type(4), aligned(4))); };
template <typename T>
__device__ __forceinline__ Quad stream_quad(const T* p)
{
    return __builtin_nontemporal_load(reinterpret_cast<const typename LooseQuad<sizeof(T)>::type*>(p));
}

template <typename T> struct Pair16 {
    typedef T Pair __attribute__((ext_vector_type(2)));
    // to nearest even: the one rounding of a result
    static __device__ __forceinline__ unsigned narrow(float a, float b)
    {
        const Pair t = {(T)a, (T)b};
        return __builtin_bit_cast(unsigned, t);
    }
};

// eight numbers from one (16 bits) or two (fp32) pieces of 16 bytes
template <typename T>
__device__ __forceinline__ void widen_quads(const Quad* q, float* v)
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(q[i >> 2][i & 3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned w = q[0][i];
            const auto t = __builtin_bit_cast(typename Pair16<T>::Pair, w);
            v[2 * i] = (float)t[0];
            v[2 * i + 1] = (float)t[1];
        }
    }
}

// 16 bytes of numbers to an address of the alignment of T
template <typename T>
__device__ __forceinline__ void store_quad(T* p, const float* v)
{
    typename LooseQuad<sizeof(T)>::type r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) r[i] = __float_as_uint(v[i]);
        else r[i] = Pair16<T>::narrow(v[2 * i], v[2 * i + 1]);
    }
    *reinterpret_cast<typename LooseQuad<sizeof(T)>::type*>(p) = r;
}

// 2^(byte - 127); 2^-127 is a subnormal number
__device__ __forceinline__ float exponent_value(int byte)
{
    return __uint_as_float(byte ? (unsigned)byte << 23 : 0x00400000u);
}

}  // namespace spinner
