// What a lane does of the rounding of rows to 8-bit whole numbers: the same steps, and so the same bits, wherever rows are quantised.
#pragma once
#include "int_rows.hpp"
#include "mx4_lane.hpp"

namespace spinner {

// A chunk's numbers of a lane (places as in LaneNumbers), zeros behind the row's end.
template <typename T>
__device__ __forceinline__ void fetch_chunk(Quad (&raw)[LaneNumbers<T>::HALVES], const T* row, int first, int k)
{
    constexpr int M = kPieceNumbers / LaneNumbers<T>::HALVES;
#pragma unroll
    for (int h = 0; h < LaneNumbers<T>::HALVES; ++h) {
        const int at = first + h * 256;
        if (at + M <= k) {
            raw[h] = stream_quad(row + at);
        } else {
            Quad v = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < M; ++i)
                if (at + i < k) {
                    if constexpr (sizeof(T) == 4) v[i] = reinterpret_cast<const unsigned*>(row)[at + i];
                    else v[i >> 1] |= (unsigned)reinterpret_cast<const unsigned short*>(row)[at + i] << (16 * (i & 1));
                }
            raw[h] = v;
        }
    }
}

// the largest magnitude as a whole number: a NaN is larger than an infinity and both larger than any number
__device__ __forceinline__ int largest_bits(const float (&v)[kPieceNumbers], int top)
{
#pragma unroll
    for (int i = 0; i < kPieceNumbers; ++i) {
        const int a = __float_as_int(v[i]) & 0x7fffffff;
        top = a > top ? a : top;
    }
    return top;
}
__device__ __forceinline__ int wave_largest(int top)
{
    static_for<0, 6>([&](auto b) {
        const int other = lane_xor_i<1 << b.value>(top);
        top = other > top ? other : top;
    });
    return top;
}

// A row's scale: its largest magnitude over 127, held at 2^-126 and above; NaN for a row with a NaN or an infinity, whose codes are 0.
struct RowScale {
    float scale, factor;                  // factor: 1 / scale
    bool bad;
    __device__ __forceinline__ explicit RowScale(int top)
    {
        bad = top >= 0x7f800000;
        const float s = __fdiv_rn(__int_as_float(top), 127.0f);
        scale = bad ? __builtin_nanf("") : (s > kSmallestScale ? s : kSmallestScale);
        factor = bad ? 0.0f : __fdiv_rn(1.0f, scale);
    }
};

// Four codes, v / scale to the nearest, ties to even: with 1.5 * 2^23 added, a number's last byte is the whole number.  The product with the rounded
// 1 / scale may take what lies within 2e-5 of a border to the other side; EXACT puts that right by what is left of v, which is exact there: v and
// code * scale are whole multiples of scale's last place, or half of it.
template <bool EXACT>
__device__ __forceinline__ unsigned four_codes(const float* v, float factor, float scale)
{
    constexpr float kWhole = 12582912.0f;
    unsigned b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float t = __builtin_fmaf(v[i], factor, kWhole);
        if constexpr (EXACT) {
            const float q = t - kWhole, left = __builtin_fmaf(-q, scale, v[i]), half = 0.5f * scale, far = __builtin_fabsf(left);
            // beyond the half, or on it from an odd number: one on, to the side that v lies on
            const bool odd = __float_as_uint(t) & 1;
            if (far > half || (far == half && odd)) t += left > 0.0f ? 1.0f : -1.0f;
        }
        b[i] = __float_as_uint(t);
    }
    const unsigned lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0c);
    return lo | hi;
}

}  // namespace spinner
