// What a lane does of the rounding of rows to 8-bit whole numbers: the same steps, and so the same bits, wherever rows are quantised.
#pragma once
#include "int_rows.hpp"
#include "mx4_lane.hpp"

namespace spinner {

// A chunk's numbers of a lane (places as in LaneNumbers), in two halves, so that loads in flight are not waited for one by one: what the row's end cuts,
// or lies behind it, is read as the numbers in front of the end, and put right when it has come.  Rows shorter than a piece (SHORT: there may be such) come number by number.
template <typename T, bool SHORT>
__device__ __forceinline__ void fetch_chunk(Quad (&raw)[LaneNumbers<T>::HALVES], const T* row, int first, int k)
{
    constexpr int M = kPieceNumbers / LaneNumbers<T>::HALVES;
#pragma unroll
    for (int h = 0; h < LaneNumbers<T>::HALVES; ++h) {
        const int at = first + h * 256;
        if (!SHORT || k >= M) {
            raw[h] = stream_quad(row + (at < k - M ? at : k - M));
        } else {
            Quad v = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < M - 1; ++i)
                if (at + i < k) {
                    if constexpr (sizeof(T) == 4) v[i] = reinterpret_cast<const unsigned*>(row)[at + i];
                    else v[i >> 1] |= (unsigned)reinterpret_cast<const unsigned short*>(row)[at + i] << (16 * (i & 1));
                }
            raw[h] = v;
        }
    }
}
template <typename T>
__device__ __forceinline__ void settle_chunk(Quad (&raw)[LaneNumbers<T>::HALVES], int chunk, int first, int k)
{
    constexpr int M = kPieceNumbers / LaneNumbers<T>::HALVES;
    if (chunk * kChunk + kChunk <= k || k < M) return;
#pragma unroll
    for (int h = 0; h < LaneNumbers<T>::HALVES; ++h) {
        const int count = k - first - h * 256, cut = count >= M ? 0 : (count > 0 ? M - count : M);
        unsigned long long lo = raw[h][0] | (unsigned long long)raw[h][1] << 32, hi = raw[h][2] | (unsigned long long)raw[h][3] << 32;
        const int bits = (cut * (int)sizeof(T) & 7) * 8;
        if (cut * (int)sizeof(T) >= 8) { lo = hi; hi = 0; }
        if (cut == M) lo = 0;
        lo = lo >> bits | (bits ? hi << (64 - bits) : 0);
        hi >>= bits;
        raw[h] = Quad{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
    }
}

// The largest magnitude as a whole number: a NaN is larger than an infinity and both larger than any number.  Numbers as they lie: positive ones in the
// order of signed whole numbers, negative ones above them in that of unsigned ones.
struct Largest {
    int above = 0;
    unsigned below = 0;
    __device__ __forceinline__ void take(const float (&v)[kPieceNumbers])
    {
#pragma unroll
        for (int i = 0; i < kPieceNumbers; ++i) {
            const int a = __float_as_int(v[i]);
            above = a > above ? a : above;
            below = (unsigned)a > below ? (unsigned)a : below;
        }
    }
    __device__ __forceinline__ int bits() const
    {
        const int b = below & 0x80000000u ? (int)(below & 0x7fffffffu) : 0;
        return above > b ? above : b;
    }
};
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
    float scale, factor;                  // factor: 1 / scale, to its last place
    bool bad;
    __device__ __forceinline__ explicit RowScale(int top)
    {
        bad = top >= 0x7f800000;
        // top / 127 as a division rounds it, for every number of this type: the quotient by 1 / 127 and what it leaves
        constexpr float kPart = 1.0f / 127.0f;
        const float a = __int_as_float(top), q = a * kPart, s = __builtin_fmaf(__builtin_fmaf(-q, 127.0f, a), kPart, q);
        scale = bad ? __builtin_nanf("") : (s > kSmallestScale ? s : kSmallestScale);
        factor = bad ? 0.0f : __builtin_amdgcn_rcpf(scale);
    }
};

// Eight codes, v / scale to the nearest, ties to even: with 1.5 * 2^23 added, a number's last byte is the whole number.  The product with the rounded
// 1 / scale may take what lies within 2e-5 of a border to the other side; EXACT puts that right by what is left of v, which is exact there: v and
// code * scale are whole multiples of scale's last place, or half of it.  (Few waves have anything to put right: looking for it and doing it only
// there, 16384 x 8192 bf16 numbers 73 us, always doing it 95.)
template <bool EXACT>
__device__ __forceinline__ void eight_codes(const float (&v)[kPieceNumbers], float factor, float scale, unsigned (&codes)[2])
{
    constexpr float kWhole = 12582912.0f;
    float t[kPieceNumbers];
#pragma unroll
    for (int i = 0; i < kPieceNumbers; ++i) t[i] = __builtin_fmaf(v[i], factor, kWhole);
    if constexpr (EXACT) {
        const float half = 0.5f * scale;
        float left[kPieceNumbers], most = 0.0f;
#pragma unroll
        for (int i = 0; i < kPieceNumbers; ++i) {
            left[i] = __builtin_fmaf(kWhole - t[i], scale, v[i]);
            most = fmaxf(most, __builtin_fabsf(left[i]));
        }
        if (__ballot(most >= half) != 0) {
#pragma unroll
            for (int i = 0; i < kPieceNumbers; ++i) {
                // beyond the half, or on it from an odd number: one on, to the side that v lies on
                const float far = __builtin_fabsf(left[i]), one = left[i] > 0.0f ? 1.0f : -1.0f;
                t[i] += (far > half) | ((far == half) & ((__float_as_uint(t[i]) & 1) != 0)) ? one : 0.0f;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const unsigned a = __float_as_uint(t[4 * i]), b = __float_as_uint(t[4 * i + 1]), c = __float_as_uint(t[4 * i + 2]), d = __float_as_uint(t[4 * i + 3]);
        codes[i] = __builtin_amdgcn_perm(b, a, 0x0c0c0400) | __builtin_amdgcn_perm(d, c, 0x04000c0c);
    }
}

}  // namespace spinner
