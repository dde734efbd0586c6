// What a lane does of the rotation and quantisation of rows to 4-bit numbers: the same steps, and so the same bits, wherever rows are quantised.
#pragma once
#include "mx4.hpp"
#include "number_io.hpp"
#include "spinner_kernels.hpp"

namespace spinner {

constexpr int kPieceNumbers = 8;                         // numbers of a lane
constexpr int kChunk = 64 * kPieceNumbers;               // numbers of a wave that lie side by side
__host__ __device__ constexpr int waves_of_run(int log) { return log > 9 ? 1 << (log - 9) : 1; }

// undoes the trade of lane_swap_stage
template <int LANE_BIT, int Q, int R>
__device__ __forceinline__ void swap_back(float (&v)[R])
{
#pragma unroll
    for (int j = 0; j < R; ++j)
        if (!(j & (1 << Q))) lane_swap<LANE_BIT>(v[j], v[j | (1 << Q)]);
}

// A lane holds eight numbers of a chunk of 512: eight neighbours of 16 bits, or four and the four 256 further on in fp32, 16 bytes each.  Runs are of 2^log
// coordinates (log: a constant or the same in all lanes).
template <typename T>
struct LaneNumbers {
    static constexpr int N = kPieceNumbers, HALVES = sizeof(T) == 4 ? 2 : 1, LOW = HALVES == 2 ? 2 : 3;      // index bit of lane bit 0
    using Numbers = float[N];

    // the places of one lane's numbers; what is not live (a whole run of coordinates is or is not) is read from the row's first
    int first, safe[HALVES];
    __device__ __forceinline__ LaneNumbers(int chunk, int lane, int k) : first(chunk * kChunk + (lane << LOW))
    {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) safe[h] = first + h * 256 < k ? first + h * 256 : 0;
    }
    __device__ __forceinline__ void fetch(Quad (&raw)[HALVES], const T* row) const
    {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) raw[h] = stream_quad(row + safe[h]);
    }
    // the transform's 1 / sqrt(2^log), `norm`, goes into the diagonal
    __device__ __forceinline__ void diagonal(Numbers& d, const float* diag, float norm) const
    {
        if (diag) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 a = *reinterpret_cast<const float4*>(diag + (HALVES == 2 ? safe[h % HALVES] : safe[0] + 4 * h));
                d[4 * h] = a.x * norm; d[4 * h + 1] = a.y * norm; d[4 * h + 2] = a.z * norm; d[4 * h + 3] = a.w * norm;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = norm;
        }
    }
    // which lanes' numbers a transform leaves negated (see lane_stage_fmac_dpp): a product of those of lane bits 0, 1 and 3 that it has
    static __device__ __forceinline__ unsigned flip(int log, int lane)
    {
        const int negating = (log > LOW) | (log > LOW + 1) << 1 | (log > LOW + 3) << 3;
        return __popc(lane & negating) & 1 ? 0x88888888u : 0u;
    }
    // The diagonal, and the butterflies within a wave, in fp32.  Index bits up to 2^8 are register and lane bits; lane bits 4 and 5
    // trade places with register bits 1 and 2 for their stage.
    static __device__ __forceinline__ void within(Numbers& v, const Numbers& d, int log, int lane)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= d[i];
        static_for<0, LOW>([&](auto q) { reg_stage<q.value>(v); });
        if constexpr (HALVES == 2)
            if (log > 8) reg_stage<2>(v);
        // (lane bits 0, 1 and 3 in one instruction a number, which leaves the upper lane's difference negated)
        static_for<0, 4>([&](auto b) {
            if (log > LOW + b.value) {
                const float coef = (lane >> b.value) & 1 ? -1.0f : 1.0f;
                if constexpr (b.value == 2) lane_stage<2>(v, coef);
                else lane_stage_fmac_dpp<b.value>(v, coef);
            }
        });
        if (log > LOW + 4) { lane_swap_stage<4, 1>(v); swap_back<4, 1>(v); }
        if (log > LOW + 5) { lane_swap_stage<5, 2>(v); swap_back<5, 2>(v); }
    }
    // The bits above: a run's chunks meet in LDS (`run`: its first one's numbers there), where each lane sums up the 2^(log - 9) numbers of its place
    // with their signs; `own`: which chunk of the run it has.
    static __device__ __forceinline__ void meet(const Numbers& v, float4* chunk, int lane)
    {
        chunk[lane] = make_float4(v[0], v[1], v[2], v[3]);
        chunk[64 + lane] = make_float4(v[4], v[5], v[6], v[7]);
    }
    static __device__ __forceinline__ void join(Numbers& v, const float4* run, int chunks, int own, int lane)
    {
        float t[N];
#pragma unroll
        for (int w = 0; w < chunks; ++w) {
            const float4 a = run[w * 128 + lane], b = run[w * 128 + 64 + lane];
            const float sign = __popc(w & own) & 1 ? -1.0f : 1.0f;
            const float u[N] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < N; ++i) t[i] = w == 0 ? u[i] : __builtin_fmaf(u[i], sign, t[i]);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = t[i];
    }
    // Scales and codes.  A scale is shared by four (fp32: eight) neighbouring lanes: the largest magnitude as a whole number (so that a NaN is larger
    // than an infinity and both larger than any number) gives the exponent.  Returns the column of the eight codes that come to lie in this lane.
    __device__ __forceinline__ int encode(const Numbers& v, unsigned flip, int lane, unsigned* codes, int (&byte)[HALVES]) const
    {
        unsigned code[HALVES];
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            constexpr int M = N / HALVES;
            const float* u = v + h * M;
            // the largest magnitude, numbers taken as they lie: positive ones in the order of signed whole numbers, negative ones above them in
            // that of unsigned ones
            int above = __float_as_int(u[0]);
            unsigned below = __float_as_uint(u[0]);
#pragma unroll
            for (int i = 1; i < M; ++i) {
                const int a = __float_as_int(u[i]);
                above = a > above ? a : above;
                below = (unsigned)a > below ? (unsigned)a : below;
            }
            int top = (int)(below & 0x7fffffffu);
            top = above > top ? above : top;
            static_for<0, 5 - LOW>([&](auto b) {
                const int other = lane_xor_i<1 << b.value>(top);
                top = other > top ? other : top;
            });
            const int e = top >> 23;                                     // largest magnitude: 2^(e - 127) and more
            byte[h] = e == 255 ? 255 : (e > 2 ? e - 2 : 0);
            const float scale = exponent_value(byte[h]);
            unsigned c = 0;
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, u[0], u[1], scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, u[2], u[3], scale, 1);
            if constexpr (HALVES == 1) {
                c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, u[4], u[5], scale, 2);
                c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, u[6], u[7], scale, 3);
            }
            c ^= flip;
            code[h] = e == 255 ? 0 : c;
        }
        // eight codes a lane side by side: fp32 lanes come by theirs in pairs, the even one of the first half
        const bool odd = HALVES == 2 && (lane & 1);
        if constexpr (HALVES == 2) {
            const unsigned own = (odd ? code[HALVES - 1] : code[0]) & 0xffff, got = lane_xor_i<1>(odd ? code[0] : code[HALVES - 1]) & 0xffff;
            code[0] = odd ? got | own << 16 : own | got << 16;
        }
        *codes = code[0];
        return odd ? first - 4 + 256 : first;
    }
};

}  // namespace spinner
