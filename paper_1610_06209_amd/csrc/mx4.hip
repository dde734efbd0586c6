// Rotation and quantisation to microscaled 4-bit floating point (e2m1 with a shared power of two for each 32 numbers), and back.
#include "mx4.hpp"
#include "number_io.hpp"
#include "spinner_kernels.hpp"

namespace spinner {
namespace {

constexpr int kPieceNumbers = 8;                         // numbers of a lane that lie side by side
constexpr int kChunk = 64 * kPieceNumbers;               // numbers of a wave that lie side by side

// undoes the trade of lane_swap_stage
template <int LANE_BIT, int Q, int R>
__device__ __forceinline__ void swap_back(float (&v)[R])
{
#pragma unroll
    for (int j = 0; j < R; ++j)
        if (!(j & (1 << Q))) lane_swap<LANE_BIT>(v[j], v[j | (1 << Q)]);
}

// Rows [rows][k] to codes and scales, v = H D x on each run of 2^LOG coordinates first (LOG = 0: v = x).
// A lane holds eight neighbours, so index bits 0..2 are register bits, 3..8 lane bits, and from 2^10 on the chunks of 512 are
// the register bits above.  Butterflies in fp32; lane bits 4 and 5 trade places with register bits 1 and 2 for their stage.
// The transform's 1 / sqrt(2^LOG) goes into the diagonal.  A scale is shared by four neighbouring lanes: the largest magnitude
// as a whole number (so that a NaN is larger than an infinity and both larger than any number) gives the exponent.
// A wave stays with its columns, whose diagonal it keeps, and goes down the rows, one row's numbers asked for ahead.
template <typename T, int LOG>
__global__ void __launch_bounds__(256) mx4_quantize_kernel(QuantizeParams p, int column_groups, int row_step)
{
    constexpr int CHUNKS = LOG > 9 ? 1 << (LOG - 9) : 1;
    constexpr int N = CHUNKS * kPieceNumbers;
    const int lane = threadIdx.x & 63;
    const int gw = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = gw % column_groups;
    int row = gw / column_groups;
    if (row >= row_step) return;
    const int col = group * CHUNKS * kChunk + lane * kPieceNumbers;      // of the first chunk
    const bool live = col < p.k;                                         // a whole run of coordinates is live or is not
    const int safe = live ? col : 0;
    float d[N];
    if constexpr (LOG > 0) {
        const float norm = 1.0f / __builtin_sqrtf((float)(1 << LOG));
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int i = 0; i < kPieceNumbers; ++i)
                d[c * kPieceNumbers + i] = p.diag ? p.diag[safe + c * kChunk + i] * norm : norm;
    }
    const T* x = static_cast<const T*>(p.x) + safe;
    typename Piece<T>::Raw raw[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) raw[c] = Piece<T>::fetch(x + row * p.x_stride + c * kChunk);
    while (row < p.rows) {
        float v[N];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) Piece<T>::widen(raw[c], v + c * kPieceNumbers);
        const int at = row;
        row += row_step;
        if (row < p.rows) {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) raw[c] = Piece<T>::fetch(x + row * p.x_stride + c * kChunk);
        }
        if constexpr (LOG > 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= d[i];
            static_for<0, 3>([&](auto q) { reg_stage<q.value>(v); });
            static_for<0, 4>([&](auto b) {
                if constexpr (LOG > 3 + b.value) lane_stage<b.value>(v, (lane >> b.value) & 1 ? -1.0f : 1.0f);
            });
            if constexpr (LOG > 7) { lane_swap_stage<4, 1>(v); swap_back<4, 1>(v); }
            if constexpr (LOG > 8) { lane_swap_stage<5, 2>(v); swap_back<5, 2>(v); }
            static_for<3, (LOG > 9 ? LOG - 6 : 3)>([&](auto q) { reg_stage<q.value>(v); });
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const float* u = v + c * kPieceNumbers;
            int top = 0;
#pragma unroll
            for (int i = 0; i < kPieceNumbers; ++i) {
                const int bits = __float_as_int(u[i]) & 0x7fffffff;
                top = bits > top ? bits : top;
            }
            int other = lane_xor_i<1>(top);
            top = other > top ? other : top;
            other = lane_xor_i<2>(top);
            top = other > top ? other : top;
            const int e = top >> 23;                                     // largest magnitude: 2^(e - 127) and more
            const int byte = e == 255 ? 255 : (e > 2 ? e - 2 : 0);
            const float scale = exponent_value(byte);
            unsigned code = 0;
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, u[0], u[1], scale, 0);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, u[2], u[3], scale, 1);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, u[4], u[5], scale, 2);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, u[6], u[7], scale, 3);
            if (e == 255) code = 0;
            if (live) {
                const long long place = (long long)at * p.k + col + c * kChunk;
                *reinterpret_cast<unsigned*>(p.codes + (place >> 1)) = code;
                if ((lane & 3) == 0) p.scales[place >> 5] = (uint8_t)byte;
            }
        }
    }
}

// Codes back to numbers, eight a thread (STRIDED: rows of `out` that do not follow one another).
template <typename T, bool STRIDED>
__global__ void __launch_bounds__(256) mx4_dequantize_kernel(const unsigned* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                             long long pieces, int row_pieces, T* __restrict__ out, long long out_stride)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;
    const unsigned code = codes[i];
    const int byte = scales[i >> 2];
    const float scale = exponent_value(byte);
    float v[kPieceNumbers];
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    static_for<0, 4>([&](auto s) {
        const floatx2 t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, s.value);
        v[2 * s.value] = t[0];
        v[2 * s.value + 1] = t[1];
    });
    if (byte == 255)
#pragma unroll
        for (int j = 0; j < kPieceNumbers; ++j) v[j] = __builtin_nanf("");
    long long place = i * kPieceNumbers;
    if constexpr (STRIDED) {
        const long long row = i / row_pieces;
        place = row * out_stride + (i - row * row_pieces) * kPieceNumbers;
    }
    Piece<T>::store(out + place, v);
}

template <typename T, int LOG>
hipError_t quantize(const QuantizeParams& p, hipStream_t s)
{
    constexpr int width = LOG > 9 ? 1 << LOG : kChunk;
    const int groups = (p.k + width - 1) / width;
    // waves enough to fill the chip, no more than rows; each then goes down several rows
    const int want = (8192 + groups - 1) / groups;
    const int row_step = p.rows < want ? p.rows : want;
    const long long waves = (long long)groups * row_step;
    hipLaunchKernelGGL((mx4_quantize_kernel<T, LOG>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, p, groups, row_step);
    return hipGetLastError();
}

template <typename T>
hipError_t quantize_any(const QuantizeParams& p, int block, hipStream_t s)
{
    switch (block) {
    case 0: return quantize<T, 0>(p, s);
    case 32: return quantize<T, 5>(p, s);
    case 64: return quantize<T, 6>(p, s);
    case 128: return quantize<T, 7>(p, s);
    case 256: return quantize<T, 8>(p, s);
    case 512: return quantize<T, 9>(p, s);
    case 1024: return quantize<T, 10>(p, s);
    case 2048: return quantize<T, 11>(p, s);
    case 4096: return quantize<T, 12>(p, s);
    default: return hipErrorInvalidValue;
    }
}

template <typename T>
hipError_t dequantize(const uint8_t* codes, const uint8_t* scales, int rows, int k, void* out, long long out_stride, hipStream_t s)
{
    const long long pieces = (long long)rows * (k / kPieceNumbers);
    const long long blocks = (pieces + 255) / 256;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const auto kernel = out_stride == k || rows == 1 ? mx4_dequantize_kernel<T, false> : mx4_dequantize_kernel<T, true>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, s, reinterpret_cast<const unsigned*>(codes), scales, pieces,
                       k / kPieceNumbers, static_cast<T*>(out), out_stride);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_quantize(const QuantizeParams& p, int dtype, int block, hipStream_t s)
{
    switch (dtype) {
    case kF32: return quantize_any<float>(p, block, s);
    case kBf16: return quantize_any<__bf16>(p, block, s);
    default: return quantize_any<_Float16>(p, block, s);
    }
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int rows, int k, void* out, int dtype,
                                 long long out_stride, hipStream_t s)
{
    switch (dtype) {
    case kF32: return dequantize<float>(codes, scales, rows, k, out, out_stride, s);
    case kBf16: return dequantize<__bf16>(codes, scales, rows, k, out, out_stride, s);
    default: return dequantize<_Float16>(codes, scales, rows, k, out, out_stride, s);
    }
}

}  // namespace spinner
