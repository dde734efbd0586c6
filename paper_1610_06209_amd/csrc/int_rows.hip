// Rotation and rounding of rows to 8-bit whole numbers with a scale for each row, and back.
#include <math.h>

#include "int_lane.hpp"

namespace spinner {
namespace {

// Rows to codes and scales, v = H D x on each run of 2^log coordinates first.  A row is WAVES waves' (1: four rows a workgroup; 8: one), HOLD chunks of
// 512 numbers each, which stay in registers from the largest magnitude to the codes; SWEEP: longer rows, which are read, and rotated, twice.
// Each of a row's slots gets the codes.
template <typename T, int WAVES, int HOLD, bool SWEEP>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : 512) int_quantize_kernel(IntQuantizeParams p)
{
    using Lane = LaneNumbers<T>;
    constexpr int ROWS = WAVES == 1 ? 4 : 1;
    __shared__ float4 meeting[WAVES > 1 ? 2 : 1][WAVES > 1 ? WAVES * 128 : 1];
    __shared__ int largest[2][8];
    const int lane = threadIdx.x & 63, in_group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = WAVES == 1 ? 0 : in_group;
    const unsigned flip = p.log > 0 ? Lane::flip(p.log, lane) : 0;
    const T* x = static_cast<const T*>(p.x);
    const long long slots = (long long)p.rows * p.top;
    const int row_chunks = (p.width + kChunk - 1) / kChunk, turns = SWEEP ? (row_chunks + WAVES * HOLD - 1) / (WAVES * HOLD) : 1;
    float d[HOLD][kPieceNumbers];
    const auto diagonals = [&](int turn) {
#pragma unroll
        for (int h = 0; h < HOLD; ++h) Lane((turn * HOLD + h) * WAVES + wave, lane, p.k).diagonal(d[h], p.diag, p.norm);
    };
    if (p.log > 0 && !SWEEP) diagonals(0);
    int parity = 0;
    for (long long r0 = (long long)blockIdx.x * ROWS; r0 < p.rows; r0 += (long long)gridDim.x * ROWS) {
        const long long own = r0 + (ROWS > 1 ? in_group : 0), row = own < p.rows ? own : p.rows - 1;
        const T* from = x + row * p.x_stride;
        float v[HOLD][kPieceNumbers];
        // the numbers of a turn, rotated
        const auto take = [&](int turn) {
            Quad raw[HOLD][Lane::HALVES];
#pragma unroll
            for (int h = 0; h < HOLD; ++h) fetch_chunk<T>(raw[h], from, ((turn * HOLD + h) * WAVES + wave) * kChunk + (lane << Lane::LOW), p.k);
            if (p.log > 0 && SWEEP) diagonals(turn);
#pragma unroll
            for (int h = 0; h < HOLD; ++h) {
                widen_quads<T>(raw[h], v[h]);
                if (p.log > 0) Lane::within(v[h], d[h], p.log, lane);
                if constexpr (WAVES > 1) {
                    if (p.log > 9) {
                        float4* m = meeting[parity];             // the other one may still be read
                        parity ^= 1;
                        Lane::meet(v[h], m + wave * 128, lane);
                        __syncthreads();
                        const int run = waves_of_run(p.log), in_run = wave & (run - 1);
                        Lane::join(v[h], m + (wave - in_run) * 128, run, in_run, lane);
                    }
                }
            }
        };
        int top = 0;
        for (int turn = 0; turn < turns; ++turn) {
            take(turn);
#pragma unroll
            for (int h = 0; h < HOLD; ++h) top = largest_bits(v[h], top);
        }
        top = wave_largest(top);
        if constexpr (WAVES > 1) {
            int* m = largest[(r0 / gridDim.x) & 1];
            if (lane == 0) m[wave] = top;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) top = m[w] > top ? m[w] : top;
        }
        const RowScale s(top);
        const float factor = flip ? -s.factor : s.factor;
        for (int turn = 0; turn < turns; ++turn) {
            if (SWEEP) take(turn);
#pragma unroll
            for (int h = 0; h < HOLD; ++h) {
                const int first = ((turn * HOLD + h) * WAVES + wave) * kChunk + (lane << Lane::LOW);
                unsigned c[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) c[i] = s.bad ? 0u : p.log > 0 ? four_codes<false>(v[h] + 4 * i, factor, 0.0f) : four_codes<true>(v[h] + 4 * i, factor, s.scale);
                for (int j = 0; j < p.top; ++j) {
                    const long long slot = p.places ? p.places[row * p.top + j] : row;
                    if (own >= p.rows || slot < 0 || slot >= slots) continue;
                    int8_t* to = p.codes + slot * p.width + first;
                    if constexpr (Lane::HALVES == 1) {
                        if (first < p.width) *reinterpret_cast<uint2*>(to) = uint2{c[0], c[1]};
                    } else {
                        if (first < p.width) *reinterpret_cast<unsigned*>(to) = c[0];
                        if (first + 256 < p.width) *reinterpret_cast<unsigned*>(to + 256) = c[1];
                    }
                }
            }
        }
        if (lane < p.top && wave == 0 && own < p.rows) {
            const long long slot = p.places ? p.places[row * p.top + lane] : row;
            if (slot >= 0 && slot < slots) p.scales[slot] = s.scale;
        }
    }
}

// Codes back to numbers, eight a lane, LANES lanes a row.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) int_dequantize_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scales, int rows, int k, int width,
                                                             T* __restrict__ out, long long out_stride)
{
    constexpr int ROWS = 256 / LANES;
    const int lane = threadIdx.x & (LANES - 1);
    for (long long row = (long long)blockIdx.x * ROWS + (LANES == 256 ? 0 : threadIdx.x / LANES); row < rows; row += (long long)gridDim.x * ROWS) {
        const float scale = scales[row];
        for (int col = ((int)blockIdx.y * LANES + lane) * 8; col < k; col += (int)gridDim.y * LANES * 8) {
            const uint2 c = *reinterpret_cast<const uint2*>(codes + row * width + col);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)((int)((i < 4 ? c.x : c.y) << (24 - 8 * (i & 3))) >> 24) * scale;
            T* to = out + row * out_stride + col;
            if (col + 8 <= k) {
                store_quad(to, v);
                if constexpr (sizeof(T) == 4) store_quad(to + 4, v + 4);
            } else {
#pragma unroll
                for (int i = 0; i < 7; ++i)
                    if (col + i < k) to[i] = (T)v[i];
            }
        }
    }
}

constexpr int kQuantizeBlocks = 8192;

template <typename T, int WAVES, int HOLD, bool SWEEP = false>
hipError_t quantize_as(const IntQuantizeParams& p, hipStream_t s)
{
    constexpr int ROWS = WAVES == 1 ? 4 : 1, MOST = kQuantizeBlocks / (2 * WAVES > 8 ? 8 : 4);
    const long long want = (p.rows + ROWS - 1LL) / ROWS;
    hipLaunchKernelGGL((int_quantize_kernel<T, WAVES, HOLD, SWEEP>), dim3((unsigned)(want < MOST ? want : MOST)), dim3(WAVES == 1 ? 256 : 512), 0, s, p);
    return hipGetLastError();
}

template <typename T>
hipError_t quantize(const IntQuantizeParams& p, hipStream_t s)
{
    const int chunks = (p.width + kChunk - 1) / kChunk;
    if (p.log <= 9) {
        if (chunks <= 1) return quantize_as<T, 1, 1>(p, s);
        if (chunks <= 2) return quantize_as<T, 1, 2>(p, s);
        if (chunks <= 4) return quantize_as<T, 1, 4>(p, s);
    }
    if (chunks <= 8) return quantize_as<T, 8, 1>(p, s);
    if (chunks <= 16) return quantize_as<T, 8, 2>(p, s);
    if (chunks <= 32) return quantize_as<T, 8, 4>(p, s);
    return quantize_as<T, 8, 2, true>(p, s);
}

template <typename T>
hipError_t dequantize(const int8_t* codes, const float* scales, int rows, int k, void* out, long long out_stride, hipStream_t s)
{
    const int width = int_width(k), pieces = (k + 7) / 8;
    const auto launch = [&](auto lanes, int runs) {
        constexpr int LANES = lanes.value, ROWS = 256 / LANES;
        const long long want = (rows + ROWS - 1LL) / ROWS, most = (1 << 22) / runs;
        hipLaunchKernelGGL((int_dequantize_kernel<T, LANES>), dim3((unsigned)(want < most ? want : most), runs), dim3(256), 0, s, codes, scales, rows, k, width,
                           static_cast<T*>(out), out_stride);
        return hipGetLastError();
    };
    if (pieces <= 32) return launch(std::integral_constant<int, 16>{}, 1);
    if (pieces <= 128) return launch(std::integral_constant<int, 64>{}, 1);
    return launch(std::integral_constant<int, 256>{}, (pieces + 255) / 256);
}

}  // namespace

hipError_t launch_int_quantize(const IntQuantizeParams& p, int dtype, hipStream_t s)
{
    switch (dtype) {
    case kF32: return quantize<float>(p, s);
    case kBf16: return quantize<__bf16>(p, s);
    default: return quantize<_Float16>(p, s);
    }
}

hipError_t launch_int_dequantize(const int8_t* codes, const float* scales, int rows, int k, void* out, int dtype, long long out_stride, hipStream_t s)
{
    switch (dtype) {
    case kF32: return dequantize<float>(codes, scales, rows, k, out, out_stride, s);
    case kBf16: return dequantize<__bf16>(codes, scales, rows, k, out, out_stride, s);
    default: return dequantize<_Float16>(codes, scales, rows, k, out, out_stride, s);
    }
}

}  // namespace spinner
