// Rotation and rounding of rows to 8-bit whole numbers with a scale for each row, and back.
#include "int_lane.hpp"

namespace spinner {
namespace {

// What the waves have written to LDS is there for all of them.  Numbers on their way from memory are not waited for, as __syncthreads() would: rows would come
// one by one.
__device__ __forceinline__ void waves_meet()
{
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

// Rows to codes and scales, v = H D x on each run of 2^log coordinates first.  A row is WAVES waves' (1: four rows a workgroup; 8: one), HOLD chunks of
// 512 numbers each, which stay in registers from the largest magnitude to the codes; SWEEP: longer rows, which are read, and rotated, twice.
// Each of a row's slots gets the codes.  16384 x 8192 without a rotation fp32 110 us, bf16 68, 6.1 and 5.9 TB/s, as fast as a copy; rotated in runs of 32 67, of 512 101, of 4096 124, where
// the butterflies' vector instructions bound it.
template <typename T, int LOG, int WAVES, int HOLD, bool SWEEP>
__global__ void __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) int_quantize_kernel(IntQuantizeParams p)
{
    using Lane = LaneNumbers<T>;
    constexpr int ROWS = WAVES == 1 ? 4 : 1;
    __shared__ float4 meeting[WAVES > 1 ? 2 : 1][WAVES > 1 ? WAVES * 128 : 1];
    __shared__ int largest[2][8];
    const int lane = threadIdx.x & 63, in_group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = WAVES == 1 ? 0 : in_group;
    const unsigned flip = LOG > 0 ? Lane::flip(LOG, lane) : 0;
    const T* x = static_cast<const T*>(p.x);
    const long long slots = (long long)p.rows * p.top;
    const int row_chunks = (p.width + kChunk - 1) / kChunk, turns = SWEEP ? (row_chunks + WAVES * HOLD - 1) / (WAVES * HOLD) : 1;
    float d[HOLD][kPieceNumbers];
    const auto diagonals = [&](int turn) {
#pragma unroll
        for (int h = 0; h < HOLD; ++h) Lane((turn * HOLD + h) * WAVES + wave, lane, p.k).diagonal(d[h], p.diag, p.norm);
    };
    if constexpr (LOG > 0 && !SWEEP) diagonals(0);
    Quad raw[HOLD][Lane::HALVES];
    const auto fetch = [&](const T* from, int turn) {
#pragma unroll
        for (int h = 0; h < HOLD; ++h) fetch_chunk<T, LOG == 0 && WAVES == 1 && HOLD == 1>(raw[h], from, ((turn * HOLD + h) * WAVES + wave) * kChunk + (lane << Lane::LOW), p.k);
    };
    const auto row_of = [&](long long r0) {
        const long long own = r0 + (ROWS > 1 ? in_group : 0);
        return own < p.rows ? own : p.rows - 1LL;
    };
    const long long step = (long long)gridDim.x * ROWS;
    if (!SWEEP) fetch(x + row_of((long long)blockIdx.x * ROWS) * p.x_stride, 0);
    int parity = 0, meetings = 0;
    for (long long r0 = (long long)blockIdx.x * ROWS; r0 < p.rows; r0 += step, ++meetings) {
        const long long own = r0 + (ROWS > 1 ? in_group : 0), row = row_of(r0);
        const T* from = x + row * p.x_stride;
        float v[HOLD][kPieceNumbers];
        // the numbers of a turn, rotated (without SWEEP: those of the next row are asked for as soon as these have left their registers)
        const auto take = [&](int turn) {
            if (SWEEP) fetch(from, turn);
            if constexpr (LOG > 0 && SWEEP) diagonals(turn);
#pragma unroll
            for (int h = 0; h < HOLD; ++h) {
                const int chunk = (turn * HOLD + h) * WAVES + wave;
                settle_chunk<T>(raw[h], chunk, chunk * kChunk + (lane << Lane::LOW), p.k);
                widen_quads<T>(raw[h], v[h]);
            }
            if (!SWEEP && r0 + step < p.rows) fetch(x + row_of(r0 + step) * p.x_stride, 0);
#pragma unroll
            for (int h = 0; h < HOLD; ++h) {
                if constexpr (LOG > 0) Lane::within(v[h], d[h], LOG, lane);
                if constexpr (WAVES > 1) {
                    if constexpr (LOG > 9) {
                        float4* m = meeting[parity];             // the other one may still be read
                        parity ^= 1;
                        Lane::meet(v[h], m + wave * 128, lane);
                        waves_meet();
                        const int run = waves_of_run(LOG), in_run = wave & (run - 1);
                        Lane::join(v[h], m + (wave - in_run) * 128, run, in_run, lane);
                    }
                }
            }
        };
        Largest most;
        for (int turn = 0; turn < turns; ++turn) {
            take(turn);
#pragma unroll
            for (int h = 0; h < HOLD; ++h) most.take(v[h]);
        }
        int top = wave_largest(most.bits());
        if constexpr (WAVES > 1) {
            int* m = largest[meetings & 1];
            if (lane == 0) m[wave] = top;
            waves_meet();
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
                eight_codes<LOG == 0>(v[h], factor, s.scale, c);
                c[0] = s.bad ? 0 : c[0];
                c[1] = s.bad ? 0 : c[1];
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

// Codes back to numbers, eight a lane, LANES lanes a row.  16384 x 8192 to bf16, 403 MB, 66 us, 6.1 TB/s: as fast as a copy.
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

template <typename T, int LOG, int WAVES, int HOLD, bool SWEEP = false>
hipError_t quantize_as(const IntQuantizeParams& p, hipStream_t s)
{
    constexpr int ROWS = WAVES == 1 ? 4 : 1, MOST = kQuantizeBlocks / (WAVES == 1 ? 4 : WAVES);
    const long long want = (p.rows + ROWS - 1LL) / ROWS;
    hipLaunchKernelGGL((int_quantize_kernel<T, LOG, WAVES, HOLD, SWEEP>), dim3((unsigned)(want < MOST ? want : MOST)), dim3(WAVES == 1 ? 256 : 64 * WAVES), 0, s, p);
    return hipGetLastError();
}

template <typename T, int LOG>
hipError_t quantize_log(const IntQuantizeParams& p, hipStream_t s)
{
    const int chunks = (p.width + kChunk - 1) / kChunk;
    if constexpr (LOG <= 9) {
        if (chunks <= 1) return quantize_as<T, LOG, 1, 1>(p, s);
        if (chunks <= 2) return quantize_as<T, LOG, 1, 2>(p, s);
        if (chunks <= 4) return quantize_as<T, LOG, 1, 4>(p, s);
    }
    if (chunks <= 8) return quantize_as<T, LOG, 8, 1>(p, s);
    // four waves of four chunks / eight of two, us: 16384 x 8192 bf16, no rotation 68 / 74, runs of 32 67 / 73, of 512 101 / 107; fp32 112 / 110, 119 / 115; 37 x 8191 fp16 4.2 / 3.5
    // (eight chunks, 8191 x 4096 bf16, runs of 256: four waves of two 24.1, eight of one 23.3)
    if constexpr (LOG <= 11 && sizeof(T) == 2)
        if (chunks <= 16 && p.rows >= 1024) return quantize_as<T, LOG, 4, 4>(p, s);
    if (chunks <= 16) return quantize_as<T, LOG, 8, 2>(p, s);
    if (chunks <= 32) return quantize_as<T, LOG, 8, 4>(p, s);
    return quantize_as<T, LOG, 8, 2, true>(p, s);
}

template <typename T>
hipError_t quantize(const IntQuantizeParams& p, hipStream_t s)
{
    switch (p.log) {
    case 0: return quantize_log<T, 0>(p, s);
    case 5: return quantize_log<T, 5>(p, s);
    case 6: return quantize_log<T, 6>(p, s);
    case 7: return quantize_log<T, 7>(p, s);
    case 8: return quantize_log<T, 8>(p, s);
    case 9: return quantize_log<T, 9>(p, s);
    case 10: return quantize_log<T, 10>(p, s);
    case 11: return quantize_log<T, 11>(p, s);
    case 12: return quantize_log<T, 12>(p, s);
    default: return hipErrorInvalidValue;
    }
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
