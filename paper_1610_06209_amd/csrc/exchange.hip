// Rows to their places in the order of the experts, their weighted sums back, and the gradients of both.
#include "mx4.hpp"
#include "number_io.hpp"
#include "route.hpp"
#include "spinner_kernels.hpp"

namespace spinner {
namespace {

constexpr int kThreads = 256;
constexpr long long kMemoryCache = 256 << 20;
constexpr long long kExchangeBlocks = 1 << 22;       // most workgroups: a grid holds fewer than 2^32 threads, and goes down the rows

template <bool STREAM = false>
__device__ __forceinline__ Quad load_piece(const char* p)
{
    const auto* q = reinterpret_cast<const LooseQuad<2>::type*>(p);
    if constexpr (STREAM) return __builtin_nontemporal_load(q);
    else return *q;
}
__device__ __forceinline__ void write_piece(char* p, Quad v) { *reinterpret_cast<LooseQuad<2>::type*>(p) = v; }

// A row of `bytes` in pieces of 16: where piece i starts (the last one ends with the row and may cover bytes of the one in front once more).
__device__ __forceinline__ long long piece_start(long long i, long long bytes) { return i * 16 + 16 <= bytes ? i * 16 : bytes - 16; }

// Geometry: a wave has a run of 64 pieces of one row (LANES 64: places and weights then are the wave's own), or four rows of up to 16 pieces.
template <int LANES>
struct RunsOfGrid {
    long long unit, units, step;
    int runs, lane;
    long long row;
    int piece;
    __device__ __forceinline__ RunsOfGrid(const ExchangeParams& p, long long pieces)
    {
        constexpr int EACH = kThreads / LANES;
        lane = threadIdx.x & (LANES - 1);
        runs = LANES == 64 ? (int)((pieces + 63) / 64) : 1;
        units = (long long)p.rows * runs;
        step = (long long)gridDim.x * EACH;
        unit = (long long)blockIdx.x * EACH + (LANES == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / LANES) : (int)threadIdx.x / LANES);
    }
    __device__ __forceinline__ bool any() const { return unit < units; }
    __device__ __forceinline__ void next() { unit += step; }
    __device__ __forceinline__ void find()
    {
        if constexpr (LANES == 64) {
            if (units <= 0xffffffffLL) row = (unsigned)unit / (unsigned)runs;
            else row = unit / runs;
            piece = (int)(unit - row * runs) * 64 + lane;
        } else {
            row = unit;
            piece = lane;
        }
    }
};

// A row is read once and written to each of its places: 16384 x 4 rows of 4096 in bf16, 671 MB, 116 to 126 us, 5.3 to 5.8 TB/s.
template <int SIZE, int LANES>
__global__ void __launch_bounds__(kThreads) dispatch_kernel(ExchangeParams p)
{
    const long long bytes = (long long)p.n * SIZE, slots = (long long)p.rows * p.top, pieces = bytes >= 16 ? (bytes + 15) / 16 : p.n;
    RunsOfGrid<LANES> at(p, pieces);
    for (; at.any(); at.next()) {
        at.find();
        const char* x = p.x + at.row * p.x_stride;
        const int* places = p.places + at.row * p.top;
        if (at.piece >= pieces) continue;
        if (bytes >= 16) {
            const long long from = piece_start(at.piece, bytes);
            const Quad v = load_piece(x + from);
            for (int j = 0; j < p.top; ++j) {
                const int place = places[j];
                if (place >= 0 && place < slots) write_piece(p.out + place * p.out_stride + from, v);
            }
        } else {
            using Number = std::conditional_t<SIZE == 4, unsigned, unsigned short>;
            const Number v = reinterpret_cast<const Number*>(x)[at.piece];
            for (int j = 0; j < p.top; ++j) {
                const int place = places[j];
                if (place >= 0 && place < slots) reinterpret_cast<Number*>(p.out + place * p.out_stride)[at.piece] = v;
            }
        }
    }
}

// 16 bytes of numbers in fp32
template <typename T, int N = 16 / (int)sizeof(T)>
__device__ __forceinline__ void widen(Quad q, float (&v)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) {
        if constexpr (sizeof(T) == 4) v[k] = __uint_as_float(q[k]);
        else v[k] = (float)__builtin_bit_cast(typename Pair16<T>::Pair, (unsigned)q[k >> 1])[k & 1];
    }
}

// 16 bytes of numbers to a place of any alignment of their type
template <bool STREAM, typename T>
__device__ __forceinline__ void store_piece(T* p, const float* v)
{
    if constexpr (STREAM) {
        typename LooseQuad<sizeof(T)>::type r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) r[i] = __float_as_uint(v[i]);
            else r[i] = Pair16<T>::narrow(v[2 * i], v[2 * i + 1]);
        }
        __builtin_nontemporal_store(r, reinterpret_cast<typename LooseQuad<sizeof(T)>::type*>(p));
    } else {
        store_quad(p, v);
    }
}

// out[r] = sum_j w[r][j] y[places[r][j]], fp32, j in order.  What has the weight 0 adds nothing, whatever its row holds: a choice of no expert has it,
// and its row may never have been written.
// Four rows on their way at a time (eight are level: 4099 x 6 rows of 1001 in fp16 14.8 us, 14.6).  STREAM: more rows than the memory's cache holds, which then
// need not keep them: 16384 x 4 rows of 4096 in bf16, 671 MB, 118 us for 127 in turn on one card (104 to 119 on others, 5.6 to 6.4 TB/s); where they would be found there it costs, 19 us for 15.
template <typename T, int LANES, bool STREAM>
__global__ void __launch_bounds__(kThreads) combine_kernel(ExchangeParams p)
{
    constexpr int N = 16 / (int)sizeof(T), GROUP = 4;
    const long long bytes = (long long)p.n * sizeof(T), slots = (long long)p.rows * p.top, pieces = bytes >= 16 ? (bytes + 15) / 16 : p.n;
    RunsOfGrid<LANES> at(p, pieces);
    for (; at.any(); at.next()) {
        at.find();
        const int* places = p.places + at.row * p.top;
        const float* weights = p.weights ? p.weights + at.row * p.top : nullptr;
        char* out = p.out + at.row * p.out_stride;
        if (at.piece >= pieces) continue;
        if (bytes >= 16) {
            const long long from = piece_start(at.piece, bytes);
            float sum[N];
#pragma unroll
            for (int k = 0; k < N; ++k) sum[k] = 0.0f;
            for (int j0 = 0; j0 < p.top; j0 += GROUP) {
                Quad q[GROUP];
                float w[GROUP];
                bool there[GROUP];
#pragma unroll
                for (int g = 0; g < GROUP; ++g) {
                    const int j = j0 + g < p.top ? j0 + g : p.top - 1, place = places[j];
                    w[g] = weights ? weights[j] : 1.0f;
                    there[g] = j0 + g < p.top && place >= 0 && place < slots && w[g] != 0.0f;
                    q[g] = load_piece<STREAM>(p.x + (there[g] ? place : 0) * p.x_stride + from);
                }
#pragma unroll
                for (int g = 0; g < GROUP; ++g) {
                    float v[N];
                    widen<T>(q[g], v);
#pragma unroll
                    for (int k = 0; k < N; ++k) sum[k] = there[g] ? __builtin_fmaf(w[g], v[k], sum[k]) : sum[k];
                }
            }
            store_piece<STREAM>(reinterpret_cast<T*>(out + from), sum);
        } else {
            float sum = 0.0f;
            for (int j = 0; j < p.top; ++j) {
                const int place = places[j];
                const float w = weights ? weights[j] : 1.0f;
                if (place >= 0 && place < slots && w != 0.0f) sum = __builtin_fmaf(w, (float)reinterpret_cast<const T*>(p.x + place * p.x_stride)[at.piece], sum);
            }
            reinterpret_cast<T*>(out)[at.piece] = (T)sum;
        }
    }
}

// dy[places[r][j]] = w[r][j] dout[r], dw[r][j] = sum_i dout[r][i] y[places[r][j]][i]: a workgroup (or LANES of its lanes) a row, a few j at a time
// 16384 x 4 rows of 4096 in bf16, 1.2 GB, 220 to 230 us, 5.3 to 5.5 TB/s (rows read but not written with the streaming hint: 220 for 228 without it in turn on one card; written with it too level).
template <typename T, int LANES, bool STREAM>
__global__ void __launch_bounds__(kThreads) combine_grad_kernel(ExchangeParams p)
{
    constexpr int N = 16 / (int)sizeof(T), GROUP = 4, ROWS = kThreads / LANES;
    __shared__ float part[kThreads / 64][GROUP];
    const int lane = threadIdx.x & (LANES - 1), wave = threadIdx.x >> 6;
    const long long bytes = (long long)p.n * sizeof(T), slots = (long long)p.rows * p.top;
    for (long long r0 = (long long)blockIdx.x * ROWS; r0 < p.rows; r0 += (long long)gridDim.x * ROWS) {
        const int in_group = LANES == 256 ? 0 : LANES == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / LANES) : (int)threadIdx.x / LANES;
        const long long own = r0 + in_group, row = own < p.rows ? own : p.rows - 1;
        const char* dout = p.x + row * p.x_stride;
        for (int j0 = 0; j0 < p.top; j0 += GROUP) {
            long long place[GROUP];
            float w[GROUP], dot[GROUP];
            bool there[GROUP];
#pragma unroll
            for (int g = 0; g < GROUP; ++g) {
                const int j = j0 + g < p.top ? j0 + g : p.top - 1;
                place[g] = p.places[row * p.top + j];
                there[g] = own < p.rows && j0 + g < p.top && place[g] >= 0 && place[g] < slots;
                if (!there[g]) place[g] = 0;
                w[g] = p.weights[row * p.top + j];
                dot[g] = 0.0f;
            }
            if (bytes >= 16) {
                for (long long i = lane; i * 16 < bytes; i += LANES) {
                    const long long from = piece_start(i, bytes);
                    const int again = (int)(i * 16 - from) / (int)sizeof(T);      // numbers that the piece in front has as well
                    float d[N];
                    const Quad qd = load_piece(dout + from);
                    Quad q[GROUP];
#pragma unroll
                    for (int g = 0; g < GROUP; ++g) q[g] = load_piece<STREAM>(p.y + place[g] * p.y_stride + from);
                    widen<T>(qd, d);
#pragma unroll
                    for (int g = 0; g < GROUP; ++g) {
                        float v[N], t[N];
                        widen<T>(q[g], v);
#pragma unroll
                        for (int k = 0; k < N; ++k) {
                            t[k] = w[g] * d[k];
                            dot[g] = k >= again ? __builtin_fmaf(d[k], v[k], dot[g]) : dot[g];
                        }
                        if (there[g]) store_quad(reinterpret_cast<T*>(p.out + place[g] * p.out_stride + from), t);
                    }
                }
            } else if (lane < p.n) {
                const float d = (float)reinterpret_cast<const T*>(dout)[lane];
#pragma unroll
                for (int g = 0; g < GROUP; ++g)
                    if (there[g]) {
                        dot[g] = d * (float)reinterpret_cast<const T*>(p.y + place[g] * p.y_stride)[lane];
                        reinterpret_cast<T*>(p.out + place[g] * p.out_stride)[lane] = (T)(w[g] * d);
                    }
            }
#pragma unroll
            for (int g = 0; g < GROUP; ++g) {
                dot[g] += lane_xor<1>(dot[g]);
                dot[g] += lane_xor<2>(dot[g]);
                dot[g] += lane_xor<4>(dot[g]);
                dot[g] += lane_xor<8>(dot[g]);
                if constexpr (LANES > 16) {
                    dot[g] += lane_xor<16>(dot[g]);
                    dot[g] += lane_xor<32>(dot[g]);
                }
            }
            if constexpr (LANES == 256) {
                if ((threadIdx.x & 63) == 0)
#pragma unroll
                    for (int g = 0; g < GROUP; ++g) part[wave][g] = dot[g];
                __syncthreads();
                if (threadIdx.x < GROUP && j0 + (int)threadIdx.x < p.top) {
                    const int g = threadIdx.x, j = j0 + g;
                    const int at = p.places[row * p.top + j];
                    const float all = (part[0][g] + part[1][g]) + (part[2][g] + part[3][g]);
                    p.dweights[row * p.top + j] = at >= 0 && at < slots ? all : 0.0f;
                }
                __syncthreads();
            } else if (lane == 0 && own < p.rows) {
#pragma unroll
                for (int g = 0; g < GROUP; ++g)
                    if (j0 + g < p.top) p.dweights[row * p.top + j0 + g] = there[g] ? dot[g] : 0.0f;
            }
        }
    }
}

dim3 grid_of(long long units, int each)
{
    const long long want = (units + each - 1) / each;
    return dim3((unsigned)(want < kExchangeBlocks ? want : kExchangeBlocks));
}
long long pieces_of(const ExchangeParams& p, int size)
{
    const long long bytes = (long long)p.n * size;
    return bytes >= 16 ? (bytes + 15) / 16 : p.n;
}

template <int SIZE>
hipError_t dispatch(const ExchangeParams& p, hipStream_t s)
{
    const long long pieces = pieces_of(p, SIZE);
    if (pieces <= 16) hipLaunchKernelGGL((dispatch_kernel<SIZE, 16>), grid_of(p.rows, 16), dim3(kThreads), 0, s, p);
    else hipLaunchKernelGGL((dispatch_kernel<SIZE, 64>), grid_of(p.rows * ((pieces + 63) / 64), 4), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}
// whether rows at their places are more than the memory-side cache of 256 MB keeps from the call that made them to this one
bool streams(const ExchangeParams& p, int size) { return (long long)p.rows * p.top * p.n * size > kMemoryCache; }

template <typename T, bool STREAM>
hipError_t combine_as(const ExchangeParams& p, bool grad, hipStream_t s)
{
    const long long pieces = pieces_of(p, sizeof(T));
    const dim3 threads(kThreads);
    if (grad) {
        if (pieces <= 16) hipLaunchKernelGGL((combine_grad_kernel<T, 16, STREAM>), grid_of(p.rows, 16), threads, 0, s, p);
        else if (pieces <= 128) hipLaunchKernelGGL((combine_grad_kernel<T, 64, STREAM>), grid_of(p.rows, 4), threads, 0, s, p);
        else hipLaunchKernelGGL((combine_grad_kernel<T, 256, STREAM>), grid_of(p.rows, 1), threads, 0, s, p);
    } else if (pieces <= 16) {
        hipLaunchKernelGGL((combine_kernel<T, 16, STREAM>), grid_of(p.rows, 16), threads, 0, s, p);
    } else {
        hipLaunchKernelGGL((combine_kernel<T, 64, STREAM>), grid_of(p.rows * ((pieces + 63) / 64), 4), threads, 0, s, p);
    }
    return hipGetLastError();
}
template <typename T>
hipError_t combine(const ExchangeParams& p, bool grad, hipStream_t s)
{
    return streams(p, sizeof(T)) ? combine_as<T, true>(p, grad, s) : combine_as<T, false>(p, grad, s);
}

}  // namespace

hipError_t launch_dispatch(const ExchangeParams& p, int size, hipStream_t s) { return size == 4 ? dispatch<4>(p, s) : dispatch<2>(p, s); }

hipError_t launch_combine(const ExchangeParams& p, int dtype, hipStream_t s)
{
    switch (dtype) {
    case kF32: return combine<float>(p, false, s);
    case kBf16: return combine<__bf16>(p, false, s);
    default: return combine<_Float16>(p, false, s);
    }
}

hipError_t launch_combine_grad(const ExchangeParams& p, int dtype, hipStream_t s)
{
    switch (dtype) {
    case kF32: return combine<float>(p, true, s);
    case kBf16: return combine<__bf16>(p, true, s);
    default: return combine<_Float16>(p, true, s);
    }
}

}  // namespace spinner
