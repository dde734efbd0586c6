// Rotation and quantisation to microscaled 4-bit floating point (e2m1 with a shared power of two for each 32 numbers), and back.
#include <math.h>

#include "int_rows.hpp"
#include "mx4_lane.hpp"

namespace spinner {
namespace {

// Rows [rows][k] to codes and scales, v = H D x on each run of 2^LOG coordinates first (LOG = 0: v = x).
// Eight numbers a lane (fp32: four and four, 16 bytes each; eight neighbours, whose two loads take every second piece of a line, 16384 x 16384 254 us;
// so 219).  Waves of a run longer than a wave's 512 numbers meet in LDS (in registers alone, 64 numbers a lane at 2^12, a wave's 240 registers
// left one wave a SIMD: one row of 4096 12.9 us, here 3.5).
// A wave stays with its columns, whose diagonal it keeps, and goes down the rows, the next row's numbers asked for ahead.
// Measured, bf16 16384 x 8192 (340 MB): no rotation 57 us, 6.0 TB/s (the copy rate is 6.2), runs of 256 64, 512 73, 1024 82, 2048 92, 4096 105.  Runs are bound by the vector
// ALU: 15 (256), 17 (512) to 24 (4096) instructions a number keep it busy 82 to 92 % of the time, without a rotation 5 and 30 %.
template <typename T, int LOG>
__global__ void __launch_bounds__(LOG > 9 ? 64 * waves_of_run(LOG) : 256) mx4_quantize_kernel(QuantizeParams p, int column_groups, int row_step)
{
    constexpr int WAVES = waves_of_run(LOG);
    using Lane = LaneNumbers<T>;
    __shared__ float4 meeting[WAVES > 1 ? 2 : 1][WAVES > 1 ? WAVES * 128 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = WAVES > 1 ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave;
    const int group = unit % column_groups;
    int row = unit / column_groups;
    if (row >= row_step) return;
    const Lane at_lane(WAVES > 1 ? group * WAVES + wave : group, lane, p.k);
    const unsigned flip = LOG > 0 ? Lane::flip(LOG, lane) : 0;
    float d[kPieceNumbers];
    if constexpr (LOG > 0) at_lane.diagonal(d, p.diag, 1.0f / __builtin_sqrtf((float)(1 << LOG)));
    const T* x = static_cast<const T*>(p.x);
    Quad raw[Lane::HALVES];
    at_lane.fetch(raw, x + row * p.x_stride);
    for (int turn = 0; row < p.rows; ++turn) {
        float v[kPieceNumbers];
        widen_quads<T>(raw, v);
        const int at = row;
        row += row_step;
        if (row < p.rows) at_lane.fetch(raw, x + row * p.x_stride);
        if constexpr (LOG > 0) Lane::within(v, d, LOG, lane);
        if constexpr (WAVES > 1) {
            float4* m = meeting[turn & 1];           // the other one may still be read
            Lane::meet(v, m + wave * 128, lane);
            __syncthreads();
            Lane::join(v, m, WAVES, wave, lane);
        }
        unsigned codes;
        int byte[Lane::HALVES];
        const int col = at_lane.encode(v, flip, lane, &codes, byte);
        const long long place = (long long)at * p.k;
        if (col < p.k) *reinterpret_cast<unsigned*>(p.codes + ((place + col) >> 1)) = codes;
        if ((lane & ((32 >> Lane::LOW) - 1)) == 0)
#pragma unroll
            for (int h = 0; h < Lane::HALVES; ++h)
                if (at_lane.first + h * 256 < p.k) p.scales[(place + at_lane.first + h * 256) >> 5] = (uint8_t)byte[h];
    }
}

// Codes back to numbers, 16 bytes of them a thread (STRIDED: rows of `out` that do not follow one another).  bf16 16384 x 16384 128 us, 5.3 TB/s.
template <typename T, bool STRIDED>
__global__ void __launch_bounds__(256) mx4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, long long first, long long pieces,
                                                             int row_pieces, T* __restrict__ out, long long out_stride)
{
    constexpr int M = 16 / sizeof(T);
    const long long i = first + (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;
    const unsigned code = M == 8 ? reinterpret_cast<const unsigned*>(codes)[i] : reinterpret_cast<const unsigned short*>(codes)[i];
    const int byte = scales[i / (32 / M)];
    const float scale = exponent_value(byte);
    float v[M];
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    static_for<0, M / 2>([&](auto s) {
        const floatx2 t = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, s.value);
        v[2 * s.value] = t[0];
        v[2 * s.value + 1] = t[1];
    });
    if (byte == 255)
#pragma unroll
        for (int j = 0; j < M; ++j) v[j] = __builtin_nanf("");
    long long place = i * M;
    if constexpr (STRIDED) {
        const long long row = i / row_pieces;
        place = row * out_stride + (i - row * row_pieces) * M;
    }
    store_quad(out + place, v);
}

template <typename T, int LOG>
hipError_t quantize(const QuantizeParams& p, hipStream_t s)
{
    constexpr int waves = waves_of_run(LOG), width = waves * kChunk;
    const int groups = (p.k + width - 1) / width;
    // waves enough to fill the chip, no more than rows; each then goes down several rows.  8192 / 16384 waves, bf16, in us: runs of 512, 16384 x 8192 74.0 / 72.8; no
    // rotation 57.4 / 57.0; runs of 1024 and 4096, 16384 x 8192 82 / 79 and 105 / 101, but 2048 x 4096 6.7 / 7.3 and 8.0 / 8.4
    const int want = ((LOG > 0 && waves == 1 ? 16384 : 8192) / waves + groups - 1) / groups;
    const int row_step = p.rows < want ? p.rows : want;
    const long long units = (long long)groups * row_step, blocks = waves > 1 ? units : (units + 3) / 4;
    hipLaunchKernelGGL((mx4_quantize_kernel<T, LOG>), dim3((unsigned)blocks), dim3(waves > 1 ? 64 * waves : 256), 0, s, p, groups, row_step);
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
    constexpr int numbers = 16 / sizeof(T);
    const long long pieces = (long long)rows * (k / numbers);
    const auto kernel = out_stride == k || rows == 1 ? mx4_dequantize_kernel<T, false> : mx4_dequantize_kernel<T, true>;
    // in grids of fewer than 2^32 threads
    constexpr long long most = 1LL << 31;
    for (long long first = 0; first < pieces; first += most) {
        const long long threads = pieces - first < most ? pieces - first : most;
        hipLaunchKernelGGL(kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, codes, scales, first, pieces, k / numbers, static_cast<T*>(out), out_stride);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

// What the forms of the product take, measured on MI355X: time of a chunk of depth (128 bytes of a row: 64 numbers of 16 bits, 256 of 4) when a
// few workgroups run and when all do, time around the chunks (where the tile lies, first loads, results), workgroups the chip holds.
//   16 bits   k = n = 4096, us for 100 / 300 / 1000 / 16384 (8 experts) rows: 256 x 256 72 / 73 / 75 / 513, 128 x 128 43 / 42 / 45 / 590, with four
//             chunks in LDS 31 / 32 / 37 / 625, 64 x 64 16 / 26 / 54 / 900; 4099 rows, 16 experts, k = 1000, n = 1032 31 / 22 / 27 / 28
//   4 bits    37 x 10007 x 8192 256 x 256 47, 128 x 128 26, 64 x 64 13.5; 300 x 4096 x 4096 28 / 15 / 16; 1000 x 10007 x 4128 44 / 53 / 90; 2000 rows, 8 experts,
//             k = n = 2048 20 / 13.5 / 26; 8192^3 269 / 328 / 519
struct Form {
    int tile, side;
    double alone, busy, around;
    int slots;
};
constexpr Form kForms16[] = {{kTile256, 256, 1.1, 1.6, 10, 256}, {kTile128, 128, 0.62, 0.95, 5, 512}, {kTile128Deep, 128, 0.45, 0.5, 5, 256}, {kTile64, 64, 0.22, 0.37, 3.5, 512}};
constexpr Form kForms4[] = {{kTile256, 256, 1.25, 2.0, 6, 256}, {kTile128, 128, 0.7, 1.15, 4, 512}, {kTile64, 64, 0.33, 0.33, 3, 256}};
// 64 x 64 tiles hold the scales of so many 4-bit numbers of a row, 33 of 100 KB of LDS; deeper sums take tiles of 128 x 128: 37 x 10007 x 8192 12.7 us, x 8224 33.0; 37 x 4096 x 8192
// 10.5, x 14336 40.7
constexpr int kHeldDepth = 8192;
constexpr size_t kMostPartial = 64u << 20;       // bytes of partial sums

template <int N>
static double shortest(const Form (&forms)[N], int direction, int chunk_numbers, ProductParams* p)
{
    const bool mx4 = chunk_numbers == 256;
    double best = 1e30;
    for (const Form& f : forms) {
        if (mx4 && f.tile == kTile64 && p->depth > kHeldDepth) continue;
        double tiles = (p->width + f.side - 1) / f.side, chunks;
        if (direction == kDw) {
            tiles *= (double)((p->height + f.side - 1) / f.side) * p->experts;
            // the longest group of several, taken as half as long again as they are on average, which the host does not know to be so: 8192 rows, 16 experts, k = n = 1024
            // 28 us where they are equal, 90 with half of the rows in one group, 163 with all; 32768 rows, 8 experts, k = n = 4096 978, 956, 960
            chunks = ceil(p->rows * (p->experts > 1 ? 1.5 : 1.0) / p->experts / 64);
        } else {
            // a group's last tile is half full on average
            tiles *= p->experts > 1 ? (double)p->rows / f.side + 0.5 * (p->experts < p->rows ? p->experts : p->rows) : (p->rows + f.side - 1) / f.side;
            chunks = ceil((double)p->depth / chunk_numbers);
        }
        for (int splits = 1; splits <= (direction == kDw ? 16 : 1); splits *= 2) {
            const double work = tiles * splits, rounds = ceil(work / f.slots), share = ceil(chunks / splits);
            double t = rounds * (share * (f.alone + (f.busy - f.alone) * (work < f.slots ? work / f.slots : 1)) + f.around);
            if (splits > 1) {
                // partial sums written and read at 4 TB/s, and one more launch (30000 rows, 3 experts, k = n = 256: 92 us, in 8 shares 21)
                const double bytes = (double)splits * p->experts * p->height * p->width * sizeof(float);
                if (bytes > kMostPartial || share < 2) break;
                t += 4 + 2 * bytes / 4e6;
            }
            if (t < best) {
                best = t;
                p->tile = f.tile;
                p->splits = splits;
            }
        }
    }
    return best;
}

// (16-bit rows that are no whole pieces of 16 bytes go by the same choice, though their kernels, 64 x 64 or 128 x 128 and a chunk ahead through registers, take longer: see
// launch_product_as)
void plan_product(int direction, bool mx4, ProductParams* p)
{
    p->splits = 1;
    if (direction == kForward) {
        // up to sixteen rows a group the weights' way from memory is all (4 bits, n = 16384, k = 4096, 16 rows: 9.8 us, 64 x 64 tiles 10.7; 32 rows: 15.2, 10.8);
        // and tiles read 4-bit operands' scales sixteen at a time.  It goes by the mean, as the rows of each group are known on the GPU only.  Few rows / tiles of 128 x 128 in us, bf16 and 4 bits:
        // 1024 rows, 64 experts, k = 2048, n = 4096, groups of 16 199 / 193 and 65 / 58, all rows in one group 175 / 25 and 57 / 9; 256 rows, 16 experts, k = n = 4096, groups of 16
        // 134 / 126 and 27 / 23, in one 87 / 42 and 28 / 11
        const long long scales = p->depth / kMx4Block;
        if ((p->rows + p->experts - 1) / p->experts <= 16 || (mx4 && (p->rows * scales < 16 || p->experts * (p->width * scales) < 16))) {
            p->tile = kFewRows;
            return;
        }
    }
    if (mx4) shortest(kForms4, direction, 256, p);
    else shortest(kForms16, direction, 64, p);
}

// 8-bit whole numbers: a chunk is 128 of them, and takes the loads, reads and products of one of 64 numbers of 16 bits.  k = n = 4096, us for 100 / 300 / 1000 / 2000 / 16384 (8 experts) rows: 256 x 256 44 / 45 / 47 / 48 /
// 253, 128 x 128 25 / 25 / 27 / 39 / 331, with four chunks in LDS 19 / 20 / 24 / 43 / 361, 64 x 64 11 / 16 / 32 / 60 / 507; n = 16384 with 16 / 17 rows 64 x 64 18.5 / 18.5, few rows 18.5 / 25.7
constexpr Form kForms8[] = {kForms16[0], kForms16[1], kForms16[2], {kTile64, 64, 0.18, 0.33, 4.4, 512}};

// The form for few rows, 16, 32 or 64 of the weights' rows a workgroup: time of a chunk, in as many rounds as workgroups of 16 rows need, or the weights' way from memory.
// 16 / 32 / 64, 64 x 64 tiles, us, k = 8192: 4 rows, n = 4096 8.9 / 12.2 / 19.1, 17.5, 5000 14.1 / 12.9 / 19.6, 21.0, 12288 20.5 / 23.0 / 22.2, 24.4; 16 rows, 4096 10.7 / 13.9 / 20.9, 18.1, 8192
// 18.6 / 15.7 / 21.7, 22.7; 32 rows, 2048 10.6 / 13.8 / 20.8, 16.1, 4096 17.7 / 14.6 / 21.3, 18.3, 8192 32 / 26 / 23, 23; 100 rows, 2048 31 / 25 / 23, 16.3; k = 512: 100 rows, 2048 5.2 / 5.1 / 5.0, 5.4,
// 4096 6.8 / 6.7 / 6.5, 5.5
int few_columns_int(const ProductParams& p, double* us)
{
    const bool scarce = p.rows <= 8LL * p.experts;
    const double chunk[] = {scarce ? 0.1 : 0.12, scarce ? 0.155 : 0.173, 0.3}, around[] = {2.7, 3.0, 3.2}, groups = p.experts < p.rows ? p.experts : p.rows;
    const double tiles = p.experts > 1 ? p.rows / 16.0 + 0.5 * groups : (p.rows + 15) / 16, memory = groups * p.width * p.depth / 5.5e6;
    int columns = 16;
    *us = 1e30;
    for (int i = 0; i < 3; ++i) {
        const int each = 16 << i;
        const double work = ceil((double)p.depth / 128) * chunk[i] * ceil(tiles * ((p.width + each - 1) / each) / 256), t = around[i] + (work > memory ? work : memory);
        if (t < *us) {
            *us = t;
            columns = each;
        }
    }
    return columns;
}

// (By the mean load, as only the GPU knows the groups.  Where all rows are in one group of many the form for few rows is far from the best, us: 1024 rows of 64 experts, 2048 to 4096, even 113 and 114 with tiles of
// 128 x 128, in one group 99 and 15; 256 rows of 16, 4096 to 4096, even 62 and 70 with 64 x 64, in one group 48 and 12.)
void plan_product_int(ProductParams* p)
{
    p->splits = 1;
    p->tile = kFewRows;
    if ((p->rows + p->experts - 1) / p->experts <= 16) return;
    double few;
    few_columns_int(*p, &few);
    if (shortest(kForms8, kForward, 128, p) > few) p->tile = kFewRows;
}

bool int_quantises_within(const ProductParams& p) { return quantises_within(p); }

bool quantises_within(const ProductParams& p)
{
    const int rows = p.rows < 16 ? p.rows : 16;
    return p.tile == kFewRows && rows * (long long)((p.depth + kChunk - 1) / kChunk) <= kRawChunks;
}

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
