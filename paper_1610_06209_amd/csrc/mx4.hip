// Rotation and quantisation to microscaled 4-bit floating point (e2m1 with a shared power of two for each 32 numbers), and back.
#include <math.h>

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
// A lane holds eight neighbours, so index bits 0..2 are register bits and 3..8 lane bits; bits above 2^9 are those of the wave in its
// workgroup.  Butterflies in fp32; lane bits 4 and 5 trade places with register bits 1 and 2 for their stage, and the waves of a run meet in LDS,
// where each lane sums up the 2^(LOG - 9) numbers of its place with their signs (in registers alone, 64 numbers a lane at 2^12, a wave's
// 240 registers left one wave a SIMD: one row of 4096 12.9 us, here 5.5).  The transform's 1 / sqrt(2^LOG) goes into the diagonal.  A scale
// is shared by four neighbouring lanes: the largest magnitude as a whole number (so that a NaN is larger than an infinity and both larger
// than any number) gives the exponent.
// A wave stays with its columns, whose diagonal it keeps, and goes down the rows, the next row's numbers asked for ahead.
template <typename T, int LOG>
__global__ void __launch_bounds__(LOG > 9 ? 64 << (LOG - 9) : 256) mx4_quantize_kernel(QuantizeParams p, int column_groups, int row_step)
{
    constexpr int WAVES = LOG > 9 ? 1 << (LOG - 9) : 1;                  // of a run
    constexpr int N = kPieceNumbers;
    __shared__ float4 meeting[WAVES > 1 ? 2 : 1][WAVES > 1 ? WAVES * 128 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = WAVES > 1 ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave;
    const int group = unit % column_groups;
    int row = unit / column_groups;
    if (row >= row_step) return;
    const int col = (WAVES > 1 ? group * WAVES + wave : group) * kChunk + lane * N;
    const bool live = col < p.k;                                         // a whole run of coordinates is live or is not
    const int safe = live ? col : 0;
    // which lanes' numbers a transform leaves negated (see lane_stage_fmac_dpp): a product of lane bits 0, 1 and 3
    const unsigned flip = __popc(lane & (LOG > 6 ? 0xB : (LOG > 4 ? 3 : 1))) & 1 ? 0x88888888u : 0u;
    float d[N];
    if constexpr (LOG > 0) {
        const float norm = 1.0f / __builtin_sqrtf((float)(1 << LOG));
        if (p.diag) {
            const float4 a = reinterpret_cast<const float4*>(p.diag + safe)[0], b = reinterpret_cast<const float4*>(p.diag + safe)[1];
            d[0] = a.x * norm; d[1] = a.y * norm; d[2] = a.z * norm; d[3] = a.w * norm;
            d[4] = b.x * norm; d[5] = b.y * norm; d[6] = b.z * norm; d[7] = b.w * norm;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = norm;
        }
    }
    const T* x = static_cast<const T*>(p.x) + safe;
    typename Piece<T>::Raw raw = Piece<T>::fetch(x + row * p.x_stride);
    for (int turn = 0; row < p.rows; ++turn) {
        float v[N];
        Piece<T>::widen(raw, v);
        const int at = row;
        row += row_step;
        if (row < p.rows) raw = Piece<T>::fetch(x + row * p.x_stride);
        if constexpr (LOG > 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= d[i];
            static_for<0, 3>([&](auto q) { reg_stage<q.value>(v); });
            // (lane bits 0, 1 and 3 in one instruction a number, which leaves the upper lane's difference negated)
            static_for<0, 4>([&](auto b) {
                if constexpr (LOG > 3 + b.value) {
                    const float coef = (lane >> b.value) & 1 ? -1.0f : 1.0f;
                    if constexpr (b.value == 2) lane_stage<2>(v, coef);
                    else lane_stage_fmac_dpp<b.value>(v, coef);
                }
            });
            if constexpr (LOG > 7) { lane_swap_stage<4, 1>(v); swap_back<4, 1>(v); }
            if constexpr (LOG > 8) { lane_swap_stage<5, 2>(v); swap_back<5, 2>(v); }
        }
        if constexpr (WAVES > 1) {
            float4* m = meeting[turn & 1];           // the other one may still be read
            m[wave * 128 + lane] = make_float4(v[0], v[1], v[2], v[3]);
            m[wave * 128 + 64 + lane] = make_float4(v[4], v[5], v[6], v[7]);
            __syncthreads();
            float t[N];
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float4 a = m[w * 128 + lane], b = m[w * 128 + 64 + lane];
                const float sign = __popc(w & wave) & 1 ? -1.0f : 1.0f;
                const float u[N] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
                for (int i = 0; i < N; ++i) t[i] = w == 0 ? u[i] : __builtin_fmaf(u[i], sign, t[i]);
            }
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = t[i];
        }
        // the largest magnitude, numbers taken as they lie: positive ones in the order of signed whole numbers, negative ones above them in
        // that of unsigned ones
        int above = __float_as_int(v[0]);
        unsigned below = __float_as_uint(v[0]);
#pragma unroll
        for (int i = 1; i < N; ++i) {
            const int a = __float_as_int(v[i]);
            above = a > above ? a : above;
            below = (unsigned)a > below ? (unsigned)a : below;
        }
        int top = (int)(below & 0x7fffffffu);
        top = above > top ? above : top;
        int other = lane_xor_i<1>(top);
        top = other > top ? other : top;
        other = lane_xor_i<2>(top);
        top = other > top ? other : top;
        const int e = top >> 23;                                         // largest magnitude: 2^(e - 127) and more
        const int byte = e == 255 ? 255 : (e > 2 ? e - 2 : 0);
        const float scale = exponent_value(byte);
        unsigned code = 0;
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[0], v[1], scale, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[2], v[3], scale, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[4], v[5], scale, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, v[6], v[7], scale, 3);
        if constexpr (LOG > 3) code ^= flip;
        if (e == 255) code = 0;
        if (live) {
            const long long place = (long long)at * p.k + col;
            *reinterpret_cast<unsigned*>(p.codes + (place >> 1)) = code;
            if ((lane & 3) == 0) p.scales[place >> 5] = (uint8_t)byte;
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
    constexpr int waves = LOG > 9 ? 1 << (LOG - 9) : 1, width = waves * kChunk;
    const int groups = (p.k + width - 1) / width;
    // waves enough to fill the chip, no more than rows; each then goes down several rows
    const int want = (8192 / waves + groups - 1) / groups;
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
    const long long pieces = (long long)rows * (k / kPieceNumbers);
    const long long blocks = (pieces + 255) / 256;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const auto kernel = out_stride == k || rows == 1 ? mx4_dequantize_kernel<T, false> : mx4_dequantize_kernel<T, true>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, s, reinterpret_cast<const unsigned*>(codes), scales, pieces,
                       k / kPieceNumbers, static_cast<T*>(out), out_stride);
    return hipGetLastError();
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
constexpr int kHeldDepth = 8192;                 // 64 x 64 tiles hold the scales of so many 4-bit numbers of a row
constexpr size_t kMostPartial = 64u << 20;       // bytes of partial sums

template <int N>
static void shortest(const Form (&forms)[N], int direction, bool mx4, ProductParams* p)
{
    double best = 1e30;
    for (const Form& f : forms) {
        if (mx4 && f.tile == kTile64 && p->depth > kHeldDepth) continue;
        double tiles = (p->width + f.side - 1) / f.side, chunks;
        if (direction == kDw) {
            tiles *= (double)((p->height + f.side - 1) / f.side) * p->experts;
            // the longest group of several, taken as half as long again as they are on average
            chunks = ceil(p->rows * (p->experts > 1 ? 1.5 : 1.0) / p->experts / 64);
        } else {
            // a group's last tile is half full on average
            tiles *= p->experts > 1 ? (double)p->rows / f.side + 0.5 * (p->experts < p->rows ? p->experts : p->rows) : (p->rows + f.side - 1) / f.side;
            chunks = ceil(p->depth / (mx4 ? 256.0 : 64.0));
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
}

void plan_product(int direction, bool mx4, ProductParams* p)
{
    p->splits = 1;
    if (direction == kForward) {
        // up to sixteen rows a group the weights' way from memory is all (4 bits, n = 16384, k = 4096, 16 rows: 9.8 us, 64 x 64 tiles 10.7; 32 rows: 15.2, 10.8);
        // and tiles read 4-bit operands' scales sixteen at a time
        const long long scales = p->depth / kMx4Block;
        if ((p->rows + p->experts - 1) / p->experts <= 16 || (mx4 && (p->rows * scales < 16 || p->experts * (p->width * scales) < 16))) {
            p->tile = kFewRows;
            return;
        }
    }
    if (mx4) shortest(kForms4, direction, true, p);
    else shortest(kForms16, direction, false, p);
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
