// Rotation and quantisation to microscaled 4-bit floating point (e2m1 with a shared power of two for each 32 numbers), and back.
#include <math.h>

#include "mx4.hpp"
#include "number_io.hpp"
#include "spinner_kernels.hpp"

namespace spinner {
namespace {

constexpr int kPieceNumbers = 8;                         // numbers of a lane
constexpr int kChunk = 64 * kPieceNumbers;               // numbers of a wave that lie side by side
constexpr int waves_of_run(int log) { return log > 9 ? 1 << (log - 9) : 1; }

// undoes the trade of lane_swap_stage
template <int LANE_BIT, int Q, int R>
__device__ __forceinline__ void swap_back(float (&v)[R])
{
#pragma unroll
    for (int j = 0; j < R; ++j)
        if (!(j & (1 << Q))) lane_swap<LANE_BIT>(v[j], v[j | (1 << Q)]);
}

// Rows [rows][k] to codes and scales, v = H D x on each run of 2^LOG coordinates first (LOG = 0: v = x).
// A lane holds eight numbers: eight neighbours of 16 bits, or four and the four 256 further on in fp32, 16 bytes each (eight fp32 neighbours, whose two
// loads take every second piece of a line, 16384 x 16384: 254 us; so 214).  Index bits up to 2^8 then are register and lane bits; those above
// are of the wave in its workgroup.  Butterflies in fp32; lane bits 4 and 5 trade places with register bits 1 and 2 for their stage, and
// the waves of a run meet in LDS, where each lane sums up the 2^(LOG - 9) numbers of its place with their signs (in registers alone, 64
// numbers a lane at 2^12, a wave's 240 registers left one wave a SIMD: one row of 4096 12.9 us, here 3.5).  The transform's 1 / sqrt(2^LOG) goes into
// the diagonal.  A scale is shared by four (fp32: eight) neighbouring lanes: the largest magnitude as a whole number (so that a NaN is larger
// than an infinity and both larger than any number) gives the exponent.
// A wave stays with its columns, whose diagonal it keeps, and goes down the rows, the next row's numbers asked for ahead.
// Measured, bf16 16384 x 8192 (340 MB): no rotation 58 us, 5.9 TB/s (the copy rate is 6.2), runs of 512 82 us (bound by the vector ALU: 15 instructions
// a number), 1024 90, 4096 112 (the sums in LDS).
template <typename T, int LOG>
__global__ void __launch_bounds__(LOG > 9 ? 64 * waves_of_run(LOG) : 256) mx4_quantize_kernel(QuantizeParams p, int column_groups, int row_step)
{
    constexpr int WAVES = waves_of_run(LOG);
    constexpr int N = kPieceNumbers, HALVES = sizeof(T) == 4 ? 2 : 1, LOW = HALVES == 2 ? 2 : 3;      // index bit of lane bit 0
    __shared__ float4 meeting[WAVES > 1 ? 2 : 1][WAVES > 1 ? WAVES * 128 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int unit = WAVES > 1 ? (int)blockIdx.x : (int)blockIdx.x * 4 + wave;
    const int group = unit % column_groups;
    int row = unit / column_groups;
    if (row >= row_step) return;
    // columns of the lane's numbers, 16 bytes of them each; what is not live (a whole run of coordinates is or is not) is read from the row's first
    const int first = (WAVES > 1 ? group * WAVES + wave : group) * kChunk + (lane << LOW);
    int safe[HALVES];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) safe[h] = first + h * 256 < p.k ? first + h * 256 : 0;
    // which lanes' numbers a transform leaves negated (see lane_stage_fmac_dpp): a product of those of lane bits 0, 1 and 3 that it has
    constexpr int negating = (LOG > LOW) | (LOG > LOW + 1) << 1 | (LOG > LOW + 3) << 3;
    const unsigned flip = __popc(lane & negating) & 1 ? 0x88888888u : 0u;
    float d[N];
    if constexpr (LOG > 0) {
        const float norm = 1.0f / __builtin_sqrtf((float)(1 << LOG));
        if (p.diag) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 a = *reinterpret_cast<const float4*>(p.diag + (HALVES == 2 ? safe[h % HALVES] : safe[0] + 4 * h));
                d[4 * h] = a.x * norm; d[4 * h + 1] = a.y * norm; d[4 * h + 2] = a.z * norm; d[4 * h + 3] = a.w * norm;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) d[i] = norm;
        }
    }
    const T* x = static_cast<const T*>(p.x);
    Quad raw[HALVES];
    const auto fetch = [&](int r) {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) raw[h] = stream_quad(x + r * p.x_stride + safe[h]);
    };
    fetch(row);
    for (int turn = 0; row < p.rows; ++turn) {
        float v[N];
        widen_quads<T>(raw, v);
        const int at = row;
        row += row_step;
        if (row < p.rows) fetch(row);
        if constexpr (LOG > 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= d[i];
            static_for<0, LOW>([&](auto q) { reg_stage<q.value>(v); });
            if constexpr (HALVES == 2 && LOG > 8) reg_stage<2>(v);
            // (lane bits 0, 1 and 3 in one instruction a number, which leaves the upper lane's difference negated)
            static_for<0, 4>([&](auto b) {
                if constexpr (LOG > LOW + b.value) {
                    const float coef = (lane >> b.value) & 1 ? -1.0f : 1.0f;
                    if constexpr (b.value == 2) lane_stage<2>(v, coef);
                    else lane_stage_fmac_dpp<b.value>(v, coef);
                }
            });
            if constexpr (LOG > LOW + 4) { lane_swap_stage<4, 1>(v); swap_back<4, 1>(v); }
            if constexpr (LOG > LOW + 5) { lane_swap_stage<5, 2>(v); swap_back<5, 2>(v); }
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
        unsigned code[HALVES];
        int byte[HALVES];
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
            if constexpr (LOG > 0) c ^= flip;
            code[h] = e == 255 ? 0 : c;
        }
        // eight codes a lane side by side: fp32 lanes come by theirs in pairs, the even one of the first half
        const bool odd = HALVES == 2 && (lane & 1);
        int col = first;
        if constexpr (HALVES == 2) {
            const unsigned own = (odd ? code[HALVES - 1] : code[0]) & 0xffff, got = lane_xor_i<1>(odd ? code[0] : code[HALVES - 1]) & 0xffff;
            code[0] = odd ? got | own << 16 : own | got << 16;
            col = odd ? first - 4 + 256 : first;
        }
        const long long place = (long long)at * p.k;
        if (col < p.k) *reinterpret_cast<unsigned*>(p.codes + ((place + col) >> 1)) = code[0];
        if ((lane & ((32 >> LOW) - 1)) == 0)
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
                if (first + h * 256 < p.k) p.scales[(place + first + h * 256) >> 5] = (uint8_t)byte[h];
    }
}

// Codes back to numbers, 16 bytes of them a thread (STRIDED: rows of `out` that do not follow one another).  bf16 16384 x 16384 128 us, 5.3 TB/s.
template <typename T, bool STRIDED>
__global__ void __launch_bounds__(256) mx4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, long long pieces,
                                                             int row_pieces, T* __restrict__ out, long long out_stride)
{
    constexpr int M = 16 / sizeof(T);
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
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
    // waves enough to fill the chip, no more than rows; each then goes down several rows (runs of 512, bf16 16384 x 8192: 8192 waves 85 us, 16384 82; no
    // rotation, runs of 1024: the same)
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
    const long long blocks = (pieces + 255) / 256;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidConfiguration;
    const auto kernel = out_stride == k || rows == 1 ? mx4_dequantize_kernel<T, false> : mx4_dequantize_kernel<T, true>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, s, codes, scales, pieces, k / numbers, static_cast<T*>(out), out_stride);
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
