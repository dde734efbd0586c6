// Microscaled 4-bit floating point and grouped matrix products: what the host code and the kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace spinner {

// element types, in the order of spinner_dtype_t; kMx4 is internal (4-bit operands)
enum { kF32 = 0, kBf16 = 1, kF16 = 2, kMx4 = 3 };

constexpr int kMx4Block = 32;             // numbers that share a scale
constexpr int kMaxRotation = 4096;        // longest run of coordinates that one rotation mixes
constexpr int kMaxExperts = 1024;

struct QuantizeParams {
    const void* x;
    const float* diag;                    // null: all ones
    uint8_t* codes;
    uint8_t* scales;
    long long x_stride;                   // elements
    int rows, k;
};
// block: 0 (no rotation) or a power of two in [32, kMaxRotation]
hipError_t launch_mx4_quantize(const QuantizeParams& p, int dtype, int block, hipStream_t s);
hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int rows, int k, void* out, int dtype,
                                 long long out_stride, hipStream_t s);

// The three products of a layer with weights w[expert][n][k] on rows that are grouped by expert (group e: rows
// [ends[e - 1], ends[e]); without ends all rows are one group):
enum { kForward = 0,      // out[row][n] = sum_k a[row][k] b[e][n][k]
       kDx = 1,           // out[row][k] = sum_n a[row][n] b[e][n][k]
       kDw = 2 };         // out[e][n][k] = sum_row a[row][n] b[row][k]
struct ProductParams {
    const char* a;                        // operand of the result's rows
    const char* b;                        // operand of the result's columns
    const uint8_t* a_scales;              // kMx4
    const uint8_t* b_scales;
    char* out;
    const long long* ends;                // null: one group
    long long a_stride, b_stride;         // bytes from one row of the operand, as it lies, to the next
    long long b_group;                    // kForward, kDx: bytes from one expert's weights to the next
    long long out_stride;                 // elements from one row of the result to the next
    int rows, experts;
    unsigned first_block;                 // (kernels) workgroup 0 of this grid in the order of all
    int height;                           // kDw: rows of one expert's result
    int width;                            // columns of the result
    int depth;                            // kForward, kDx: numbers in a sum
    int tile;                             // form of the kernel, see plan_product
    int splits;                           // shares of the depth that workgroups of their own sum up (kDw; 1: whole sums)
    long long split_stride;               // (kernels) numbers from one share's partial results to the next
    void* workspace;                      // fp32 [splits][rows of the result][width], splits > 1
};
// Forms of the product: a few rows a group; tiles of 256 x 256, 128 x 128 with two or four chunks in LDS, 64 x 64.
enum { kFewRows, kTile256, kTile128, kTile128Deep, kTile64 };
// The form (and, kDw, the shares of the depth) that takes the shortest by what was measured of each: p.tile and p.splits.  It goes by the sizes alone: the
// rows of each expert are known on the GPU only.
void plan_product(int direction, bool mx4, ProductParams* p);
inline size_t product_workspace(const ProductParams& p)      // bytes of partial sums, kDw
{
    return p.splits > 1 ? (size_t)p.splits * p.experts * p.height * p.width * sizeof(float) : 0;
}

// Rows that the product's kernel quantises for itself.
struct RawRows {
    const void* x;                        // of the result's type
    const float* diag;
    long long stride;                     // elements
    float norm;                           // 1 / sqrt(2^log)
    int log;                              // runs of 2^log coordinates; 0: no rotation
};
constexpr int kRawChunks = 8;             // chunks of 512 numbers that a workgroup's eight waves quantise, one each
// whether a group's rows are so few that every workgroup of the product does
bool quantises_within(const ProductParams& p);
hipError_t launch_product_raw(int type, const ProductParams& p, const RawRows& raw, hipStream_t s);

hipError_t launch_product_mx4(int out_type, const ProductParams& p, hipStream_t s);           // kForward
hipError_t launch_product_bf16(int direction, int out_type, const ProductParams& p, hipStream_t s);
hipError_t launch_product_f16(int direction, int out_type, const ProductParams& p, hipStream_t s);

}  // namespace spinner
