// Rows as 8-bit whole numbers with a scale each: what the host code and the kernels share.
#pragma once
#include "mx4.hpp"

namespace spinner {

constexpr int kIntPiece = 16;                        // codes of a row come in whole pieces of so many, zeros behind the numbers
constexpr int kMostIntDepth = (1 << 17) - kIntPiece; // numbers of a sum: 2^17 products of -128 and -128 would leave 32 bits
constexpr float kSmallestScale = 1.17549435e-38f;    // 2^-126
inline int int_width(int k) { return (k + kIntPiece - 1) / kIntPiece * kIntPiece; }

struct IntQuantizeParams {
    const void* x;
    const float* diag;                    // null: all ones
    int8_t* codes;                        // [slots][width]
    float* scales;                        // [slots]
    const int* places;                    // [rows][top]; null: row r to slot r
    long long x_stride;                   // elements
    int rows, k, width, top;
    float norm;                           // 1 / sqrt(2^log)
    int log;                              // runs of 2^log coordinates; 0: no rotation
};
hipError_t launch_int_quantize(const IntQuantizeParams& p, int dtype, hipStream_t s);
hipError_t launch_int_dequantize(const int8_t* codes, const float* scales, int rows, int k, void* out, int dtype, long long out_stride, hipStream_t s);

void plan_product_int(ProductParams* p);
// weights' rows that a workgroup of the form for few rows takes: 16, 32 or 64; *us: about what that form takes
int few_columns_int(const ProductParams& p, double* us);
hipError_t launch_product_int(int out_type, const ProductParams& p, hipStream_t s);           // kForward
// rows that the product's kernel quantises for itself
bool int_quantises_within(const ProductParams& p);
hipError_t launch_product_int_raw(int type, const ProductParams& p, const RawRows& raw, hipStream_t s);

}  // namespace spinner
