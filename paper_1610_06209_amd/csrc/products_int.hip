// Products of 8-bit whole numbers (see product_kernels.hpp).
#include "product_kernels.hpp"

namespace spinner {

hipError_t launch_product_int(int out_type, const ProductParams& p, hipStream_t s)
{
    switch (out_type) {
    case kF32: return launch_product_as<kForward, kInt8, float>(p, s);
    case kBf16: return launch_product_as<kForward, kInt8, __bf16>(p, s);
    default: return launch_product_as<kForward, kInt8, _Float16>(p, s);
    }
}

hipError_t launch_product_int_raw(int type, const ProductParams& p, const RawRows& raw, hipStream_t s)
{
    switch (type) {
    case kF32: return launch_few_rows_as<kInt8, float, true>(p, raw, s);
    case kBf16: return launch_few_rows_as<kInt8, __bf16, true>(p, raw, s);
    default: return launch_few_rows_as<kInt8, _Float16, true>(p, raw, s);
    }
}

}  // namespace spinner
