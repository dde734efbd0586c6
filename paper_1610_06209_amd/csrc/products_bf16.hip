// Products of bf16 operands (see product_kernels.hpp).
#include "product_kernels.hpp"

namespace spinner {

hipError_t launch_product_bf16(int direction, int out_type, const ProductParams& p, hipStream_t s)
{
    switch (direction) {
    case kForward: return launch_product_as<kForward, kBf16, __bf16>(p, s);
    case kDx: return launch_product_as<kDx, kBf16, __bf16>(p, s);
    default:
        return out_type == kF32 ? launch_product_as<kDw, kBf16, float>(p, s) : launch_product_as<kDw, kBf16, __bf16>(p, s);
    }
}

}  // namespace spinner
