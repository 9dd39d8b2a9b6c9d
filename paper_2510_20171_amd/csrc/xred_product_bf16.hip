// xred_product_bf16.hip -- the experts' products in bf16.
#include "xred_product_choice.hpp"

namespace xred {

hipError_t launch_product_bf16(const ProductParams &p, bool grad, bool across, hipStream_t s)
{
    return launch_product_plain<PBF16>(p, grad, across, s);
}

}  // namespace xred
