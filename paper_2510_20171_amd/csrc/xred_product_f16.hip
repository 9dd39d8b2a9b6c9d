// xred_product_f16.hip -- the experts' products in f16.
#include "xred_product_choice.hpp"

namespace xred {

hipError_t launch_product_f16(const ProductParams &p, bool grad, bool across, hipStream_t s)
{
    return launch_product_plain<PF16>(p, grad, across, s);
}

}  // namespace xred
