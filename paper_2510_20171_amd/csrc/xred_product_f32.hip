// xred_product_f32.hip -- the experts' products in f32.
#include "xred_product_choice.hpp"

namespace xred {

hipError_t launch_product_f32(const ProductParams &p, bool grad, bool across, hipStream_t s)
{
    return launch_product_plain<PF32>(p, grad, across, s);
}

}  // namespace xred
