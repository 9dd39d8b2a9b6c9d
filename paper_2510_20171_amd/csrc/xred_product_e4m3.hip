// xred_product_e4m3.hip -- the experts' products in e4m3 with scales by 128 elements.
#include "xred_product_choice.hpp"

namespace xred {

hipError_t launch_product_e4m3(const ProductParams &p, hipStream_t s)
{
    return launch_product_scaled<PE4M3>(p, s);
}

}  // namespace xred
