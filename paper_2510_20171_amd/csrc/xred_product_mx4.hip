// xred_product_mx4.hip -- the experts' products in mx4 (e2m1 with exponents by 32).
#include "xred_product_choice.hpp"

namespace xred {

hipError_t launch_product_mx4(const ProductParams &p, hipStream_t s)
{
    return launch_product_scaled<PMx4>(p, s);
}

}  // namespace xred
