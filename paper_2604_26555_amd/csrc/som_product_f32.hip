#include "som_product_launch.hpp"

namespace som {

template int product_typed<float>(som_ctx* ctx, const NodeProduct& p);
template int product_grad_typed<float>(som_ctx* ctx, const NodeProductGrad& p);

} // namespace som
