#include "som_product_launch.hpp"

namespace som {

template int product_typed<_Float16>(som_ctx* ctx, const NodeProduct& p);
template int product_grad_typed<_Float16>(som_ctx* ctx, const NodeProductGrad& p);

} // namespace som
