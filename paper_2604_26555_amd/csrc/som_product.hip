// Products with the nodes' matrices: the element type's own kernels (som_product_tile.hpp, som_product_narrow.hpp, som_product_launch.hpp), which are compiled one type a unit.
#include "som_internal.hpp"

namespace som {

template <class T>
int product_typed(som_ctx* ctx, const NodeProduct& p);
template <class T>
int product_grad_typed(som_ctx* ctx, const NodeProductGrad& p);
extern template int product_typed<float>(som_ctx*, const NodeProduct&);
extern template int product_typed<__bf16>(som_ctx*, const NodeProduct&);
extern template int product_typed<_Float16>(som_ctx*, const NodeProduct&);
extern template int product_grad_typed<float>(som_ctx*, const NodeProductGrad&);
extern template int product_grad_typed<__bf16>(som_ctx*, const NodeProductGrad&);
extern template int product_grad_typed<_Float16>(som_ctx*, const NodeProductGrad&);

int node_product_run(som_ctx* ctx, int type, const NodeProduct& p)
{
    if (p.rows == 0) return SOM_OK;
    if (type == SOM_ROWS_FLOAT) return product_typed<float>(ctx, p);
    if (type == SOM_ROWS_BFLOAT) return product_typed<__bf16>(ctx, p);
    return product_typed<_Float16>(ctx, p);
}

int node_product_grad_run(som_ctx* ctx, int type, const NodeProductGrad& p)
{
    if (type == SOM_ROWS_FLOAT) return product_grad_typed<float>(ctx, p);
    if (type == SOM_ROWS_BFLOAT) return product_grad_typed<__bf16>(ctx, p);
    return product_grad_typed<_Float16>(ctx, p);
}

} // namespace som
