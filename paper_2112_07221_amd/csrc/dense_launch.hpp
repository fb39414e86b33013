// Which kernel a product takes, and its launch (dense_product.hip).
#pragma once
#include "dense_product.hpp"

namespace het {

struct ProductPlan {
    bool ok;                    // the grid fits
    int few;                    // 16-row tiles of the kernel for few rows; 0: tiles of product_any_kernel
    int m, n, k, tiles_m, tiles_n, splits, k_split;
    int64_t partial_bytes;
};

// D[m][n] over k; `a_k`, `b_k`: the operands are read along k.  type: HET_F32, ...
ProductPlan product_plan(int64_t m, int64_t n, int64_t k, int type, bool a_k, bool b_k);

// Fills in the sizes of `a` and enqueues the product.
void launch_product(ProductArgs a, const ProductPlan &p, int type, bool a_k, bool b_k, hipStream_t st);

} // namespace het
