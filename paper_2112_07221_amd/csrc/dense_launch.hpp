// Which kernel a call takes, and its launch (dense_product.hip, dense_norm.hip).
#pragma once
#include "dense_product.hpp"
#include "dense_rows.hpp"

namespace het {

struct ProductPlan {
    bool ok;                    // the grid fits
    int small_m, small_n;       // 16-row and -column tiles of product_small_kernel's workgroups; 0: another kernel
    bool aligned;               // product_kernel, else product_any_kernel
    int tile;                   // its tile's edge
    int m, n, k, splits, k_split;
    int64_t partial_bytes;
};

// D[m][n] over k; `a_k`, `b_k`: the operands are read along k.  type: HET_F32, ...
// aligned: both operands are as product_copies asks.
ProductPlan product_plan(int64_t m, int64_t n, int64_t k, int type, bool a_k, bool b_k, bool aligned);
bool product_copies(const void *p, int64_t ld, int width, int type);

// Fills in the sizes of `a` and enqueues the product.
void launch_product(ProductArgs a, const ProductPlan &p, int type, bool a_k, bool b_k, hipStream_t st);

// How layer norm's rows lie: RowShape, rows a workgroup holds at a time, chunks a lane.
struct NormShape {
    RowShape s;
    int rows, nv;
    bool block;
};

NormShape norm_shape(int dim);
template <typename TX, typename TY> void launch_norm(const NormArgs &a, const NormShape &h, hipStream_t st);
template <typename TX, typename TY> void launch_norm_back(const NormBackArgs &a, const NormShape &h, int groups, hipStream_t st);

} // namespace het
