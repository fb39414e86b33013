// Which kernel a call takes, and its launch (dense_product.hip, dense_norm.hip).
#pragma once
#include "dense_product.hpp"
#include "dense_rows.hpp"

namespace het {

struct ProductPlan {
    bool ok;                    // the grid fits
    int small_m, small_n;       // 16-row and -column tiles of product_small_kernel's workgroups; 0: product_kernel
    int tile;                   // its tile's edge
    bool lay_a, lay_b;          // which operands are laid out for it first
    int m, n, k, splits, k_split;
    int64_t partial_bytes;
};

// D[m][n] over k; `a_k`, `b_k`: the operands are read along k; `lies_a`, `lies_b`: they are as product_lies asks.  type: HET_F32, ...
ProductPlan product_plan(int64_t m, int64_t n, int64_t k, int type, bool a_k, bool b_k, bool lies_a, bool lies_b);
bool product_lies(const void *p, int64_t ld, int64_t width, int type);

// Rows of `width` values as product_kernel takes them: values from a row to the next, and their launch.
int64_t laid_pitch(int64_t width, int type);
void launch_lay(const void *p, int64_t ld, int64_t rows, int width, void *to, int type, hipStream_t st);

// Fills in the sizes of `a` and enqueues the product.
void launch_product(ProductArgs a, const ProductPlan &p, int type, bool a_k, bool b_k, hipStream_t st);

// How layer norm's rows lie: RowShape, rows a workgroup holds at a time, chunks a lane, the backward pass' workgroups at most.
struct NormShape {
    RowShape s;
    int rows, nv, groups;
    bool block;
};

NormShape norm_shape(int dim);
template <typename TX, typename TY> void launch_norm(const NormArgs &a, const NormShape &h, hipStream_t st);
template <typename TX, typename TY> void launch_norm_back(const NormBackArgs &a, const NormShape &h, int groups, hipStream_t st);

} // namespace het
