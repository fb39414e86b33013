// Which kernel a call takes, and its launch (dense_product.hip, dense_norm.hip).
#pragma once
#include <algorithm>

#include "dense_product.hpp"

namespace het {

// A launch's threads are counted in 32 bits.  Rows of `threads` threads each go in launches of at most 2^31 (and, but for the last, of a
// multiple of 256 rows, so that no workgroup lies in two): f(first row, rows).
template <typename F>
void in_launches(int64_t rows, int64_t threads, F &&f)
{
    const int64_t most = std::max<int64_t>((1ll << 31) / threads / 256 * 256, 256);
    for (int64_t first = 0; first < rows; first += most) f(first, std::min(most, rows - first));
}

// `p` moved on by a number of values of `size` bytes; null stays null.
template <typename P> P *moved(P *p, int64_t values, int64_t size)
{
    return p ? reinterpret_cast<P *>(reinterpret_cast<uintptr_t>(p) + (uintptr_t)(values * size)) : p;
}

struct ProductPlan {
    bool ok;                    // the grid fits
    int small_m, small_n;       // 16-row and -column tiles of product_small_kernel's workgroups; 0: product_kernel
    int tile;                   // its tile's edge
    bool lay_a, lay_b;          // which operands are laid out for it first
    int m, n, k, splits, k_split;
    int64_t partial_bytes;
};

// D[m][n] over k; `a_k`, `b_k`: the operands are read along k; `lay_a`, `lay_b`: what laying them out takes
// (us; 0: they are as product_lies asks).  type: HET_F32, ...
ProductPlan product_plan(int64_t m, int64_t n, int64_t k, int type, bool a_k, bool b_k, double lay_a, double lay_b);
double lay_us(bool lies, int64_t rows, int64_t width, int type);
double written_us(bool lies, int64_t rows, int64_t width, int type);
bool product_lies(const void *p, int64_t ld, int64_t width, int type);

// Rows of `width` values as product_kernel takes them: values from a row to the next, and their launch.
int64_t laid_pitch(int64_t width, int type);
void launch_lay(const void *p, int64_t ld, int64_t rows, int width, void *to, int type, hipStream_t st);

// Both products of a small layer's backward pass and the sums of dbias' parts (bias.n: 0 for none) in one launch; false if they are not for one, and
// nothing is enqueued.
bool launch_small_back(ProductArgs dw, const ProductPlan &dw_plan, ProductArgs dx, const ProductPlan &dx_plan, const ColumnSumArgs &bias, int type, hipStream_t st);

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
