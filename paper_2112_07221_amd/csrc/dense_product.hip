// Launches of the matrix products; compiled in one part for each type (HET_PART: HET_F32, HET_BF16, HET_F16), the first with the plan.
#include "../../include/het_dense.h"

#include <algorithm>

#include "dense_launch.hpp"

#define HET_PRODUCT_PARTS 3
static_assert(HET_PARTS == HET_PRODUCT_PARTS, "the build compiles other parts than there are: kernels would be missing in the library");

namespace het {

template <typename T> void launch_product_of(const ProductArgs &a, const ProductPlan &p, bool a_k, bool b_k, hipStream_t st);

#if HET_PART == 0
using PartType = float;
#elif HET_PART == 1
using PartType = bf16;
#else
using PartType = f16;
#endif

template <typename T, int NT>
static void launch_few(const ProductArgs &a, int mt, hipStream_t st)
{
    const uint32_t grid = (uint32_t)((a.n + 16 * NT - 1) / (16 * NT));
    if (mt == 1) product_few_kernel<T, 1, NT><<<grid, 64 * FEW_WAVES, 0, st>>>(a);
    else if (mt == 2) product_few_kernel<T, 2, NT><<<grid, 64 * FEW_WAVES, 0, st>>>(a);
    else product_few_kernel<T, 4, NT><<<grid, 64 * FEW_WAVES, 0, st>>>(a);
}

template <typename T>
void launch_product_of(const ProductArgs &a, const ProductPlan &p, bool a_k, bool b_k, hipStream_t st)
{
    if (p.few) {
        if (a.f.q) launch_few<T, 2>(a, p.few, st);
        else launch_few<T, 1>(a, p.few, st);
        return;
    }
    const uint32_t grid = (uint32_t)(a.tiles_m * a.tiles_n * a.splits);
    if (a_k && b_k) product_any_kernel<T, true, true><<<grid, 256, 0, st>>>(a);
    else if (a_k) product_any_kernel<T, true, false><<<grid, 256, 0, st>>>(a);
    else product_any_kernel<T, false, false><<<grid, 256, 0, st>>>(a);
    if (a.splits > 1) {
        const int64_t per = (a.n + PACK_BLOCK - 1) / PACK_BLOCK * 4;
        join_kernel<T><<<(uint32_t)((a.m * per + 255) / 256), 256, 0, st>>>(a);
    }
}

template void launch_product_of<PartType>(const ProductArgs &, const ProductPlan &, bool, bool, hipStream_t);

#if HET_PART == 0
extern template void launch_product_of<bf16>(const ProductArgs &, const ProductPlan &, bool, bool, hipStream_t);
extern template void launch_product_of<f16>(const ProductArgs &, const ProductPlan &, bool, bool, hipStream_t);

constexpr int FEW_ROWS = 64;
constexpr int CUS = 256;

ProductPlan product_plan(int64_t m, int64_t n, int64_t k, int type, bool a_k, bool b_k)
{
    ProductPlan p{};
    p.m = (int)m; p.n = (int)n; p.k = (int)k;
    p.splits = 1; p.k_split = (int)k;
    p.ok = true;
    if (a_k && b_k && m <= FEW_ROWS) {
        p.few = m <= 16 ? 1 : m <= 32 ? 2 : 4;
        return p;
    }
    const int64_t step = type == HET_F32 ? 32 : 64, steps = (k + step - 1) / step;
    const int64_t tm = (m + ANY_TILE - 1) / ANY_TILE, tn = (n + ANY_TILE - 1) / ANY_TILE, tiles = tm * tn;
    if (tiles < CUS && steps > 8) p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({2 * CUS / std::max<int64_t>(tiles, 1), steps / 4, 16}));
    p.k_split = (int)((steps + p.splits - 1) / p.splits * step);
    p.splits = (int)std::max<int64_t>(1, (k + p.k_split - 1) / std::max(p.k_split, 1));
    p.tiles_m = (int)tm; p.tiles_n = (int)std::min<int64_t>(tn, INT32_MAX);
    p.ok = tiles * p.splits <= INT32_MAX && m * ((n + 31) / 32 * 4) / 256 < INT32_MAX;
    p.partial_bytes = p.splits > 1 ? p.splits * m * (int64_t)((n + 15) / 16 * 16) * 4 : 0;
    return p;
}

void launch_product(ProductArgs a, const ProductPlan &p, int type, bool a_k, bool b_k, hipStream_t st)
{
    a.m = p.m; a.n = p.n; a.k = p.k;
    a.tiles_m = p.tiles_m; a.tiles_n = p.tiles_n; a.splits = p.splits; a.k_split = p.k_split;
    if (type == HET_F32) launch_product_of<float>(a, p, a_k, b_k, st);
    else if (type == HET_BF16) launch_product_of<bf16>(a, p, a_k, b_k, st);
    else launch_product_of<f16>(a, p, a_k, b_k, st);
}
#endif

} // namespace het
