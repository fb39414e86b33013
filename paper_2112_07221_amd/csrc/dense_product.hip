// Launches of the matrix products; compiled in one part for each type (HET_PART: HET_F32, HET_BF16, HET_F16), the first with the plan.
#include "../../include/het_dense.h"

#include <algorithm>

#include "dense_launch.hpp"

#define HET_PRODUCT_PARTS 3
static_assert(HET_PARTS == HET_PRODUCT_PARTS, "the build compiles other parts than there are: kernels would be missing in the library");

namespace het {

template <typename T> void launch_product_of(const ProductArgs &a, const ProductPlan &p, bool direct, bool a_k, bool b_k, hipStream_t st);

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
void launch_product_of(const ProductArgs &a, const ProductPlan &p, bool direct, bool a_k, bool b_k, hipStream_t st)
{
    if (p.few) {
        if (a.f.q) launch_few<T, 2>(a, p.few, st);
        else launch_few<T, 1>(a, p.few, st);
        return;
    }
    const uint32_t grid = (uint32_t)(a.tiles_m * a.tiles_n * a.splits);
    if (direct && p.tile == 256) {
        if (a_k && b_k) product_kernel<T, true, true, 256, 256, 2, 4><<<grid, 512, 0, st>>>(a);
        else if (a_k) product_kernel<T, true, false, 256, 256, 2, 4><<<grid, 512, 0, st>>>(a);
        else product_kernel<T, false, false, 256, 256, 2, 4><<<grid, 512, 0, st>>>(a);
    } else if (direct) {
        if (a_k && b_k) product_kernel<T, true, true, 128, 128, 2, 2><<<grid, 256, 0, st>>>(a);
        else if (a_k) product_kernel<T, true, false, 128, 128, 2, 2><<<grid, 256, 0, st>>>(a);
        else product_kernel<T, false, false, 128, 128, 2, 2><<<grid, 256, 0, st>>>(a);
    } else if (a_k && b_k) product_any_kernel<T, true, true><<<grid, 256, 0, st>>>(a);
    else if (a_k) product_any_kernel<T, true, false><<<grid, 256, 0, st>>>(a);
    else product_any_kernel<T, false, false><<<grid, 256, 0, st>>>(a);
    if (a.splits > 1) {
        const int64_t per = (a.n + PACK_BLOCK - 1) / PACK_BLOCK * 4;
        join_kernel<T><<<(uint32_t)((a.m * per + 255) / 256), 256, 0, st>>>(a);
    }
}

template void launch_product_of<PartType>(const ProductArgs &, const ProductPlan &, bool, bool, bool, hipStream_t);

#if HET_PART == 0
extern template void launch_product_of<bf16>(const ProductArgs &, const ProductPlan &, bool, bool, bool, hipStream_t);
extern template void launch_product_of<f16>(const ProductArgs &, const ProductPlan &, bool, bool, bool, hipStream_t);

constexpr int FEW_ROWS = 64;
constexpr int64_t CUS = 256;

// Microseconds a product takes with tiles of 256 or 128 and its k's split, by the times measured at 2048 .. 8192 rows and columns, 64 .. 8192
// k's, bf16 (fp32's steps take 4.8 times as long): a tile of 256 has a compute unit to itself, of 128 two share one.  Adding up the splits costs a
// launch and the sums' way through memory.
static double product_us(int tile, int64_t tiles, int64_t splits, int64_t steps, int64_t m, int64_t n, bool f32)
{
    const double s = (double)((steps + splits - 1) / splits) * (f32 ? 4.8 : 1.0);
    const int64_t groups = tiles * splits, turns = groups / CUS, more = groups % CUS != 0;
    double us = 0;
    if (tile == 256) us = (double)(turns + more) * (10 + 1.5 * s);
    else us = (double)((turns + more) / 2) * (6 + 0.86 * s) + (double)((turns + more) % 2) * (4 + 0.5 * s);
    return splits > 1 ? us + 4 + (double)splits * (double)m * (double)n * 2e-6 : us;
}

ProductPlan product_plan(int64_t m, int64_t n, int64_t k, int type, bool a_k, bool b_k)
{
    ProductPlan p{};
    p.m = (int)m; p.n = (int)n; p.k = (int)k;
    p.splits = 1; p.k_split = (int)k; p.tile = ANY_TILE;
    p.ok = true;
    if (a_k && b_k && m <= FEW_ROWS) {
        p.few = m <= 16 ? 1 : m <= 32 ? 2 : 4;
        return p;
    }
    const int64_t step = type == HET_F32 ? 32 : 64, steps = (k + step - 1) / step;
    double best = 1e30;
    for (int tile = 256; tile >= 128; tile /= 2) {
        const int64_t tiles = ((m + tile - 1) / tile) * ((n + tile - 1) / tile);
        for (int64_t splits = 1; splits <= 32 && (splits == 1 || (splits * 4 <= steps && tiles * splits <= 2 * CUS)); ++splits) {
            const double us = product_us(tile, tiles, splits, steps, m, n, type == HET_F32);
            if (us < best) { best = us; p.tile = tile; p.splits = (int)splits; }
        }
    }
    p.k_split = (int)((steps + p.splits - 1) / p.splits * step);
    p.splits = (int)std::max<int64_t>(1, (k + p.k_split - 1) / std::max(p.k_split, 1));
    p.ok = ((m + 127) / 128) * ((n + 127) / 128) * p.splits <= INT32_MAX && m * ((n + 31) / 32 * 4) / 256 < INT32_MAX;
    p.partial_bytes = p.splits > 1 ? p.splits * m * (int64_t)((n + 15) / 16 * 16) * 4 : 0;
    return p;
}

// Whether product_kernel takes an operand as it lies: rows at multiples of 16 bytes, whole pieces of them along k or across, and a tile within 2 GB.
static bool copies(const void *p, int64_t ld, int width, int rows_of_tile, int64_t size)
{
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * size % 16 == 0 && width * size % 16 == 0 && rows_of_tile * ld * size < (1ll << 31);
}

void launch_product(ProductArgs a, const ProductPlan &p, int type, bool a_k, bool b_k, hipStream_t st)
{
    a.m = p.m; a.n = p.n; a.k = p.k;
    a.splits = p.splits; a.k_split = p.k_split;
    const int64_t size = type == HET_F32 ? 4 : 2;
    const bool direct = copies(a.a, a.lda, a_k ? a.k : a.m, 256, size) && copies(a.b, a.ldb, b_k ? a.k : a.n, 256, size);
    const int tile = direct ? p.tile : ANY_TILE;
    a.tiles_m = (a.m + tile - 1) / tile; a.tiles_n = (a.n + tile - 1) / tile;
    if (type == HET_F32) launch_product_of<float>(a, p, direct, a_k, b_k, st);
    else if (type == HET_BF16) launch_product_of<bf16>(a, p, direct, a_k, b_k, st);
    else launch_product_of<f16>(a, p, direct, a_k, b_k, st);
}
#endif

} // namespace het
