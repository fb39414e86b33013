// Launches of the matrix products; compiled in one part for each type (HET_PART: HET_F32, HET_BF16, HET_F16), the first with the plan.
#include "../../include/het_dense.h"

#include "dense_launch.hpp"

#define HET_PRODUCT_PARTS 3
static_assert(HET_PARTS == HET_PRODUCT_PARTS, "the build compiles other parts than there are: kernels would be missing in the library");

namespace het {

constexpr int64_t CUS = 256, MOST_SPLITS = 128, DEEP_STEPS = 4;

template <typename T> void launch_product_of(const ProductArgs &a, const ProductPlan &p, bool a_k, bool b_k, hipStream_t st);
template <typename T> void launch_small_back_of(const SmallBackArgs &a, int nw, int nx, uint32_t grid, hipStream_t st);

#if HET_PART == 0
using PartType = float;
#elif HET_PART == 1
using PartType = bf16;
#else
using PartType = f16;
#endif

template <typename T, int MT, int NT>
static void launch_small(const ProductArgs &a, bool a_k, bool b_k, hipStream_t st)
{
    const uint32_t grid = (uint32_t)(a.tiles_m * a.tiles_n);
    if (a_k && b_k) product_small_kernel<T, true, true, MT, NT><<<grid, 64 * SMALL_WAVES, 0, st>>>(a);
    else if constexpr (MT == 2) {
        if (a_k) product_small_kernel<T, true, false, MT, NT><<<grid, 64 * SMALL_WAVES, 0, st>>>(a);
        else product_small_kernel<T, false, false, MT, NT><<<grid, 64 * SMALL_WAVES, 0, st>>>(a);
    }
}

template <typename T>
void launch_product_of(const ProductArgs &a, const ProductPlan &p, bool a_k, bool b_k, hipStream_t st)
{
    if (p.small_m) {
        const bool wide = p.small_n == 2 || a.f.q;          // (a block of the 8-bit form needs its 32 columns together)
        if (p.small_m == 1) { if (wide) launch_small<T, 1, 2>(a, a_k, b_k, st); else launch_small<T, 1, 1>(a, a_k, b_k, st); }
        else { if (wide) launch_small<T, 2, 2>(a, a_k, b_k, st); else launch_small<T, 2, 1>(a, a_k, b_k, st); }
        return;
    }
    const uint32_t grid = (uint32_t)(a.tiles_m * a.tiles_n * a.splits);
    const auto joined = [&] {
        if (a.splits == 1) return;
        const int64_t per = (a.n + PACK_BLOCK - 1) / PACK_BLOCK * 4;
        if (a.splits > 8) join_kernel<T, 8><<<(uint32_t)((a.m * per + 31) / 32), 256, 0, st>>>(a);
        else join_kernel<T, 1><<<(uint32_t)((a.m * per + 255) / 256), 256, 0, st>>>(a);
    };
    if (p.tile == 256) {
        if (a_k && b_k) product_kernel<T, true, true, 256, 256, 2, 4, 2><<<grid, 512, 0, st>>>(a);
        else if (a_k) product_kernel<T, true, false, 256, 256, 2, 4, 2><<<grid, 512, 0, st>>>(a);
        else product_kernel<T, false, false, 256, 256, 2, 4, 2><<<grid, 512, 0, st>>>(a);
        return joined();
    }
    // A tile alone on its compute unit waits for its copies unless they are further ahead, a pair for each other's; in fp32 the products take longer than
    // the copies (2048 x 2048 -> 2048 in bf16 28.0 us with two buffers, 20.8 with four; 1024 x 4096 -> 4096 46.3 and 35.3; fp32 62.5 and 66.3).  It goes in turns of four
    // steps: fewer are not worth it.
    if constexpr (sizeof(T) == 2)
        if (grid <= CUS && a.k_split >= DEEP_STEPS * 64) {
            if (a_k && b_k) product_kernel<T, true, true, 128, 128, 2, 2, 4><<<grid, 256, 0, st>>>(a);
            else if (a_k) product_kernel<T, true, false, 128, 128, 2, 2, 4><<<grid, 256, 0, st>>>(a);
            else product_kernel<T, false, false, 128, 128, 2, 2, 4><<<grid, 256, 0, st>>>(a);
            return joined();
        }
    if (a_k && b_k) product_kernel<T, true, true, 128, 128, 2, 2, 2><<<grid, 256, 0, st>>>(a);
    else if (a_k) product_kernel<T, true, false, 128, 128, 2, 2, 2><<<grid, 256, 0, st>>>(a);
    else product_kernel<T, false, false, 128, 128, 2, 2, 2><<<grid, 256, 0, st>>>(a);
    joined();
}

template <typename T>
void launch_small_back_of(const SmallBackArgs &a, int nw, int nx, uint32_t grid, hipStream_t st)
{
    if (nw == 1) {
        if (nx == 1) small_back_kernel<T, 1, 1><<<grid, 64 * SMALL_WAVES, 0, st>>>(a);
        else small_back_kernel<T, 1, 2><<<grid, 64 * SMALL_WAVES, 0, st>>>(a);
    } else {
        if (nx == 1) small_back_kernel<T, 2, 1><<<grid, 64 * SMALL_WAVES, 0, st>>>(a);
        else small_back_kernel<T, 2, 2><<<grid, 64 * SMALL_WAVES, 0, st>>>(a);
    }
}

template void launch_small_back_of<PartType>(const SmallBackArgs &, int, int, uint32_t, hipStream_t);
template void launch_product_of<PartType>(const ProductArgs &, const ProductPlan &, bool, bool, hipStream_t);

#if HET_PART == 0
extern template void launch_small_back_of<bf16>(const SmallBackArgs &, int, int, uint32_t, hipStream_t);
extern template void launch_small_back_of<f16>(const SmallBackArgs &, int, int, uint32_t, hipStream_t);
extern template void launch_product_of<bf16>(const ProductArgs &, const ProductPlan &, bool, bool, hipStream_t);
extern template void launch_product_of<f16>(const ProductArgs &, const ProductPlan &, bool, bool, hipStream_t);

// Microseconds a product takes with tiles of 256 or 128 and its k's split, by the times measured at 16 .. 16384 rows, columns and k's in bf16 and
// fp32: a tile of 256 has a compute unit to itself, of 128 two share one if there are so many.  Adding up the splits costs a launch and the sums' way through memory.
// 4096 x 1664 -> 4096 in bf16: 256 48, 128 54 us; 2048 x 2048 -> 2048: 43 and 20; dw of 16384 x 896 -> 4096: 128 175, split in two 126, 256 split in
// four 129; dw of 100000 x 64 -> 64: split in 32 34 + 10, in 128 13 + 6.  Tiles of 256 x 128 (two waves' 64 x 64 side by side, one workgroup a compute
// unit) were slower than one of the two everywhere.
static double tiles_us(int tile, int64_t tiles, int64_t splits, int64_t steps, int64_t m, int64_t n, bool f32, bool b_k)
{
    const double s = (double)((steps + splits - 1) / splits), start = b_k ? 4 : 7;
    const int64_t groups = tiles * splits, turns = (groups + CUS - 1) / CUS;
    double us = 0;
    if (tile == 128 && !f32 && groups <= CUS && s >= DEEP_STEPS) us = start + (0.35 + 0.1 * (double)groups / CUS) * s;
    else if (tile == 256) us = (double)turns * (10 + (f32 ? 7.3 : 1.5) * s);
    else us = (double)(turns / 2) * (start + 2 + (f32 ? 4.1 : 0.8) * s) + (double)(turns % 2) * (start + (f32 ? 2.1 : 0.62) * s);
    return splits > 1 ? us + 3 + (double)splits * (double)m * (double)n * 1.4e-6 : us;
}

// ... and with product_small_kernel: its waves' turns through k (a step is a span, two of them at a time), a thousand workgroups at a time, and the
// operands out of the L2 once for every 32 rows or columns.  1001 x 500 -> 250 in fp16: 7.6 .. 8.4 us a product, tiles 16.6 .. 20.4; 2048 x 1024 ->
// 1024 in bf16: 30.6, tiles 11.4; a single token 1664 -> 1024: 7.9, tiles 12.7; dx of 16384 x 16 -> 64: 3.8, tiles 7.3 (each with the launch).
static double small_us(int64_t steps, int64_t m, int64_t n, int64_t k, bool a_k, bool b_k, bool f32)
{
    const int64_t high = a_k && b_k && m <= 16 ? 16 : (m + 31) / 32 * 32, wide = (n + 31) / 32 * 32;
    const double turn = !a_k ? 2.5 : f32 ? 2 : 1.5, each = f32 ? 28e-9 : b_k ? 16e-9 : 20e-9;
    return 0.5 + turn * (double)((steps + 2 * SMALL_WAVES - 1) / (2 * SMALL_WAVES)) + 4.0 / 1024 * (double)high * (double)wide / 1024 +
           each * (double)high * (double)wide * (double)k;
}

// ... and laying out an operand: a launch, and its way there and back through memory; only there if slope_kernel does it.
double lay_us(bool lies, int64_t rows, int64_t width, int type) { return lies ? 0 : 3 + 2 * written_us(lies, rows, width, type); }
double written_us(bool lies, int64_t rows, int64_t width, int type) { return lies ? 0 : 0.1 + (double)rows * (double)width * (type == HET_F32 ? 4 : 2) / 4e6; }

ProductPlan product_plan(int64_t m, int64_t n, int64_t k, int type, bool a_k, bool b_k, double lay_a, double lay_b)
{
    const bool f32 = type == HET_F32;
    ProductPlan p{};
    p.lay_a = lay_a > 0; p.lay_b = lay_b > 0;
    p.m = (int)m; p.n = (int)n; p.k = (int)k;
    double best = 1e30;
    const int64_t step = f32 ? 32 : 64, steps = (k + step - 1) / step;
    for (int tile = 256; tile >= 128; tile /= 2) {
        const int64_t tiles = std::max<int64_t>(1, ((m + tile - 1) / tile) * ((n + tile - 1) / tile));
        const int64_t most = std::max<int64_t>(1, std::min({MOST_SPLITS, steps / 4, 4 * CUS / tiles}));
        const auto of = [&](int64_t splits) {
            const double us = tiles_us(tile, tiles, splits, steps, m, n, f32, b_k);
            if (us < best) { best = us; p.tile = tile; p.splits = (int)splits; }
        };
        // every number of splits up to 8, then fewer and fewer, and those that fill the compute units' turns
        for (int64_t splits = 1; splits <= most; splits += splits < 8 ? 1 : splits / 4) of(splits);
        for (int64_t turns = 1; turns <= 4 && most > 8; turns *= 2) of(std::max<int64_t>(1, std::min(most, turns * CUS / tiles)));
    }
    best += lay_a + lay_b;
    if (small_us(steps, m, n, k, a_k, b_k, f32) < best) {
        p.small_m = a_k && b_k && m <= 16 ? 1 : 2;
        p.small_n = ((m + 31) / 32) * ((n + 31) / 32) < CUS ? 1 : 2;
        p.splits = 1;
        p.lay_a = p.lay_b = false;
    }
    p.k_split = (int)((steps + p.splits - 1) / p.splits * step);
    p.splits = (int)std::max<int64_t>(1, (k + p.k_split - 1) / std::max(p.k_split, 1));
    // (rows of x or dz go in several launches if they have to)
    const int64_t high = p.small_m ? 16 * p.small_m : p.tile, wide = p.small_m ? 16 * p.small_n : p.tile;
    p.ok = a_k || (m + high - 1) / high * ((n + wide - 1) / wide) * p.splits * (p.small_m ? 64 * SMALL_WAVES : 2 * p.tile) < (1ll << 32);
    p.partial_bytes = p.splits > 1 ? p.splits * m * (int64_t)((n + 15) / 16 * 16) * 4 : 0;
    return p;
}

// Whether product_kernel takes an operand as it lies: rows at multiples of 16 bytes and of whole pieces, a tile within 2 GB.
bool product_lies(const void *p, int64_t ld, int64_t width, int type)
{
    const int64_t size = type == HET_F32 ? 4 : 2;
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * size % 16 == 0 && width * size % 16 == 0 && 256 * ld * size < (1ll << 31);
}

int64_t laid_pitch(int64_t width, int type) { return type == HET_F32 ? (width + 3) / 4 * 4 : (width + 7) / 8 * 8; }

void launch_lay(const void *p, int64_t ld, int64_t rows, int width, void *to, int type, hipStream_t st)
{
    const int64_t pitch = laid_pitch(width, type), pieces = pitch / (type == HET_F32 ? 4 : 8);
    in_launches(rows, pieces, [&](int64_t first, int64_t some) {
        const uint32_t grid = (uint32_t)((some * pieces + 255) / 256);
        if (type == HET_F32) lay_kernel<uint32_t><<<grid, 256, 0, st>>>(static_cast<const uint32_t *>(p) + first * ld, ld, some, width, static_cast<uint32_t *>(to) + first * pitch, (int)pitch);
        else lay_kernel<uint16_t><<<grid, 256, 0, st>>>(static_cast<const uint16_t *>(p) + first * ld, ld, some, width, static_cast<uint16_t *>(to) + first * pitch, (int)pitch);
    });
}

void launch_product(ProductArgs all, const ProductPlan &p, int type, bool a_k, bool b_k, hipStream_t st)
{
    all.n = p.n; all.k = p.k;
    all.splits = p.splits; all.k_split = p.k_split;
    const int tile = p.tile, high = p.small_m ? 16 * p.small_m : tile, wide = p.small_m ? 16 * (all.f.q ? 2 : p.small_n) : tile;
    all.tiles_n = (all.n + wide - 1) / wide;
    const int64_t size = type == HET_F32 ? 4 : 2, y_size = all.f.y_f32 ? 4 : 2, threads = (int64_t)all.tiles_n * all.splits * (p.small_m ? 64 * SMALL_WAVES : 2 * tile) / high;
    const auto part = [&](int64_t first, int64_t rows) {
        ProductArgs a = all;
        a.m = (int)rows;
        a.tiles_m = (a.m + high - 1) / high;
        if (first) {
            a.a = moved(a.a, first * a.lda, size);
            a.f.y = moved(a.f.y, first * a.f.ldy, y_size); a.f.residual = moved(a.f.residual, first * a.f.ldr, y_size); a.f.z = moved(a.f.z, first * a.f.ldz, size);
            a.f.q = moved(a.f.q, first * a.f.pitch, 1); a.f.e = moved(a.f.e, first * (a.f.pitch / PACK_BLOCK), 1);
        }
        if (type == HET_F32) launch_product_of<float>(a, p, a_k, b_k, st);
        else if (type == HET_BF16) launch_product_of<bf16>(a, p, a_k, b_k, st);
        else launch_product_of<f16>(a, p, a_k, b_k, st);
    };
    if (a_k) in_launches(p.m, threads, part);         // (A's rows are the product's)
    else part(0, p.m);
}

// Sizes of a product of product_small_kernel's; its workgroups.
static int64_t small_sizes(ProductArgs &a, const ProductPlan &p)
{
    a.m = p.m; a.n = p.n; a.k = p.k;
    a.splits = p.splits; a.k_split = p.k_split;
    a.tiles_m = (a.m + 16 * p.small_m - 1) / (16 * p.small_m); a.tiles_n = (a.n + 16 * p.small_n - 1) / (16 * p.small_n);
    return (int64_t)a.tiles_m * a.tiles_n;
}

bool launch_small_back(ProductArgs dw, const ProductPlan &dw_plan, ProductArgs dx, const ProductPlan &dx_plan, const ColumnSumArgs &bias, int type, hipStream_t st)
{
    if (dw_plan.small_m != 2 || dx_plan.small_m != 2) return false;
    SmallBackArgs a{dw, dx, bias, 0, 0, dx_plan.k > dw_plan.k};
    const int64_t w = small_sizes(a.dw, dw_plan), x = small_sizes(a.dx, dx_plan), b = bias.n ? (bias.sets * bias.width + 15) / 16 : 0;
    if ((w + x + b) * 64 * SMALL_WAVES >= 1ll << 31) return false;
    a.dw_groups = (int)w; a.dx_groups = (int)x;
    const uint32_t grid = (uint32_t)(w + x + b);
    if (type == HET_F32) launch_small_back_of<float>(a, dw_plan.small_n, dx_plan.small_n, grid, st);
    else if (type == HET_BF16) launch_small_back_of<bf16>(a, dw_plan.small_n, dx_plan.small_n, grid, st);
    else launch_small_back_of<f16>(a, dw_plan.small_n, dx_plan.small_n, grid, st);
    return true;
}
#endif

} // namespace het
