// Launches of layer norm; compiled in one part for each pair of types.
#include "dense_launch.hpp"

#define HET_NORM_PARTS 5
static_assert(HET_PARTS == HET_NORM_PARTS, "the build compiles other parts than there are: kernels would be missing in the library");

namespace het {

#if HET_PART == 0
using X = float; using Y = float;
#elif HET_PART == 1
using X = float; using Y = bf16;
#elif HET_PART == 2
using X = float; using Y = f16;
#elif HET_PART == 3
using X = bf16; using Y = bf16;
#else
using X = f16; using Y = f16;
#endif

#if HET_PART == 0
// A row's lanes: few where it is narrow, so that a wave holds several rows; a workgroup from ROW_WIDE on, with a chunk a thread as far as 512
// threads reach (more chunks a lane leave too few registers for the loads of the next row: 4096 x 1664 backward, 4 chunks in each of 64
// lanes of a wave 43.8 us, one in each of 256 threads 18.1).
NormShape norm_shape(int dim)
{
    NormShape h;
    const int chunks = (dim + CHUNK - 1) / CHUNK;
    h.s.dim = dim;
    h.s.pitch = (dim + PACK_BLOCK - 1) / PACK_BLOCK * PACK_BLOCK;
    h.block = dim > ROW_WIDE;
    if (h.block) {
        h.s.lanes = chunks <= 128 ? 128 : chunks <= 256 ? 256 : chunks <= 512 * 4 ? 512 : 1024;
        h.rows = 1;
    } else {
        h.s.lanes = 4;
        while (h.s.lanes < chunks) h.s.lanes *= 2;
        h.rows = ROW_THREADS / h.s.lanes;
    }
    const int n = (chunks + h.s.lanes - 1) / h.s.lanes;
    h.nv = n <= 1 ? 1 : n <= 2 ? 2 : 4;
    // two workgroups of 256 or 512 threads a compute unit, four of 128, and one where a lane has several chunks (their registers leave no more room): backward
    // of 20000 x 1000 53 us with 512 workgroups of 256 threads, 39 with 1024 of 128; 16384 x 4096 107 with 512, 134 with 256; 8192 x 8192 119 and 109
    h.groups = h.block && h.s.lanes == 128 ? 2 * (int)PARTIALS : h.nv > 1 ? (int)PARTIALS / 2 : (int)PARTIALS;
    return h;
}
#endif

template <bool WHOLE>
static void norm_part_of(const NormArgs &a, const NormShape &h, hipStream_t st)
{
    const uint32_t grid = (uint32_t)((a.rows + h.rows - 1) / h.rows);
    if (!h.block) norm_kernel<X, Y, 1, ROW_THREADS, WHOLE><<<grid, ROW_THREADS, 0, st>>>(a);
    else if (h.nv == 1) norm_kernel<X, Y, 1, 512, WHOLE><<<grid, h.s.lanes, 0, st>>>(a);
    else if (h.nv == 2) norm_kernel<X, Y, 2, 512, WHOLE><<<grid, h.s.lanes, 0, st>>>(a);
    else if (h.s.lanes == 512) norm_kernel<X, Y, 4, 512, WHOLE><<<grid, h.s.lanes, 0, st>>>(a);
    else norm_kernel<X, Y, 4, 1024, WHOLE><<<grid, h.s.lanes, 0, st>>>(a);
}

template <bool WHOLE>
static void norm_of(const NormArgs &all, const NormShape &h, hipStream_t st)
{
    in_launches(all.rows, h.s.lanes, [&](int64_t first, int64_t rows) {
        NormArgs a = all;
        a.x = moved(a.x, first * a.ldx, sizeof(X)); a.y = moved(a.y, first * a.ldy, sizeof(Y));
        a.mean = moved(a.mean, first, 4); a.rstd = moved(a.rstd, first, 4);
        a.q = moved(a.q, first * h.s.pitch, 1); a.e = moved(a.e, first * (h.s.pitch / PACK_BLOCK), 1);
        a.rows = rows;
        norm_part_of<WHOLE>(a, h, st);
    });
}

template <bool KEPT, bool WHOLE>
static void norm_back_of(const NormBackArgs &a, const NormShape &h, int groups, hipStream_t st)
{
    const size_t lds = 2 * sizeof(float) * ((h.s.dim + CHUNK - 1) / CHUNK * CHUNK);
    if (!h.block) norm_back_kernel<X, Y, 1, ROW_THREADS, KEPT, WHOLE><<<groups, ROW_THREADS, lds, st>>>(a);
    else if (h.nv == 1) norm_back_kernel<X, Y, 1, 512, KEPT, WHOLE><<<groups, h.s.lanes, 0, st>>>(a);
    else if (h.nv == 2) norm_back_kernel<X, Y, 2, 512, KEPT, WHOLE><<<groups, h.s.lanes, 0, st>>>(a);
    else if (h.s.lanes == 512) norm_back_kernel<X, Y, 4, 512, KEPT, WHOLE><<<groups, h.s.lanes, 0, st>>>(a);
    else norm_back_kernel<X, Y, 4, 1024, KEPT, WHOLE><<<groups, h.s.lanes, 0, st>>>(a);
}

template <> void launch_norm<X, Y>(const NormArgs &a, const NormShape &h, hipStream_t st)
{
    if (h.s.dim % CHUNK == 0) norm_of<true>(a, h, st);
    else norm_of<false>(a, h, st);
}

template <> void launch_norm_back<X, Y>(const NormBackArgs &a, const NormShape &h, int groups, hipStream_t st)
{
    const bool whole = h.s.dim % CHUNK == 0;
    if (a.q) { if (whole) norm_back_of<true, true>(a, h, groups, st); else norm_back_of<true, false>(a, h, groups, st); }
    else { if (whole) norm_back_of<false, true>(a, h, groups, st); else norm_back_of<false, false>(a, h, groups, st); }
}

} // namespace het
