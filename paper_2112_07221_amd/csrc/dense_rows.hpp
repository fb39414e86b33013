// Row-wise kernels of the dense layers: layer norm, its backward pass, the slope of an activation with the bias' gradient, and the
// 8-bit form of activations.  All are bound by HBM (or, where rows are few, by a launch): every value is read once, kept in
// registers while its row's sums are formed, and written once.
#pragma once
#include "dense_types.hpp"

namespace het {

constexpr int ROW_THREADS = 256;
constexpr int ROW_WAVES = ROW_THREADS / 64;
constexpr int ROW_WIDE = 64 * CHUNK;               // widest row that a wave holds, a chunk a lane
constexpr int ROW_WIDEST = 1024 * CHUNK * 4;       // and a workgroup
constexpr uint32_t PARTIALS = 512;                 // workgroups that leave partial column sums, about

// How a row lies over lanes.  Rows of up to ROW_WIDE values belong to `lanes` (a power of two, at least a block's four) consecutive lanes of
// a wave, wider ones to a whole workgroup; lane l holds the chunks l, l + lanes, ...
struct RowShape {
    int dim;           // values of a row
    int pitch;         // ... in the 8-bit form: rounded up to whole blocks
    int lanes;         // lanes of a row, or threads of a workgroup that holds one
};

// Sum over the `lanes` lanes of a row; every lane gets it, all the same bits (each step adds two equal sums' worth in either order).
__device__ __forceinline__ float lanes_sum(float v, int lanes)
{
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0xB1, 0xf, 0xf, false));       // lanes 1 0 3 2
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x4E, 0xf, 0xf, false));       // lanes 2 3 0 1
    if (lanes >= 8) v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x141, 0xf, 0xf, false));    // mirrored in 8
    if (lanes >= 16) v += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x140, 0xf, 0xf, false));   // mirrored in 16
    if (lanes >= 32) v += __shfl_xor(v, 16);
    if (lanes >= 64) v += __shfl_xor(v, 32);
    return v;
}

// The sums of a row: over its lanes, or over the workgroup (`lds`: 32 floats; calls alternate between two areas, so one barrier does).
template <bool BLOCK>
struct RowSum {
    float *lds;
    int lanes;
    int turn = 0;
    __device__ __forceinline__ RowSum(float *lds_, int lanes_) : lds(lds_), lanes(lanes_) {}
    // Two sums at once: one trip.
    __device__ __forceinline__ void two(float &a, float &b)
    {
        a = lanes_sum(a, BLOCK ? 64 : lanes);
        b = lanes_sum(b, BLOCK ? 64 : lanes);
        if (!BLOCK) return;
        float *at = lds + 32 * turn;
        turn ^= 1;
        const int w = threadIdx.x / 64, waves = lanes / 64;
        if (threadIdx.x % 64 == 0) { at[w] = a; at[16 + w] = b; }
        __syncthreads();
        a = at[0]; b = at[16];
        for (int i = 1; i < waves; ++i) { a += at[i]; b += at[16 + i]; }
    }
    __device__ __forceinline__ float one(float a) { float b = 0.f; two(a, b); return a; }
};

__device__ __forceinline__ int chunk_values(int c, int dim)      // values of chunk c that are in the row
{
    const int n = dim - c * CHUNK;
    return n < 0 ? 0 : n;
}

// ---- layer norm ---------------------------------------------------------------------------------------
// y = gamma (x - mean) rstd + beta, rstd = 1 / sqrt(var + eps).  The variance is summed from the differences to the mean (the row is in
// registers), not as a difference of two large sums.  All sums in 32 bits.
struct NormArgs {
    const void *x;
    const float *gamma, *beta;
    void *y;
    float *mean, *rstd;
    int8_t *q;              // normalised rows in 8 bits, or null
    uint8_t *e;
    int64_t ldx, ldy, rows;
    RowShape s;
    float eps;
};

template <typename TX, typename TY, int NV, int MOST, bool WHOLE>
__global__ __launch_bounds__(MOST) void norm_kernel(NormArgs a)
{
    constexpr bool BLOCK = MOST > ROW_THREADS;
    __shared__ float lds[64];
    const int lanes = a.s.lanes, gl = threadIdx.x % lanes, dim = a.s.dim;
    const int64_t row = BLOCK ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * (ROW_THREADS / lanes) + threadIdx.x / lanes;
    if (row >= a.rows) return;                     // (whole rows of lanes; a workgroup that holds one row has one)
    const TX *x = static_cast<const TX *>(a.x) + row * a.ldx;
    RowSum<BLOCK> sum(lds, lanes);
    vec<TX, 8> raw[NV];
    f32x8 v[NV];
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = load_raw<WHOLE>(x, gl + i * lanes, dim);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        v[i] = raw_values<WHOLE>(raw[i], gl + i * lanes, dim);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[i][j];
    }
    const float mean = sum.one(s) / (float)dim;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] -= mean;
        v[i] = chunk_only<WHOLE>(v[i], gl + i * lanes, dim);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[i][j] * v[i][j];
    }
    const float rstd = 1.f / sqrtf(sum.one(s) / (float)dim + a.eps);
    if (gl == 0) {
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    TY *y = static_cast<TY *>(a.y) + row * a.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = gl + i * lanes, n = chunk_values(c, dim);
        f32x8 h;
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = v[i][j] * rstd;
        if (a.q && c * CHUNK < a.s.pitch) pack_chunk(a.q + row * a.s.pitch, a.e + row * (a.s.pitch / PACK_BLOCK), c, h, WHOLE ? 0 : chunk_skip(c, dim));
        if (n <= 0) continue;
        const f32x8 g = a.gamma ? load_row<WHOLE>(a.gamma, c, dim) : f32x8{1, 1, 1, 1, 1, 1, 1, 1};
        const f32x8 b = a.beta ? load_row<WHOLE>(a.beta, c, dim) : f32x8{};
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = h[j] * g[j] + b[j];
        // Past the L2: 106496 x 64 to bf16 alone 6.3 us (through it 7.8), 4096 x 1664 8.2 (9.4).  With the product that reads them: 2048 x 1664 -> 4096 37.2 (39.1),
        // 4096 x 1664 -> 4096 61.4 (60.9), 16384 x 896 -> 4096 141.3 (138.9), 106496 x 64 -> 64 25.6 (22.7); below 1024 x 1664 values no difference.
        store_row<WHOLE, true>(y, c, dim, h);
    }
}

// Backward: with n the normalised row and g = dy gamma, dx = rstd (g - mean(g) - n mean(g n)) + residual; dgamma = sum over rows of
// dy n, dbeta of dy.  A workgroup goes through rows in steps of the grid and keeps its columns' sums in registers; what it has summed goes
// to `partial` ([workgroup][dgamma, dbeta][width rounded up to a chunk]), and column_sum_kernel adds that up in the order of the
// workgroups: the same bits every time.
struct NormBackArgs {
    const void *dy, *x;
    const float *mean, *rstd;
    const int8_t *q;        // normalised rows in 8 bits; null: from x, mean and rstd
    const uint8_t *e;
    const float *gamma;
    const void *residual;   // added to dx, or null
    void *dx;
    float *partial;
    int64_t lddy, ldx, ldr, lddx, rows;
    RowShape s;
};

// What a lane loads of a row: dy, and x or its normalised values in 8 bits.
template <typename TX, typename TY, int NV, bool KEPT, bool WHOLE>
struct NormRow {
    vec<TY, 8> dy[NV];
    vec<TX, 8> x[KEPT ? 1 : NV];
    uint64_t q[KEPT ? NV : 1];
    uint8_t e[KEPT ? NV : 1];
    float rstd, mean;

    __device__ __forceinline__ void load(const NormBackArgs &a, int64_t row, int gl)
    {
        const int lanes = a.s.lanes, dim = a.s.dim;
        rstd = a.rstd[row];
        mean = KEPT ? 0.f : a.mean[row];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = gl + i * lanes;
            dy[i] = load_raw<WHOLE>(static_cast<const TY *>(a.dy) + row * a.lddy, c, dim);
            if (KEPT) {
                __builtin_memcpy(&q[i], a.q + row * a.s.pitch + chunk_from(c, dim), 8);
                e[i] = a.e[row * (a.s.pitch / PACK_BLOCK) + (c * CHUNK < dim ? c >> 2 : 0)];
            } else {
                x[i] = load_raw<WHOLE>(static_cast<const TX *>(a.x) + row * a.ldx, c, dim);
            }
        }
    }
};

template <typename TX, typename TY, int NV, int MOST, bool KEPT, bool WHOLE>
__global__ __launch_bounds__(MOST) void norm_back_kernel(NormBackArgs a)
{
    constexpr bool BLOCK = MOST > ROW_THREADS;
    extern __shared__ __attribute__((aligned(16))) float cols[];      // [chunk][dgamma, dbeta][8], where several rows' lanes share columns
    __shared__ float lds[64];
    const int lanes = a.s.lanes, gl = threadIdx.x % lanes, dim = a.s.dim;
    const int64_t per = BLOCK ? 1 : ROW_THREADS / lanes, step = per * gridDim.x;
    RowSum<BLOCK> sum(lds, lanes);
    f32x8 dg[NV], db[NV], gamma[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        dg[i] = db[i] = f32x8{};
        gamma[i] = a.gamma ? load_row<WHOLE>(a.gamma, gl + i * lanes, dim) : f32x8{1, 1, 1, 1, 1, 1, 1, 1};
    }
    int64_t row = (int64_t)blockIdx.x * per + (BLOCK ? 0 : threadIdx.x / lanes);
    NormRow<TX, TY, NV, KEPT, WHOLE> now, next;
    if (row < a.rows) now.load(a, row, gl);
    for (; row < a.rows; row += step, now = next) {
        vec<TX, 8> r[NV];
        if (a.residual)
#pragma unroll
            for (int i = 0; i < NV; ++i) r[i] = load_raw<WHOLE>(static_cast<const TX *>(a.residual) + row * a.ldr, gl + i * lanes, dim);
        if (row + step < a.rows) next.load(a, row + step, gl);        // on its way while this row is summed and written
        f32x8 d[NV], h[NV];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = gl + i * lanes;
            d[i] = raw_values<WHOLE>(now.dy[i], c, dim);
            if (KEPT) {
                h[i] = unpack_chunk(now.q[i], now.e[i]);
            } else {
                h[i] = __builtin_convertvector(now.x[i], f32x8);
#pragma unroll
                for (int j = 0; j < 8; ++j) h[i][j] = (h[i][j] - now.mean) * now.rstd;
            }
            h[i] = chunk_only<WHOLE>(h[i], c, dim);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                dg[i][j] += d[i][j] * h[i][j];
                db[i][j] += d[i][j];
                d[i][j] *= gamma[i][j];
                s1 += d[i][j];
                s2 += d[i][j] * h[i][j];
            }
        }
        sum.two(s1, s2);
        s1 /= (float)dim; s2 /= (float)dim;
        TX *dx = static_cast<TX *>(a.dx) + row * a.lddx;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = gl + i * lanes;
            f32x8 o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = now.rstd * (d[i][j] - s1 - h[i][j] * s2);
            if (a.residual) {
                const f32x8 f = raw_values<WHOLE>(r[i], c, dim);
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] += f[j];
            }
            store_row<WHOLE>(dx, c, dim, o);
        }
    }
    const int width = (dim + CHUNK - 1) / CHUNK * CHUNK;
    float *out = a.partial + (size_t)blockIdx.x * 2 * width;
    if (BLOCK) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = gl + i * lanes;
            if (c * CHUNK >= width) continue;
            store_chunk(out + c * CHUNK, chunk_own<WHOLE>(dg[i], c, dim));
            store_chunk(out + width + c * CHUNK, chunk_own<WHOLE>(db[i], c, dim));
        }
        return;
    }
    // lanes of a wave that hold the same columns of other rows, then the waves one after the other (a chunk a lane here)
    for (int o = lanes; o < 64; o <<= 1)
#pragma unroll
        for (int j = 0; j < 8; ++j) { dg[0][j] += __shfl_xor(dg[0][j], o); db[0][j] += __shfl_xor(db[0][j], o); }
    const bool mine = (int)threadIdx.x % 64 < lanes && gl * CHUNK < width;
    f32x4 *at = reinterpret_cast<f32x4 *>(cols) + 4 * gl;
    // (before the waves take turns: 333 x 260 7.6 -> 5.7 us)
    const f32x8 own[2] = {chunk_own<WHOLE>(dg[0], gl, dim), chunk_own<WHOLE>(db[0], gl, dim)};
    for (int w = 0; w < ROW_WAVES; ++w) {
        if ((int)threadIdx.x / 64 == w && mine) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const f32x8 s = own[u / 2];
                f32x4 v = {s[4 * (u % 2)], s[4 * (u % 2) + 1], s[4 * (u % 2) + 2], s[4 * (u % 2) + 3]};
                if (w) for (int j = 0; j < 4; ++j) v[j] += at[u][j];
                at[u] = v;
            }
        }
        __syncthreads();
    }
    for (int c = threadIdx.x; c < 2 * width; c += ROW_THREADS) {
        const int col = c < width ? c : c - width;
        out[c] = cols[col / CHUNK * 2 * CHUNK + (c < width ? 0 : CHUNK) + col % CHUNK];
    }
}

// Column sums of partial[n][sets][width]: set s goes to out[s] (null: nobody asks).  16 columns a workgroup, for each of them 64 sums of
// every 64th row, eight rows in flight, which are added in order: the same bits whatever the number of threads.
struct ColumnSumArgs {
    const float *partial;
    float *out[2];
    int n, sets, width, dim;
};

constexpr int COLUMN_THREADS = 1024;

constexpr int COLUMN_DEEP = 64;

template <int THREADS>
__device__ __forceinline__ void column_sum(const ColumnSumArgs &a, int block, float (*lds)[17])       // lds: [COLUMN_DEEP]
{
    constexpr int DEEP = COLUMN_DEEP;
    const int cx = threadIdx.x % 16, ry = threadIdx.x / 16, col = block * 16 + cx, total = a.sets * a.width;
    const float *p = a.partial + (col < total ? col : 0);
    float s = 0.f;
#pragma unroll
    for (int first = DEEP - THREADS / 16; first >= 0; first -= THREADS / 16) {             // (the thread's own row of sums last: it goes on with it)
        s = 0.f;
        for (int r = ry + first; r < a.n; r += 8 * DEEP) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = p[(size_t)(r + u * DEEP < a.n ? r + u * DEEP : r) * total];
#pragma unroll
            for (int u = 0; u < 8; ++u) s += r + u * DEEP < a.n ? v[u] : 0.f;
        }
        lds[ry + first][cx] = s;
    }
    __syncthreads();
    if (ry >= 4) return;                                  // four threads a column, then one
#pragma unroll
    for (int u = 1; u < DEEP / 4; ++u) s += lds[ry + 4 * u][cx];
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    if (ry || col >= total) return;
    const int set = col / a.width, at = col % a.width;
    if (at < a.dim && a.out[set]) a.out[set][at] = s;
}

static __global__ __launch_bounds__(COLUMN_THREADS) void column_sum_kernel(ColumnSumArgs a)
{
    __shared__ float lds[COLUMN_DEEP][17];
    column_sum<COLUMN_THREADS>(a, blockIdx.x, lds);
}

// ---- the slope of the activation and the bias' gradient -------------------------------------------------
// dz = dy act'(z), handed on in the layer's type (the matrix instructions take it so); dbias = column sums of dz before that rounding.
// A thread holds 8 columns and goes down the rows.
struct SlopeArgs {
    const void *dy, *z;
    const int8_t *q;         // z in 8 bits; null: z, or no activation
    const uint8_t *e;
    void *dz;
    void *laid;              // dz once more, as product_kernel takes it, or null
    float *sums;             // column sums, [workgroups down][sums_width]; null: no bias
    int64_t lddy, ldz, lddz, laid_pitch, rows;
    int dim, pitch, act, sums_width;
};

// Many rows: 32 threads beside each other and 8 below (8 and 32 where the layer is narrow: 100000 x 64 30.7 -> 12.9 us), partial sums of
// many workgroups.  Few rows: one workgroup goes down all of them, 8 threads beside each other and 128 below, and ends the sums itself: no
// second launch (100 x 4096: 4.7 us; 512 x 512 9.1 and 1001 x 250 21.2, bound by the slope's arithmetic on so few compute units, where
// workgroups down the rows and the second launch take 5.9 + 3.0).
constexpr int SLOPE_THREADS = 256, SLOPE_ALONE_ACROSS = 8, SLOPE_ALONE_THREADS = 1024;
constexpr int SLOPE_ROWS = 2;              // rows a thread has in flight
constexpr int64_t SLOPE_ALONE_ROWS = 256;  // one turn of them

template <typename T, typename TY, bool WHOLE, int THREADS, int ACROSS>
__global__ __launch_bounds__(THREADS) void slope_kernel(SlopeArgs a)
{
    constexpr int DOWN = THREADS / ACROSS, COLS = ACROSS * CHUNK, PARTS = THREADS / COLS;
    __shared__ float lds[THREADS * CHUNK];
    const int cx = threadIdx.x % ACROSS, ry = threadIdx.x / ACROSS, c = blockIdx.x * ACROSS + cx, n = chunk_values(c, a.dim);
    f32x8 s = {};
    if (n > 0)
        for (int64_t row = (int64_t)blockIdx.y * DOWN + ry; row < a.rows; row += SLOPE_ROWS * DOWN * (int64_t)gridDim.y) {
            vec<TY, 8> dy[SLOPE_ROWS];
            vec<T, 8> z[SLOPE_ROWS];
            uint64_t q[SLOPE_ROWS];
            uint8_t e[SLOPE_ROWS];
#pragma unroll
            for (int u = 0; u < SLOPE_ROWS; ++u) {
                const int64_t at = row + u * DOWN * (int64_t)gridDim.y, in = at < a.rows ? at : row;
                dy[u] = load_raw<WHOLE>(static_cast<const TY *>(a.dy) + in * a.lddy, c, a.dim);
                if (a.act == DENSE_ACT_NONE) continue;
                if (a.q) {
                    __builtin_memcpy(&q[u], a.q + in * a.pitch + chunk_from(c, a.dim), 8);
                    e[u] = a.e[in * (a.pitch / PACK_BLOCK) + (c >> 2)];
                } else {
                    z[u] = load_raw<WHOLE>(static_cast<const T *>(a.z) + in * a.ldz, c, a.dim);
                }
            }
#pragma unroll
            for (int u = 0; u < SLOPE_ROWS; ++u) {
                const int64_t at = row + u * DOWN * (int64_t)gridDim.y;
                if (at >= a.rows) break;
                f32x8 d = raw_values<WHOLE>(dy[u], c, a.dim);
                if (a.act != DENSE_ACT_NONE) {
                    const f32x8 slope = act_chunk<true>(a.act, a.q ? unpack_chunk(q[u], e[u]) : __builtin_convertvector(z[u], f32x8));
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[j] *= slope[j];
                    d = chunk_only<WHOLE>(d, c, a.dim);
                }
                if (a.dz) store_row<WHOLE>(static_cast<T *>(a.dz) + at * a.lddz, c, a.dim, d);
                if (a.laid) store_some(static_cast<T *>(a.laid) + at * a.laid_pitch + c * CHUNK, chunk_own<WHOLE>(d, c, a.dim), (int)a.laid_pitch - c * CHUNK);
#pragma unroll
                for (int j = 0; j < 8; ++j) s[j] += d[j];
            }
        }
    if (!a.sums) return;
    s = chunk_own<WHOLE>(s, c, a.dim);
#pragma unroll
    for (int j = 0; j < 8; ++j) lds[threadIdx.x * CHUNK + j] = s[j];       // [row of threads][column]
    __syncthreads();
    const int at = threadIdx.x % COLS, part = threadIdx.x / COLS, col = blockIdx.x * COLS + at;
    float t = lds[part * (DOWN / PARTS) * COLS + at];
#pragma unroll
    for (int u = 1; u < DOWN / PARTS; ++u) t += lds[(part * (DOWN / PARTS) + u) * COLS + at];
    if (PARTS > 1) {
        __syncthreads();
        lds[threadIdx.x] = t;
        __syncthreads();
        if (part) return;
#pragma unroll
        for (int u = 1; u < PARTS; ++u) t += lds[u * COLS + at];
    }
    if (col < a.sums_width) a.sums[(size_t)blockIdx.y * a.sums_width + col] = t;
}

// ---- to 8 bits and back -------------------------------------------------------------------------------
struct PackArgs {
    const void *x;
    int8_t *q;
    uint8_t *e;
    int64_t ldx, rows;
    int dim, pitch;
};

// One chunk a thread; the four lanes of a block lie in one wave (the pitch is whole blocks).
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(PackArgs a)
{
    const int per = a.pitch / CHUNK;
    int64_t row;
    int c;
    row_and_piece((int64_t)blockIdx.x * 256 + threadIdx.x, per, row, c);
    if (row >= a.rows) return;                      // (whole blocks: a row has four lanes or a multiple)
    const int n = chunk_values(c, a.dim);
    const f32x8 v = n > 0 ? load_some(static_cast<const T *>(a.x) + row * a.ldx + c * CHUNK, n) : f32x8{};
    pack_chunk(a.q + row * a.pitch, a.e + row * (a.pitch / PACK_BLOCK), c, v);
}

// y = act(gamma v + beta) of the values v that q and e stand for.
struct ExpandArgs {
    const int8_t *q;
    const uint8_t *e;
    const float *gamma, *beta;
    void *y;
    int64_t ldy, rows;
    int dim, pitch, act;
};

// A value that fits the 8-bit form may lie above fp16's largest number by the rounding to whole steps alone (65536 for 65504): it is that number.
template <typename T> __device__ __forceinline__ float within(float v) { return v; }
template <> __device__ __forceinline__ float within<f16>(float v)
{
    return v >= 65520.f && v <= 65536.f ? 65504.f : v <= -65520.f && v >= -65536.f ? -65504.f : v;
}

template <typename T>
__global__ __launch_bounds__(256) void expand_kernel(ExpandArgs a)
{
    const int per = (a.dim + CHUNK - 1) / CHUNK;
    int64_t row;
    int c;
    row_and_piece((int64_t)blockIdx.x * 256 + threadIdx.x, per, row, c);
    if (row >= a.rows) return;
    const int n = chunk_values(c, a.dim);
    uint64_t q;
    __builtin_memcpy(&q, a.q + row * a.pitch + c * CHUNK, 8);
    f32x8 v = unpack_chunk(q, a.e[row * (a.pitch / PACK_BLOCK) + (c >> 2)]);
    if (a.gamma) {
        const f32x8 g = load_some(a.gamma + c * CHUNK, n);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= g[j];
    }
    if (a.beta) {
        const f32x8 b = load_some(a.beta + c * CHUNK, n);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += b[j];
    }
    v = act_chunk<false>(a.act, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = within<T>(v[j]);
    store_some(static_cast<T *>(a.y) + row * a.ldy + c * CHUNK, v, n);
}

} // namespace het
