// Matrix products of the dense layers on the matrix cores, with what follows them (bias, activation, residual, 8-bit copy) done while the
// sums are still in registers.
//
// All are D[m][n] = sum over k of A(m, k) B(n, k).  An operand is read along k (K: its rows are A's or B's, as x and w are in x w^T) or
// across (its rows are k's, as w is in dz w, and both are in dz^T x); nothing is transposed in memory.
#pragma once
#include "dense_rows.hpp"

namespace het {

// What becomes of a sum: z = sum + bias is kept where the backward pass needs it, y = act(z) + residual.
struct Finish {
    const float *bias;        // null: none
    const void *residual;     // of y's type, or null
    void *y;
    void *z;                  // z in the operands' type, or null
    int8_t *q;                // z in 8 bits, or null
    uint8_t *e;
    int64_t ldr, ldy, ldz;
    int pitch, act;
    int y_f32;                // y and residual are fp32 whatever the operands are
};

struct ProductArgs {
    const void *a, *b;
    int64_t lda, ldb;
    int m, n, k;
    int tiles_m, tiles_n;
    int splits, k_split;      // the k's of a workgroup: k_split of them, a multiple of the kernel's step
    float *partial;           // splits > 1: [split][m][n rounded up to 16], joined by join_kernel
    Finish f;
};

__device__ __forceinline__ int partial_width(int n) { return (n + 15) & ~15; }

// The n values of bias and residual that belong to a chunk at (row, col); zero behind the row's end and where there are none.
__device__ __forceinline__ f32x8 finish_bias(const Finish &f, int col, int n) { return f.bias && n > 0 ? load_some(f.bias + col, n) : f32x8{}; }
template <typename T>
__device__ __forceinline__ f32x8 finish_residual(const Finish &f, int64_t row, int col, int n)
{
    if (!f.residual || n <= 0) return f32x8{};
    const int64_t at = row * f.ldr + col;
    return f.y_f32 ? load_some(static_cast<const float *>(f.residual) + at, n) : load_some(static_cast<const T *>(f.residual) + at, n);
}

// Ends z of that chunk.
template <typename T>
__device__ __forceinline__ void finish_value(const Finish &f, int64_t row, int col, int n, f32x8 v, f32x8 residual)
{
    if (n <= 0) return;
    if (f.z) store_some(static_cast<T *>(f.z) + row * f.ldz + col, v, n);
    v = act_chunk<false>(f.act, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += residual[j];
    if (f.y_f32) store_some(static_cast<float *>(f.y) + row * f.ldy + col, v, n);
    else store_some(static_cast<T *>(f.y) + row * f.ldy + col, v, n);
}

__device__ __forceinline__ f32x8 plus(f32x8 a, f32x8 b)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] += b[j];
    return a;
}

// ---- operands in LDS ------------------------------------------------------------------------------------
// A step takes 128 bytes of k from each row of a tile: 64 values of 16 bits, 32 of fp32.  The matrix instructions take 16 bytes of k a lane
// (`frag`): one 32x32x16 product of 16-bit values, or four 32x32x2 products of fp32, so a step is four frags in either case.
//
// The first operand of an instruction is B, the second A: a lane then holds one row of D and 16 columns.  Which row of the tile stands at
// which of the instruction's 32 rows is free; B's stand so that these 16 columns are neighbours (col_of).
template <typename T> struct Frag;
template <> struct Frag<bf16> { using type = vec<bf16, 8>; };
template <> struct Frag<f16> { using type = vec<f16, 8>; };
template <> struct Frag<float> { using type = f32x4; };

__device__ __forceinline__ f32x16 multiply(vec<bf16, 8> a, vec<bf16, 8> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 multiply(vec<f16, 8> a, vec<f16, 8> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 multiply(f32x4 a, f32x4 b, f32x16 c)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ f32x4 multiply_small(vec<bf16, 8> a, vec<bf16, 8> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply_small(vec<f16, 8> a, vec<f16, 8> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 multiply_small(f32x4 a, f32x4 b, f32x4 c)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

// The instruction's row i of 32 -> column of D within the tile's 32: lane half h holds rows 8 (v / 4) + 4 h + v % 4 of the result (v = 0 .. 15),
// which are to be the columns 16 h + v.
__device__ __forceinline__ int col_of(int i) { return 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3); }

// An operand's tile in LDS: R rows and 128 bytes of k.
//   K:  [row][128 bytes], pieces of 16 bytes;  across:  [k][R values].
// The order of a row's pieces is mixed by the row's (or k's) number, so that the 16 lanes whose 16 bytes are read at a time meet all 64 banks: rows
// of 128 bytes two by two, and of the permuted operand the rows that col_of brings together.  (Mixed by the last three bits, as 32 banks would
// want it, half of the reads conflicted: 2.5e7 cycles in 8192 x 4096 -> 4096; now none do.)
template <typename T, int R, bool K, bool PERMUTED>
struct Tile {
    static constexpr int PIECE = 16 / (int)sizeof(T);             // values of a piece
    static constexpr int STEP = 128 / (int)sizeof(T);             // k's of a step
    static constexpr int PIECES = R * 8;
    static constexpr int WIDE = K ? 8 : R / PIECE;                // pieces of a row of the tile in LDS
    using F = typename Frag<T>::type;

    __device__ static __forceinline__ int mixed(int r, int c)     // place of piece c of row (or k) r
    {
        if (K) return r * 8 + (c ^ (PERMUTED ? (r >> 1 & 3) | (r >> 2 & 4) : r >> 1 & 7));
        if (sizeof(T) == 2) return r * WIDE + (c ^ (4 * (r & 3)));
        return r * WIDE + (c ^ (8 * ((r >> 2) & 1)));
    }
    // Frag `s` (0 .. 3) of the 32 rows from r0.
    __device__ static __forceinline__ F read(const i32x4 *lds, int r0, int s)
    {
        const int lane = threadIdx.x % 64, h = lane / 32;
        if (K) {
            const int r = r0 + (PERMUTED ? col_of(lane % 32) : lane % 32);
            return __builtin_bit_cast(F, lds[mixed(r, 2 * s + h)]);
        }
        return across(lds, r0, s, F{});
    }
    // 16 bits, across: two transposing reads.  In each, the 16 lanes of a group name 4 k's of 16 rows, 4 values a lane, and every lane gets the 4 k's of
    // one row.
    template <typename V>
    __device__ static __forceinline__ V across(const i32x4 *lds, int r0, int s, V)
    {
        using S = vec<short, 4>;
        using P = __attribute__((address_space(3))) S *;
        const int lane = threadIdx.x % 64, g = lane / 16, i = lane % 16, k = 16 * s + 8 * (g / 2) + i / 4;
        const int in = 16 * (g % 2) + 4 * (i % 4), r = r0 + (PERMUTED ? col_of(in) : in);
        const char *base = reinterpret_cast<const char *>(lds);
        const S lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(base + mixed(k, r / 8) * 16 + r % 8 * 2));
        const S hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(base + mixed(k + 4, r / 8) * 16 + r % 8 * 2));
        return __builtin_bit_cast(V, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    __device__ static __forceinline__ f32x4 across(const i32x4 *lds, int r0, int s, f32x4)
    {
        const int lane = threadIdx.x % 64, k = 8 * s + 4 * (lane / 32), r = r0 + (PERMUTED ? col_of(lane % 32) : lane % 32);
        const float *base = reinterpret_cast<const float *>(lds);
        f32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = base[mixed(k + j, r / 4) * 4 + r % 4];
        return v;
    }
};

// Workgroups are handed to the 8 XCDs in turn; each gets a run of neighbouring tiles, whose operands its own L2 then holds.
__device__ __forceinline__ int tile_of(int block, int tiles)
{
    const int x = block % 8, each = tiles / 8, more = tiles % 8;
    return x * each + (x < more ? x : more) + block / 8;
}

// Tiles in bands of 8 rows of tiles: neighbours share A's rows or B's.
__device__ __forceinline__ void tile_at(int t, int tiles_m, int tiles_n, int &tm, int &tn)
{
    const int band = t / (8 * tiles_n), first = band * 8, high = tiles_m - first < 8 ? tiles_m - first : 8, in = t - band * 8 * tiles_n;
    tm = first + in % high;
    tn = in / high;
}

// Outputs and residuals pass the L2, which holds the operands that neighbouring tiles share (4096 x 1664 -> 4096 with gelu and z in 8 bits 72.5 -> 70.5 us
// with its expansion).

// Four chunks at `col` of the rows row, row + 8, ... of 16-bit outputs, or of any with z kept; sums(r): the chunk of row r of the 32.
template <typename T, typename TY, typename S>
__device__ __forceinline__ void finish_whole(const Finish &f, int64_t row, int col, S &&sums)
{
    const int first = threadIdx.x % 64 / 8;
    vec<TY, 8> res[4];
    if (f.residual)
#pragma unroll
        for (int it = 0; it < 4; ++it) __builtin_memcpy(&res[it], static_cast<const TY *>(f.residual) + (row + 8 * it) * f.ldr + col, sizeof(res[it]));
    const f32x8 bias = f.bias ? load_chunk(f.bias + col) : f32x8{};
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int64_t at = row + 8 * it;
        f32x8 v = plus(sums(first + 8 * it), bias);
        if (f.q) pack_chunk(f.q + at * f.pitch, f.e + at * (f.pitch / PACK_BLOCK), col / CHUNK, v);
        if (f.z) store_chunk(static_cast<T *>(f.z) + at * f.ldz + col, v);
        v = act_chunk<false>(f.act, v);
        if (f.residual) v = plus(v, __builtin_convertvector(res[it], f32x8));
        TY *y = static_cast<TY *>(f.y) + at * f.ldy + col;
        if constexpr (sizeof(TY) == 2) store_past(y, __builtin_convertvector(v, vec<TY, 8>));
        else store_chunk(y, v);
    }
}

// The same for fp32 outputs alone: a lane has two pieces of four columns, col and col + 32, so that eight lanes' pieces are whole 128-byte lines (with
// eight neighbouring columns a lane each store is half of every line: 8192 x 4096 -> 4096 with an fp32 residual 287 us, so 276).
template <typename S>
__device__ __forceinline__ void finish_pieces(const Finish &f, int64_t row, int col, S &&sums)
{
    const int first = threadIdx.x % 64 / 8;
    f32x4 res[4][2], bias[2] = {};
    if (f.residual)
#pragma unroll
        for (int it = 0; it < 4; ++it)
#pragma unroll
            for (int h = 0; h < 2; ++h) res[it][h] = load_past<f32x4>(static_cast<const float *>(f.residual) + (row + 8 * it) * f.ldr + col + 32 * h);
    if (f.bias)
#pragma unroll
        for (int h = 0; h < 2; ++h) __builtin_memcpy(&bias[h], f.bias + col + 32 * h, 16);
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        f32x8 v = plus(sums(first + 8 * it), __builtin_shufflevector(bias[0], bias[1], 0, 1, 2, 3, 4, 5, 6, 7));
        v = act_chunk<false>(f.act, v);
        if (f.residual) v = plus(v, __builtin_shufflevector(res[it][0], res[it][1], 0, 1, 2, 3, 4, 5, 6, 7));
        float *y = static_cast<float *>(f.y) + (row + 8 * it) * f.ldy + col;
        store_past(y, __builtin_shufflevector(v, v, 0, 1, 2, 3));
        store_past(y + 32, __builtin_shufflevector(v, v, 4, 5, 6, 7));
    }
}

// Ends a wave's 32 x 64 sums at (row0, col0).  They go through the wave's own 8 KB of LDS (the tiles' are free by then), so that eight lanes
// hold a row's 64 columns side by side: whole 128-byte pieces of rows are stored, four lanes share a block of the 8-bit form, and the
// code is there once for all of a lane's sums.
constexpr int FINISH_PIECES = 32 * 64 / 4;

template <typename T>
__device__ __forceinline__ void finish_tile(const ProductArgs &a, int split, int row0, int col0, const f32x16 &left, const f32x16 &right, f32x4 *lds)
{
    const int lane = threadIdx.x % 64;
    {
        const int r = lane % 32, h = lane / 32;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");        // the lanes' reads of what was there before
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            lds[r * 16 + ((4 * h + q) ^ (r & 7))] = f32x4{left[4 * q], left[4 * q + 1], left[4 * q + 2], left[4 * q + 3]};
            lds[r * 16 + ((8 + 4 * h + q) ^ (r & 7))] = f32x4{right[4 * q], right[4 * q + 1], right[4 * q + 2], right[4 * q + 3]};
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    const int c = lane % 8, col = col0 + c * CHUNK;
    auto sums = [&](int r) {
        const f32x4 lo = lds[r * 16 + ((2 * c) ^ (r & 7))], hi = lds[r * 16 + ((2 * c + 1) ^ (r & 7))];
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    const bool whole = row0 + 32 <= a.m && col0 + 64 <= a.n;           // all of it in the matrix: no edge is looked for, four rows' residuals are under way
    auto pieces = [&](int r) {                                         // two pieces of four columns, 32 apart
        const f32x4 lo = lds[r * 16 + (c ^ (r & 7))], hi = lds[r * 16 + ((8 + c) ^ (r & 7))];
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    if (a.splits > 1) {
        const int width = partial_width(a.n);
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int r = 8 * it + lane / 8, row = row0 + r;
            if (col < width && row < a.m) store_chunk(a.partial + ((int64_t)split * a.m + row) * width + col, sums(r));
        }
    } else if (whole && a.f.y_f32 && !a.f.q && !a.f.z) {
        finish_pieces(a.f, row0 + lane / 8, col0 + 4 * c, pieces);
    } else if (whole) {
        if (a.f.y_f32) finish_whole<T, float>(a.f, row0 + lane / 8, col, sums);
        else finish_whole<T, T>(a.f, row0 + lane / 8, col, sums);
    } else if (col0 + (c & ~3) * CHUNK < a.n) {                        // (a block's four lanes go together)
#pragma unroll 1
        for (int it = 0; it < 4; ++it) {
            const int r = 8 * it + lane / 8, row = row0 + r, n = a.n - col;
            if (row >= a.m) return;
            const f32x8 v = plus(sums(r), finish_bias(a.f, col, n));
            if (a.f.q) pack_chunk(a.f.q + (int64_t)row * a.f.pitch, a.f.e + (int64_t)row * (a.f.pitch / PACK_BLOCK), col / CHUNK, v);
            finish_value<T>(a.f, row, col, n, v, finish_residual<T>(a.f, row, col, n));
        }
    }
}

// The wave's part of two tiles' LDS.
template <int WAVES>
__device__ __forceinline__ f32x4 *finish_room(i32x4 *first, i32x4 *second)
{
    const int wave = threadIdx.x / 64;
    return reinterpret_cast<f32x4 *>(wave < WAVES / 2 ? first : second) + wave % (WAVES / 2) * FINISH_PIECES;
}

// ---- aligned operands -------------------------------------------------------------------------------------
// TM x TN tiles, WM x WN waves.  Memory goes straight to LDS, 16 bytes a lane, STAGES - 1 steps ahead of the products: the next steps' pieces are on their
// way while a step is multiplied, and nothing passes through registers.  Pieces behind an edge are asked for outside the buffer's range, which
// reads as zero.  Operands' rows begin at multiples of 16 bytes and are whole pieces wide; others are laid out so first (lay_kernel): pieces taken
// through registers from rows that begin anywhere cost more (2051 x 3001 -> 2049 in bf16 172 us, laid out 51; in fp32 484 and 275).
// The workgroup's barrier between two steps: every wave has its LDS reads in registers (lgkmcnt(0)) and its copies done but for the last N asked
// for (vmcnt(N)).  __syncthreads() would wait for all copies, those of later steps too; the fences keep the compiler from moving reads or copies
// across.
template <int N> __device__ __forceinline__ void step_barrier()
{
    static_assert(N < 64, "vmcnt's range");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | N >> 4 << 14);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_sched_barrier(0);
}

template <typename T, int R, bool K, bool PERMUTED, int THREADS>
struct Copy : Tile<T, R, K, PERMUTED> {
    using B = Tile<T, R, K, PERMUTED>;
    static constexpr int EACH = B::PIECES / THREADS;
    static constexpr int OUTSIDE = (int)0x80000000;
    int at[EACH];               // byte offsets of this thread's pieces from the tile's corner; OUTSIDE: behind the matrix' last row
    int64_t advance;            // bytes from a step to the next
    const char *corner;

    // row0: the tile's first row; k0: the first k.
    __device__ __forceinline__ Copy(const T *p, int64_t ld, int row0, int rows, int k0)
    {
        corner = reinterpret_cast<const char *>(p + (K ? (int64_t)row0 * ld + k0 : (int64_t)k0 * ld + row0));
        advance = (K ? (int64_t)B::STEP : B::STEP * ld) * (int64_t)sizeof(T);
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            const int i = u * THREADS + threadIdx.x, down = i / B::WIDE, along = along_of(i);
            const int row = K ? down : along * B::PIECE;
            at[u] = row0 + row < rows ? (int)((down * ld + along * B::PIECE) * (int64_t)sizeof(T)) : OUTSIDE;
        }
    }
    // The piece that belongs at place i: mixing is its own inverse.
    __device__ static __forceinline__ int along_of(int i) { return B::mixed(i / B::WIDE, i % B::WIDE) % B::WIDE; }

    // The step's pieces to `lds`; `left`: k's from its first to the end (a step beyond the last whole one is cut off).
    __device__ __forceinline__ void step(i32x4 *lds, int left)
    {
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(corner), 0, 0x7FFFFFFF, 0x00020000);
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            const int i = u * THREADS + threadIdx.x, k = K ? along_of(i) * B::PIECE : i / B::WIDE;
            const int from = left >= B::STEP || k < left ? at[u] : OUTSIDE;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)(lds + u * THREADS + wave * 64), 16, from, 0, 0, 0);
        }
        corner += advance;
    }
};

template <typename T, bool AK, bool BK, int TM, int TN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(ProductArgs a)
{
    constexpr int THREADS = 64 * WM * WN, MI = TM / WM / 32, NI = TN / WN / 32, S = STAGES;
    static_assert(S == 2 || S == 4, "the loop's buffers");
    using CA = Copy<T, TM, AK, false, THREADS>;
    using CB = Copy<T, TN, BK, true, THREADS>;
    // (arrays of their own, and a loop of as many steps: the compiler sees that a step's reads do not wait for the other buffers' copies)
    __shared__ i32x4 a0[CA::PIECES], a1[CA::PIECES], b0[CB::PIECES], b1[CB::PIECES];
    __shared__ i32x4 a2[S > 2 ? CA::PIECES : 1], a3[S > 2 ? CA::PIECES : 1], b2[S > 2 ? CB::PIECES : 1], b3[S > 2 ? CB::PIECES : 1];
    const int tiles = a.tiles_m * a.tiles_n, split = blockIdx.x / tiles;
    int tm, tn;
    tile_at(tile_of(blockIdx.x % tiles, tiles), a.tiles_m, a.tiles_n, tm, tn);
    const int row0 = tm * TM, col0 = tn * TN;
    const int k_begin = split * a.k_split, k_end = a.k - k_begin < a.k_split ? a.k : k_begin + a.k_split;
    const int wave = threadIdx.x / 64, wm = wave / WN * (TM / WM), wn = wave % WN * (TN / WN);
    CA ca(static_cast<const T *>(a.a), a.lda, row0, a.m, k_begin);
    CB cb(static_cast<const T *>(a.b), a.ldb, col0, a.n, k_begin);
    f32x16 acc[MI][NI] = {};
    typename CA::F fa[2][MI];
    typename CB::F fb[2][NI];
    auto read = [&](const i32x4 *la, const i32x4 *lb, int s, int to) {
#pragma unroll
        for (int i = 0; i < MI; ++i) fa[to][i] = CA::read(la, wm + 32 * i, s);
#pragma unroll
        for (int j = 0; j < NI; ++j) fb[to][j] = CB::read(lb, wn + 32 * j, s);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto products = [&](int of) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = multiply(fb[of][j], fa[of][i], acc[i][j]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // A frag's reads go out before the products of the frag before.  The last frag of a step is in registers before its products start: at that point
    // the buffer is free for the step S ahead, and the next step's first frag can be read.  The copies of one operand go out among those
    // last products, the other's among the first ones of the next step: all of them at once held the products up (8192 x 4096 -> 4096 bf16: dw 231 -> 216 us).
    constexpr int EACH = CA::EACH + CB::EACH, STEP = CA::STEP;
    int left = k_end - k_begin;                     // from the step's first k on
    auto step = [&](i32x4 *la, i32x4 *lb, i32x4 *next_a, i32x4 *next_b, i32x4 *before_b) {
        read(la, lb, 1, 1);
        cb.step(before_b, left - (S - 1) * STEP);
        products(0);
        read(la, lb, 2, 0);
        products(1);
        read(la, lb, 3, 1);
        products(0);
        step_barrier<(S - 2) * EACH>();
        left -= STEP;
        read(next_a, next_b, 0, 0);
        ca.step(la, left - (S - 1) * STEP);
        products(1);
    };
    // S steps a turn, the last of them perhaps of zeros: with a step of its own behind the loop the compiler keeps the sums twice (and spills).
    const int steps = (left + STEP - 1) / STEP;
    ca.step(a0, left); cb.step(b0, left);
    if constexpr (S > 2) {
        ca.step(a1, left - STEP); cb.step(b1, left - STEP);
        ca.step(a2, left - 2 * STEP); cb.step(b2, left - 2 * STEP);
    }
    step_barrier<(S - 2) * EACH>();
    ca.step(S > 2 ? a3 : a1, left - (S - 1) * STEP);
    read(a0, b0, 0, 0);
    for (int t = 0; t < (steps + S - 1) / S; ++t) {
        if constexpr (S > 2) {
            step(a0, b0, a1, b1, b3);
            step(a1, b1, a2, b2, b0);
            step(a2, b2, a3, b3, b1);
            step(a3, b3, a0, b0, b2);
        } else {
            step(a0, b0, a1, b1, b1);
            step(a1, b1, a0, b0, b0);
        }
    }
    static_assert(NI == 2 && CA::PIECES >= WM * WN / 2 * FINISH_PIECES, "a wave ends 64 columns, in the tiles' LDS");
    step_barrier<0>();                              // (zeros for steps that do not come)
    f32x4 *room = finish_room<WM * WN>(a0, a1);
    // (the code once, with the sums moved up: four copies of it are more than the instruction cache holds)
#pragma unroll 1
    for (int i = 0; i < MI; ++i) {
        finish_tile<T>(a, split, row0 + wm + 32 * i, col0 + wn, acc[0][0], acc[0][1], room);
#pragma unroll
        for (int u = 0; u + 1 < MI; ++u) { acc[u][0] = acc[u + 1][0]; acc[u][1] = acc[u + 1][1]; }
    }
}

// Rows that begin anywhere -> rows of `pitch` values that begin at multiples of 16 bytes, zero behind the end.  A piece a thread.
template <typename U>
__global__ __launch_bounds__(256) void lay_kernel(const U *p, int64_t ld, int64_t rows, int width, U *to, int pitch)
{
    constexpr int PIECE = 16 / (int)sizeof(U);
    const int per = pitch / PIECE;
    int64_t row;
    int at;
    row_and_piece((int64_t)blockIdx.x * 256 + threadIdx.x, per, row, at);
    if (row >= rows) return;
    at *= PIECE;
    const U *from = p + row * ld;
    vec<U, PIECE> v = {};
    if (at + PIECE <= width) {
        __builtin_memcpy(&v, from + at, 16);
    } else {
#pragma unroll
        for (int j = 0; j < PIECE - 1; ++j) if (at + j < width) v[j] = from[at + j];
    }
    *reinterpret_cast<vec<U, PIECE> *>(to + row * pitch + at) = v;
}

// Adds the splits' sums and ends them.  A chunk a thread, four for each block of 32 columns (the 8-bit copy needs them side by side); of many splits
// every PARTS-th for each of PARTS threads, whose sums are added in order.  Four loads are under way: one after the other they took 10 us for 32 splits
// of a 16 x 16 product.
template <typename T, int PARTS>
__global__ __launch_bounds__(256) void join_kernel(ProductArgs a)
{
    constexpr int CHUNKS = 256 / PARTS, DEEP = 4;
    __shared__ float lds[PARTS > 1 ? PARTS : 1][PARTS > 1 ? CHUNKS : 1][CHUNK + 1];
    const int width = partial_width(a.n), per = (a.n + PACK_BLOCK - 1) / PACK_BLOCK * 4, at = threadIdx.x % CHUNKS, part = threadIdx.x / CHUNKS;
    int64_t row;
    int c;
    row_and_piece((int64_t)blockIdx.x * CHUNKS + at, per, row, c);
    const int col = c * CHUNK, n = a.n - col;
    const bool ends = part == 0 && row < a.m;
    const f32x8 bias = ends ? finish_bias(a.f, col, n) : f32x8{}, residual = ends ? finish_residual<T>(a.f, row, col, n) : f32x8{};
    f32x8 v = {};
    if (row < a.m && n > 0) {
        const float *p = a.partial + row * width + col;
        for (int s = part; s < a.splits; s += DEEP * PARTS) {
            f32x8 x[DEEP];
#pragma unroll
            for (int u = 0; u < DEEP; ++u) x[u] = load_chunk(p + (int64_t)(s + u * PARTS < a.splits ? s + u * PARTS : s) * a.m * width);
#pragma unroll
            for (int u = 0; u < DEEP; ++u)
                if (s + u * PARTS < a.splits)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] += x[u][j];
        }
    }
    if (PARTS > 1) {
#pragma unroll
        for (int j = 0; j < 8; ++j) lds[part][at][j] = v[j];
        __syncthreads();
    }
    if (!ends) return;
#pragma unroll
    for (int u = 1; u < PARTS; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += lds[u][at][j];
    v = plus(v, bias);
    if (a.f.q) pack_chunk(a.f.q + row * a.f.pitch, a.f.e + row * (a.f.pitch / PACK_BLOCK), c, v);
    finish_value<T>(a.f, row, col, n, v, residual);
}

// ---- few rows, or small products --------------------------------------------------------------------------
// Bound by latency, or by reading w once for a request's few rows.  A workgroup takes 16 MT x 16 NT of D and its waves share k, each every
// SMALL_WAVES-th span of 128 bytes; operands go from memory into the matrix instructions' registers, two spans at a time, and the waves' sums meet in
// LDS.  A lane's two pieces of a span lie side by side, so that the four lanes of a row take whole lines.
constexpr int SMALL_WAVES = 8;

template <typename T, bool K>
struct Direct {
    static constexpr int PIECE = 16 / (int)sizeof(T);
    using F = typename Frag<T>::type;
    const T *p;                  // the lane's row, or its column of the first row of k's
    int64_t ld;
    __device__ __forceinline__ void set(const T *base, int64_t ld_, int row, int rows)
    {
        ld = ld_;
        const int r = row < rows ? row : rows - 1;          // (rows behind the last one are its copies; what comes of them is not stored)
        p = base + (K ? (int64_t)r * ld : (int64_t)r);
    }
    __device__ __forceinline__ F load(int k) const
    {
        F f;
        if (K) __builtin_memcpy(&f, p + k, 16);
        else
#pragma unroll
            for (int j = 0; j < PIECE; ++j) f[j] = p[(k + j) * ld];
        return f;
    }
    // Zero from `end` on.  No lane takes a branch of its own: a piece that would cross the end is the last one before it, shifted.
    __device__ __forceinline__ F load_edge(int k, int end) const
    {
        if (K && end >= PIECE) {
            const int from = k < end - PIECE ? k : end - PIECE, over = k - from;
            unsigned __int128 v;
            __builtin_memcpy(&v, p + from, 16);
            v = over < PIECE ? v >> (8 * (int)sizeof(T) * over) : 0;
            return __builtin_bit_cast(F, v);
        }
        F f;
#pragma unroll
        for (int j = 0; j < PIECE; ++j) {
            const int at = k + j < end ? k + j : end - 1;
            f[j] = p[K ? (int64_t)at : at * ld];
        }
#pragma unroll
        for (int j = 0; j < PIECE; ++j) f[j] = k + j < end ? f[j] : (T)0.f;
        return f;
    }
};

template <int MT, int NT> struct SmallRoom { float sums[SMALL_WAVES][16 * MT][16 * NT + 4]; };

template <typename T, bool AK, bool BK, int MT, int NT>
__device__ __forceinline__ void product_small(const ProductArgs &a, int block, float (*lds)[16 * MT][16 * NT + 4])
{
    using DA = Direct<T, AK>;
    using DB = Direct<T, BK>;
    constexpr int SPAN = 8 * DA::PIECE, AHEAD = MT * NT == 1 ? 4 : 2;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), r = lane % 16, g = lane / 16;
    const int row0 = block / a.tiles_n * 16 * MT, col0 = block % a.tiles_n * 16 * NT;
    // the chunk this thread ends, and what is added to it, asked for ahead
    const int c = threadIdx.x % (2 * NT), at = threadIdx.x / (2 * NT), row = row0 + at, col = col0 + c * CHUNK, n = a.n - col;
    const bool ends = at < 16 * MT && row < a.m;
    const f32x8 bias = ends ? finish_bias(a.f, col, n) : f32x8{}, residual = ends ? finish_residual<T>(a.f, row, col, n) : f32x8{};
    f32x4 acc[MT][NT] = {};
    auto products = [&](const typename DA::F *fa, const typename DB::F *fb) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = multiply_small(fb[j], fa[i], acc[i][j]);
    };
    DA da[MT];
    DB db[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) da[i].set(static_cast<const T *>(a.a), a.lda, row0 + 16 * i + r, a.m);
#pragma unroll
    for (int j = 0; j < NT; ++j) db[j].set(static_cast<const T *>(a.b), a.ldb, col0 + 16 * j + r, a.n);
    const int whole = a.k / SPAN;                     // spans without an edge
    for (int t = wave; t < whole; t += AHEAD * SMALL_WAVES) {
        typename DA::F fa[AHEAD][2][MT];
        typename DB::F fb[AHEAD][2][NT];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int span = t + u * SMALL_WAVES, k = (span < whole ? span : t) * SPAN + 2 * g * DA::PIECE;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
#pragma unroll
                for (int j = 0; j < NT; ++j) fb[u][s][j] = db[j].load(k + s * DA::PIECE);
#pragma unroll
                for (int i = 0; i < MT; ++i) fa[u][s][i] = da[i].load(k + s * DA::PIECE);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (t + u * SMALL_WAVES < whole) { products(fa[u][0], fb[u][0]); products(fa[u][1], fb[u][1]); }
    }
    if (whole * SPAN < a.k && wave == whole % SMALL_WAVES) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int k = whole * SPAN + (2 * g + s) * DA::PIECE;
            typename DA::F fa[MT];
            typename DB::F fb[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) fb[j] = db[j].load_edge(k, a.k);
#pragma unroll
            for (int i = 0; i < MT; ++i) fa[i] = da[i].load_edge(k, a.k);
            products(fa, fb);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) *reinterpret_cast<f32x4 *>(&lds[wave][16 * i + r][16 * j + 4 * g]) = acc[i][j];
    __syncthreads();
    if (!ends) return;
    f32x8 v = {};
#pragma unroll
    for (int w = 0; w < SMALL_WAVES; ++w)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += lds[w][at][c * CHUNK + j];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? v[j] : 0.f;
    v = plus(v, bias);
    if (NT == 2 && a.f.q) pack_chunk(a.f.q + (int64_t)row * a.f.pitch, a.f.e + (int64_t)row * (a.f.pitch / PACK_BLOCK), col / CHUNK, v);
    finish_value<T>(a.f, row, col, n, v, residual);
}

template <typename T, bool AK, bool BK, int MT, int NT>
__global__ __launch_bounds__(64 * SMALL_WAVES) void product_small_kernel(ProductArgs a)
{
    __shared__ SmallRoom<MT, NT> lds;
    product_small<T, AK, BK, MT, NT>(a, blockIdx.x, lds.sums);
}

// What a small layer's backward pass does once dz is there, in one launch: dw, dx, and the sums of dbias' parts.  None needs another's results, and
// each alone leaves most of the chip waiting for memory: 1001 x 500 -> 250 in fp16, 2.9 + 5.7 + 6.8 us one after the other, 11.0 together (and two
// launches fewer).
struct SmallBackArgs {
    ProductArgs dw, dx;
    ColumnSumArgs bias;
    int dw_groups, dx_groups;           // workgroups of each; those behind them are the sums'
    int dx_first;                       // the products' order: the one with the longer sums starts first
};

template <typename T, int NW, int NX>
__global__ __launch_bounds__(64 * SMALL_WAVES) void small_back_kernel(SmallBackArgs a)
{
    __shared__ union { SmallRoom<2, NW> dw; SmallRoom<2, NX> dx; float bias[COLUMN_DEEP][17]; } lds;
    const int block = blockIdx.x, dw = block - (a.dx_first ? a.dx_groups : 0), dx = block - (a.dx_first ? 0 : a.dw_groups);
    if (dw >= 0 && dw < a.dw_groups) product_small<T, false, false, 2, NW>(a.dw, dw, lds.dw.sums);
    else if (dx >= 0 && dx < a.dx_groups) product_small<T, true, false, 2, NX>(a.dx, dx, lds.dx.sums);
    else column_sum<64 * SMALL_WAVES>(a.bias, block - a.dw_groups - a.dx_groups, lds.bias);
}

} // namespace het
