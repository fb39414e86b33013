// Host side of include/het_dense.h: argument checks and launch shapes.  Nothing is allocated, nothing is kept from call to call.
#include "../../include/het_dense.h"

#include <algorithm>
#include <cstdio>

#include "dense_launch.hpp"

using namespace het;

namespace {

constexpr int64_t MOST_ROWS = (1ll << 31) - 1;
constexpr int32_t MOST_DIM = 1 << 20;
constexpr int64_t MOST_VALUES = 1ll << 40;          // of one matrix (terabytes)

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t align16(int64_t a) { return (a + 15) / 16 * 16; }
int pitch_of(int dim) { return (dim + PACK_BLOCK - 1) / PACK_BLOCK * PACK_BLOCK; }
int width_of(int dim) { return (dim + CHUNK - 1) / CHUNK * CHUNK; }
bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool known_type(int32_t t) { return t == HET_F32 || t == HET_BF16 || t == HET_F16; }
bool known_act(int32_t a) { return a >= HET_ACT_NONE && a <= HET_ACT_SILU; }
int64_t size_of(int32_t t) { return t == HET_F32 ? 4 : 2; }

int launched()
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return HET_OK;
    std::fprintf(stderr, "het_dense: kernel launch: %s\n", hipGetErrorString(e));
    return HET_EHIP;
}

int norm_groups(int64_t rows, const NormShape &h) { return (int)std::min<int64_t>(h.groups, cdiv(rows, h.rows)); }

ColumnSumArgs column_sums(const float *partial, int n, int sets, int dim, float *out0, float *out1)
{
    return ColumnSumArgs{partial, {out0, out1}, n, sets, width_of(dim), dim};
}
void launch_column_sum(const ColumnSumArgs &s, hipStream_t st)
{
    column_sum_kernel<<<(uint32_t)cdiv((int64_t)s.sets * s.width, 16), COLUMN_THREADS, 0, st>>>(s);
}

// f(tag of x's type, tag of y's type) of a known pair.
template <typename T> struct Tag { using type = T; };
template <typename F>
void with_types(int32_t x, int32_t y, F &&f)
{
    if (x == HET_F32) {
        if (y == HET_F32) f(Tag<float>(), Tag<float>());
        else if (y == HET_BF16) f(Tag<float>(), Tag<bf16>());
        else f(Tag<float>(), Tag<f16>());
    } else if (x == HET_BF16) {
        f(Tag<bf16>(), Tag<bf16>());
    } else {
        f(Tag<f16>(), Tag<f16>());
    }
}
template <typename F>
void with_type(int32_t t, F &&f)
{
    if (t == HET_F32) f(Tag<float>());
    else if (t == HET_BF16) f(Tag<bf16>());
    else f(Tag<f16>());
}
void launch_expand(const ExpandArgs &all, int32_t type, hipStream_t st)
{
    const int64_t threads = cdiv(all.dim, CHUNK);
    in_launches(all.rows, threads, [&](int64_t first, int64_t rows) {
        ExpandArgs a = all;
        a.q = moved(a.q, first * a.pitch, 1); a.e = moved(a.e, first * (a.pitch / PACK_BLOCK), 1);
        a.y = moved(a.y, first * a.ldy, size_of(type));
        a.rows = rows;
        with_type(type, [&](auto t) { expand_kernel<typename decltype(t)::type><<<(uint32_t)cdiv(rows * threads, 256), 256, 0, st>>>(a); });
    });
}

// An operand laid out at `to`, which it then is.
void lay(const void *&p, int64_t &ld, int64_t rows, int32_t width, void *to, int32_t type, hipStream_t st)
{
    if (rows > 0) launch_lay(p, ld, rows, width, to, type, st);
    p = to; ld = laid_pitch(width, type);
}

bool known_pair(int32_t x, int32_t y) { return known_type(x) && known_type(y) && (x == y || x == HET_F32); }

bool pack_sizes(int64_t rows, int32_t dim) { return rows >= 0 && rows <= MOST_ROWS && dim >= 1 && dim <= MOST_DIM && rows * dim <= MOST_VALUES; }
bool norm_sizes(int64_t rows, int32_t dim) { return dim >= 1 && dim <= ROW_WIDEST && rows >= 0 && rows <= MOST_ROWS; }

// ---- linear layers ------------------------------------------------------------------------------------
bool linear_sizes(const het_linear_t *l)
{
    return l && l->rows >= 0 && l->rows <= MOST_ROWS - 255 && l->in >= 1 && l->in <= MOST_DIM && l->out >= 1 && l->out <= MOST_DIM && known_type(l->type) &&
           l->rows * std::max(l->in, l->out) <= MOST_VALUES;
}

// Threads beside each other in slope_kernel, and workgroups down the rows: one where they are few, else enough to fill the chip, a turn of rows for
// each at least.
int slope_across(int32_t out) { return out <= 8 * CHUNK ? 8 : out <= 16 * CHUNK ? 16 : 32; }
int slope_splits(int64_t rows, int32_t out)
{
    if (rows <= SLOPE_ALONE_ROWS) return 1;
    const int across = slope_across(out);
    return (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)PARTIALS, cdiv(rows, SLOPE_THREADS / across * SLOPE_ROWS), cdiv(2048, cdiv(out, across * CHUNK))}));
}

template <typename T, typename TY, int THREADS, int ACROSS>
void launch_slope_of(const SlopeArgs &s, int splits, hipStream_t st)
{
    const dim3 grid((uint32_t)cdiv(s.dim, ACROSS * CHUNK), (uint32_t)splits);
    if (s.dim % CHUNK == 0) slope_kernel<T, TY, true, THREADS, ACROSS><<<grid, THREADS, 0, st>>>(s);
    else slope_kernel<T, TY, false, THREADS, ACROSS><<<grid, THREADS, 0, st>>>(s);
}
template <typename T, typename TY>
void launch_slope(const SlopeArgs &s, int splits, hipStream_t st)
{
    const int across = slope_across(s.dim);
    if (splits == 1) launch_slope_of<T, TY, SLOPE_ALONE_THREADS, SLOPE_ALONE_ACROSS>(s, 1, st);
    else if (across == 8) launch_slope_of<T, TY, SLOPE_THREADS, 8>(s, splits, st);
    else if (across == 16) launch_slope_of<T, TY, SLOPE_THREADS, 16>(s, splits, st);
    else launch_slope_of<T, TY, SLOPE_THREADS, 32>(s, splits, st);
}

// Where a call's scratch lies in its workspace, from 0 on in order, each piece at a multiple of 16 bytes.
struct Room {
    int64_t bytes = 0;
    int64_t take(int64_t n) { const int64_t at = bytes; bytes += align16(n); return at; }
    int64_t take_laid(bool lay, int64_t rows, int64_t width, int32_t type) { return take(lay ? rows * laid_pitch(width, type) * size_of(type) : 0); }
};

struct ForwardPlan {
    ProductPlan y;
    int64_t partial_at, x_at, w_at, bytes;
};

ForwardPlan forward_plan(const het_linear_t *l)
{
    ForwardPlan p;
    Room room;
    p.y = product_plan(l->rows, l->out, l->in, l->type, true, true, lay_us(product_lies(l->x, l->ldx, l->in, l->type), l->rows, l->in, l->type),
                       lay_us(product_lies(l->w, l->ldw, l->in, l->type), l->out, l->in, l->type));
    p.partial_at = room.take(p.y.partial_bytes);
    p.x_at = room.take_laid(p.y.lay_a, l->rows, l->in, l->type);
    p.w_at = room.take_laid(p.y.lay_b, l->out, l->in, l->type);
    p.bytes = room.bytes;
    return p;
}

struct BackPlan {
    ProductPlan dx{}, dw{};
    int slope;                  // workgroups down the rows
    bool runs_slope, lay_dz;
    int64_t bias_at, partial_at, dz_at, w_at, x_at, ldx, bytes;
};

BackPlan back_plan(const het_linear_t *l)
{
    BackPlan p;
    Room room;
    const void *dz = l->dz ? l->dz : l->dy;
    const bool dz_lies = product_lies(dz, l->dz ? l->lddz : l->lddy, l->out, l->type);
    p.runs_slope = l->dz || l->dbias;
    p.slope = slope_splits(l->rows, l->out);
    const double dz_us = (p.runs_slope ? written_us : lay_us)(dz_lies, l->rows, l->out, l->type);       // (for each product as if it were the only one)
    if (l->dx) p.dx = product_plan(l->rows, l->in, l->out, l->type, true, false, dz_us, lay_us(product_lies(l->w, l->ldw, l->in, l->type), l->out, l->in, l->type));
    // x in 8 bits is expanded into rows that lie well
    p.ldx = l->xq ? laid_pitch(l->in, l->type) : l->ldx;
    if (l->dw) p.dw = product_plan(l->out, l->in, l->rows, l->type, false, false, dz_us, lay_us(l->xq || product_lies(l->x, l->ldx, l->in, l->type), l->rows, l->in, l->type));
    p.lay_dz = p.dx.lay_a || p.dw.lay_a;
    p.bias_at = room.take(l->dbias && p.slope > 1 ? (int64_t)p.slope * width_of(l->out) * 4 : 0);
    p.partial_at = room.take(std::max(p.dx.partial_bytes, p.dw.partial_bytes));
    p.dz_at = room.take_laid(p.lay_dz, l->rows, l->out, l->type);
    p.w_at = room.take_laid(p.dx.lay_b, l->out, l->in, l->type);
    p.x_at = room.take_laid(l->dw && (l->xq || p.dw.lay_b), l->rows, l->in, l->type);
    p.bytes = room.bytes;
    return p;
}

bool workspace_ok(const void *ws, int64_t have, int64_t need) { return need == 0 || (ws && aligned16(ws) && have >= need); }

} // namespace

extern "C" {

int het_layer_norm(const void *x, int32_t x_type, int64_t ldx, const float *gamma, const float *beta, void *y, int32_t y_type,
                   int64_t ldy, float *mean, float *rstd, int8_t *q, uint8_t *e, int64_t rows, int32_t dim, float eps, void *hip_stream)
{
    if (!norm_sizes(rows, dim) || !known_pair(x_type, y_type) || !(eps >= 0.f) || ldx < dim || ldy < dim || !q != !e) return HET_EINVAL;
    if (rows == 0) return HET_OK;
    if (!x || !y || !aligned16(q)) return HET_EINVAL;
    const NormShape h = norm_shape(dim);
    NormArgs a{x, gamma, beta, y, mean, rstd, q, e, ldx, ldy, rows, h.s, eps};
    with_types(x_type, y_type, [&](auto tx, auto ty) {
        launch_norm<typename decltype(tx)::type, typename decltype(ty)::type>(a, h, static_cast<hipStream_t>(hip_stream));
    });
    return launched();
}

int64_t het_layer_norm_workspace(int64_t rows, int32_t dim)
{
    if (!norm_sizes(rows, dim)) return HET_EINVAL;
    return (int64_t)norm_groups(rows, norm_shape(dim)) * 2 * width_of(dim) * 4;
}

int het_layer_norm_backward(const void *dy, int32_t y_type, int64_t lddy, const void *x, int32_t x_type, int64_t ldx,
                            const float *mean, const float *rstd, const int8_t *q, const uint8_t *e, const float *gamma,
                            const void *residual, int64_t ld_residual, void *dx, int64_t lddx, float *dgamma, float *dbeta,
                            int64_t rows, int32_t dim, void *workspace, int64_t workspace_bytes, void *hip_stream)
{
    if (!norm_sizes(rows, dim) || !known_pair(x_type, y_type) || lddy < dim || lddx < dim || !q != !e) return HET_EINVAL;
    if ((rows > 0 && !q && ldx < dim) || (residual && ld_residual < dim)) return HET_EINVAL;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (rows > 0 && (!dy || !dx || !rstd || (!q && (!x || !mean)) || !aligned16(q))) return HET_EINVAL;
    if (!workspace_ok(workspace, workspace_bytes, het_layer_norm_workspace(rows, dim))) return HET_EINVAL;
    if (rows == 0 && !dgamma && !dbeta) return HET_OK;
    const NormShape h = norm_shape(dim);
    const int groups = norm_groups(rows, h);
    float *partial = static_cast<float *>(workspace);
    if (rows > 0) {
        NormBackArgs a{dy, x, mean, rstd, q, e, gamma, residual, dx, partial, lddy, ldx, ld_residual, lddx, rows, h.s};
        with_types(x_type, y_type, [&](auto tx, auto ty) {
            launch_norm_back<typename decltype(tx)::type, typename decltype(ty)::type>(a, h, groups, st);
        });
    }
    if (dgamma || dbeta) launch_column_sum(column_sums(partial, groups, 2, dim, dgamma, dbeta), st);
    return launched();
}

int het_pack(const void *x, int32_t type, int64_t ldx, int8_t *q, uint8_t *e, int64_t rows, int32_t dim, void *hip_stream)
{
    if (!pack_sizes(rows, dim) || !known_type(type) || ldx < dim) return HET_EINVAL;
    if (rows == 0) return HET_OK;
    if (!x || !q || !e || !aligned16(q)) return HET_EINVAL;
    const int pitch = pitch_of(dim), threads = pitch / CHUNK;
    in_launches(rows, threads, [&](int64_t first, int64_t some) {
        const PackArgs a{moved(x, first * ldx, size_of(type)), q + first * pitch, e + first * (pitch / PACK_BLOCK), ldx, some, dim, pitch};
        with_type(type, [&](auto t) { pack_kernel<typename decltype(t)::type><<<(uint32_t)cdiv(some * threads, 256), 256, 0, static_cast<hipStream_t>(hip_stream)>>>(a); });
    });
    return launched();
}

int het_expand(const int8_t *q, const uint8_t *e, int64_t rows, int32_t dim, const float *gamma, const float *beta, int32_t act,
               void *y, int32_t type, int64_t ldy, void *hip_stream)
{
    if (!pack_sizes(rows, dim) || !known_type(type) || !known_act(act) || ldy < dim) return HET_EINVAL;
    if (rows == 0) return HET_OK;
    if (!y || !q || !e || !aligned16(q)) return HET_EINVAL;
    launch_expand(ExpandArgs{q, e, gamma, beta, y, ldy, rows, dim, pitch_of(dim), act}, type, static_cast<hipStream_t>(hip_stream));
    return launched();
}

int64_t het_linear_workspace(const het_linear_t *l, int32_t backward)
{
    if (!linear_sizes(l)) return HET_EINVAL;
    return backward ? back_plan(l).bytes : forward_plan(l).bytes;
}

int het_linear(const het_linear_t *l, void *hip_stream)
{
    if (!linear_sizes(l) || !known_act(l->act) || (l->y_type != l->type && l->y_type != HET_F32)) return HET_EINVAL;
    if (l->ldx < l->in || l->ldw < l->in || l->ldy < l->out || (l->residual && l->ld_residual < l->out) || (l->z && l->ldz < l->out) || !l->zq != !l->ze) return HET_EINVAL;
    if (l->rows == 0) return HET_OK;
    if (!l->x || !l->w || !l->y || !aligned16(l->zq)) return HET_EINVAL;
    const ForwardPlan p = forward_plan(l);
    if (!p.y.ok || !workspace_ok(l->workspace, l->workspace_bytes, p.bytes)) return HET_EINVAL;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    char *ws = static_cast<char *>(l->workspace);
    ProductArgs a{};
    a.a = l->x; a.lda = l->ldx; a.b = l->w; a.ldb = l->ldw;
    if (p.y.lay_a) lay(a.a, a.lda, l->rows, l->in, ws + p.x_at, l->type, st);
    if (p.y.lay_b) lay(a.b, a.ldb, l->out, l->in, ws + p.w_at, l->type, st);
    a.partial = reinterpret_cast<float *>(ws + p.partial_at);
    a.f.bias = l->bias;
    a.f.residual = l->residual; a.f.ldr = l->ld_residual;
    a.f.y = l->y; a.f.ldy = l->ldy;
    a.f.z = l->z; a.f.ldz = l->ldz;
    a.f.q = l->zq; a.f.e = l->ze; a.f.pitch = pitch_of(l->out);
    a.f.act = l->act;
    a.f.y_f32 = l->y_type == HET_F32;
    launch_product(a, p.y, l->type, true, true, st);
    return launched();
}

int het_linear_backward(const het_linear_t *l, void *hip_stream)
{
    if (!linear_sizes(l) || !known_act(l->act) || !known_act(l->x_act) || (l->y_type != l->type && l->y_type != HET_F32)) return HET_EINVAL;
    const bool has_act = l->act != HET_ACT_NONE, some = l->rows > 0;
    const bool dz_is_dy = !l->dz;
    if (some && dz_is_dy && (has_act || l->y_type != l->type)) return HET_EINVAL;
    if (l->lddy < l->out || (l->dz && l->lddz < l->out)) return HET_EINVAL;
    if (has_act && (!l->zq != !l->ze || (some && !l->zq && l->ldz < l->out))) return HET_EINVAL;
    if (l->dx && (l->lddx < l->in || l->ldw < l->in)) return HET_EINVAL;
    if (l->dw && (l->lddw < l->in || !l->xq != !l->xe || (some && !l->xq && l->ldx < l->in))) return HET_EINVAL;
    if (some) {
        if (!l->dy || (has_act && !l->zq && !l->z) || (has_act && !aligned16(l->zq))) return HET_EINVAL;
        if ((l->dx && !l->w) || (l->dw && !l->xq && !l->x) || (l->dw && !aligned16(l->xq))) return HET_EINVAL;
    }
    const BackPlan p = back_plan(l);
    if ((l->dx && !p.dx.ok) || (l->dw && !p.dw.ok) || !workspace_ok(l->workspace, l->workspace_bytes, p.bytes)) return HET_EINVAL;
    if (!some && !l->dw && !l->dbias) return HET_OK;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    char *ws = static_cast<char *>(l->workspace);
    const void *dz = dz_is_dy ? l->dy : l->dz, *laid = dz;
    int64_t lddz = dz_is_dy ? l->lddy : l->lddz, ld_laid = lddz;
    ColumnSumArgs bias{};               // dbias' parts, if they are still to be added up
    if (p.runs_slope) {
        SlopeArgs s{};
        s.dy = l->dy; s.lddy = l->lddy;
        s.z = l->z; s.ldz = l->ldz; s.q = l->zq; s.e = l->ze;
        s.dz = l->dz; s.lddz = l->lddz;
        if (p.lay_dz) { laid = s.laid = ws + p.dz_at; ld_laid = s.laid_pitch = laid_pitch(l->out, l->type); }
        const bool alone = p.slope == 1;
        s.sums = !l->dbias ? nullptr : alone ? l->dbias : reinterpret_cast<float *>(ws + p.bias_at);
        s.sums_width = alone ? l->out : width_of(l->out);
        s.rows = l->rows; s.dim = l->out; s.pitch = pitch_of(l->out); s.act = l->act;
        with_types(l->y_type, l->type, [&](auto ty, auto t) { launch_slope<typename decltype(t)::type, typename decltype(ty)::type>(s, p.slope, st); });
        if (l->dbias && !alone) bias = column_sums(s.sums, p.slope, 1, l->out, l->dbias, nullptr);
    } else if (p.lay_dz) {
        lay(laid, ld_laid, l->rows, l->out, ws + p.dz_at, l->type, st);
    }
    ProductArgs dx{}, dw{};
    dx.partial = dw.partial = reinterpret_cast<float *>(ws + p.partial_at);
    dx.f.y_f32 = dw.f.y_f32 = l->type == HET_F32;
    const bool wants_dx = l->dx && some;
    if (wants_dx) {
        dx.a = p.dx.lay_a ? laid : dz; dx.lda = p.dx.lay_a ? ld_laid : lddz;
        dx.b = l->w; dx.ldb = l->ldw;
        if (p.dx.lay_b) lay(dx.b, dx.ldb, l->out, l->in, ws + p.w_at, l->type, st);
        dx.f.y = l->dx; dx.f.ldy = l->lddx;
    }
    if (l->dw) {
        dw.a = p.dw.lay_a ? laid : dz; dw.lda = p.dw.lay_a ? ld_laid : lddz;
        dw.b = l->x; dw.ldb = l->ldx;
        if (l->xq) {
            dw.b = ws + p.x_at; dw.ldb = p.ldx;
            if (some) launch_expand(ExpandArgs{l->xq, l->xe, l->x_gamma, l->x_beta, ws + p.x_at, p.ldx, l->rows, l->in, pitch_of(l->in), l->x_act}, l->type, st);
        } else if (p.dw.lay_b) {
            lay(dw.b, dw.ldb, l->rows, l->in, ws + p.x_at, l->type, st);
        }
        dw.f.y = l->dw; dw.f.ldy = l->lddw;
    }
    if (wants_dx && l->dw && launch_small_back(dw, p.dw, dx, p.dx, bias, l->type, st)) return launched();
    if (bias.n) launch_column_sum(bias, st);
    if (wants_dx) launch_product(dx, p.dx, l->type, true, false, st);
    if (l->dw) launch_product(dw, p.dw, l->type, false, false, st);
    return launched();
}

} // extern "C"
