// C entry points of the layers in 8-bit floating point, group norm and the
// gradients' norm: validation and dispatch.  The contract of every entry point
// is in include/hpacmlt.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <new>
#include <vector>

#include "columns.hpp"
#include "f8.hpp"
#include "gradients.hpp"
#include "group_norm.hpp"
#include "operands.hpp"

using namespace hpacml;
using f8::Matrix;

namespace {

hpacml_status matrix_status(const hpacmlt_matrix *m) {
    if (!m || m->rows < 0 || m->width < 0)
        return HPACML_E_INVAL;
    return m->rows > kMaxRows || m->width > kMaxRows || f8::too_many_blocks(m->rows, m->width) ? HPACML_E_UNSUPPORTED : HPACML_OK;
}
Matrix matrix_of(const hpacmlt_matrix &m) { return {(char *)m.codes, (char *)m.scales, m.rows, m.width}; }
void add_matrix(Operands *o, const hpacmlt_matrix &m, bool written) {
    const int64_t codes = f8::codes_bytes(m.rows, m.width), scales = f8::scales_bytes(m.rows, m.width);
    o->add(m.codes, codes > 0, codes, codes, 1, 16, written);
    o->add(m.scales, scales > 0, scales, scales, 1, 16, written);
}

// Parts of a call's scratch memory, one after another.
struct Layout {
    size_t bytes = 0;
    size_t take(int64_t n) {
        const size_t at = bytes;
        bytes += ((size_t)n + 255) / 256 * 256;
        return at;
    }
};
struct MatrixAt {
    size_t codes, scales;
    Matrix in(char *scratch, int64_t rows, int64_t width) const { return {scratch + codes, scratch + scales, rows, width}; }
};
MatrixAt take_matrix(Layout *l, int64_t rows, int64_t width) {
    MatrixAt m;
    m.codes = l->take(f8::codes_bytes(rows, width));
    m.scales = l->take(f8::scales_bytes(rows, width));
    return m;
}

struct LinearLayout : Layout {
    MatrixAt x{};
    size_t partial = 0;
    LinearLayout(int64_t rows, int64_t n_in, int64_t n_out) {
        if (f8::few_rows(rows, n_out, n_in))
            return;
        x = take_matrix(this, rows, n_in);
        partial = take(f8::product_partial_bytes(rows, n_out, n_in));
    }
};

struct BackwardLayout : Layout {
    MatrixAt by_row{}, by_column{};
    size_t sums = 0, room = 0, partial = 0;
    BackwardLayout(int64_t rows, int64_t n_in, int64_t n_out, bool dw, bool db, bool dx) {
        int64_t most = 0;
        if (dx) {
            by_row = take_matrix(this, rows, n_out);
            most = f8::product_partial_bytes(rows, n_in, n_out);
        }
        if (dw) {
            by_column = take_matrix(this, n_out, rows);
            const int64_t b = f8::product_partial_bytes(n_out, n_in, rows);
            most = b > most ? b : most;
        }
        if (db) {
            sums = take(f8::blocks_of(rows) * n_out * 4);
            room = take(column_sums_room(f8::blocks_of(rows), n_out) * 4);
        }
        partial = take(most);
    }
};

hpacml_status norm_status(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups) {
    if (!is_type(dtype) || images < 0 || points < 1 || channels < 1 || groups < 1 || channels % groups != 0)
        return HPACML_E_INVAL;
    if (channels > HPACMLT_MAX_CHANNELS || points > kMaxRows || images > kMaxRows / points || images > INT32_MAX / groups)
        return HPACML_E_UNSUPPORTED;
    return HPACML_OK;
}
bool is_norm_act(int32_t a) { return is_act(a) || a == HPACMLT_ACT_SILU; }

// Whether device memory of `device` holds `bytes` from p on.  Gradients share
// allocations: the last few found are looked at first.
class Allocations {
    static constexpr int kMost = 8;
    struct Range {
        const char *base = nullptr;
        size_t size = 0;
    } known[kMost];
    int next = 0;

  public:
    hpacml_status holds(const void *p, int64_t bytes, int device) {
        const Span v{(const char *)p, 1, bytes, bytes, false};
        for (const Range &r : known)
            if (r.base && inside(v, r.base, r.size))
                return HPACML_OK;
        hipPointerAttribute_t attr;
        hipDeviceptr_t base = nullptr;
        size_t size = 0;
        if (!p || hipPointerGetAttributes(&attr, p) != hipSuccess ||
            (attr.type != hipMemoryTypeDevice && attr.type != hipMemoryTypeManaged) || attr.device != device ||
            hipMemGetAddressRange(&base, &size, (hipDeviceptr_t)p) != hipSuccess) {
            (void)hipGetLastError();
            return HPACML_E_INVAL;
        }
        known[next++ % kMost] = {(const char *)base, size};
        return inside(v, (const char *)base, size) ? HPACML_OK : HPACML_E_RANGE;
    }
};

struct Extent {
    const char *at, *end;
    bool written;
};

}  // namespace

struct hpacmlt_gradients_s {
    int device = 0;
    GradChunk *chunks = nullptr;
    int64_t n = 0;
    std::vector<Extent> extents;        // by address
    // whether [at, at + bytes) is apart from every gradient
    bool apart(const void *p, int64_t bytes) const {
        const char *at = (const char *)p;
        for (const Extent &e : extents)
            if (e.at < at + bytes && at < e.end)
                return false;
        return true;
    }
};

namespace {

hpacml_status gradients_status(const hpacmlt_gradients *set, int32_t kind, float *norm, void *scratch, size_t scratch_bytes) {
    if (!set || (kind != HPACMLT_NORM_2 && kind != HPACMLT_NORM_MAX))
        return HPACML_E_INVAL;
    if (scratch_bytes < kGradScratch)
        return HPACML_E_RANGE;
    Operands o;
    o.add(norm, 1, 1, 1, 4, 4, true);
    o.add(scratch, 1, kGradScratch, kGradScratch, 1, 16, true);
    if (o.check() != HPACML_OK)
        return o.status;
    if (o.device != set->device)
        return HPACML_E_INVAL;
    return set->apart(norm, 4) && set->apart(scratch, kGradScratch) ? HPACML_OK : HPACML_E_ALIAS;
}

}  // namespace

extern "C" {

hpacml_status hpacmlt_matrix_bytes(int64_t rows, int64_t width, size_t *codes, size_t *scales) {
    const hpacmlt_matrix m = {nullptr, nullptr, rows, width};
    const hpacml_status s = matrix_status(&m);
    if (s != HPACML_OK)
        return s;
    if (!codes || !scales)
        return HPACML_E_INVAL;
    *codes = (size_t)f8::codes_bytes(rows, width);
    *scales = (size_t)f8::scales_bytes(rows, width);
    return HPACML_OK;
}

hpacml_status hpacmlt_quantize(const void *x, int32_t dtype, int64_t ldx, int64_t rows, int64_t width, const hpacmlt_matrix *by_row,
                               const hpacmlt_matrix *by_column, int32_t square, void *stream) {
    if (!is_type(dtype) || rows < 0 || width < 0 || (!by_row && !by_column) || !pitch_ok(ldx, width))
        return HPACML_E_INVAL;
    if (rows > kMaxRows || width > kMaxRows || f8::too_many_blocks(rows, width))
        return HPACML_E_UNSUPPORTED;
    for (const hpacmlt_matrix *m : {by_row, by_column})
        if (m) {
            const hpacml_status s = matrix_status(m);
            if (s != HPACML_OK)
                return s;
        }
    if ((by_row && (by_row->rows != rows || by_row->width != width)) || (by_column && (by_column->rows != width || by_column->width != rows)))
        return HPACML_E_SHAPE;
    if (rows == 0 || width == 0)
        return HPACML_OK;
    Operands o;
    o.add(x, rows, width, ldx, size_of(dtype), size_of(dtype), false);
    if (by_row)
        add_matrix(&o, *by_row, true);
    if (by_column)
        add_matrix(&o, *by_column, true);
    if (o.check() != HPACML_OK)
        return o.status;
    f8::QuantizeArgs a = {x, nullptr, ldx, 0, rows, width, {}, {}, nullptr, square != 0};
    if (by_row)
        a.by_row = matrix_of(*by_row);
    if (by_column)
        a.by_column = matrix_of(*by_column);
    return status_of(f8::launch_quantize(a, dtype, (hipStream_t)stream));
}

hpacml_status hpacmlt_load(const hpacmlt_matrix *m, void *x, int32_t dtype, int64_t ldx, void *stream) {
    const hpacml_status s = matrix_status(m);
    if (s != HPACML_OK)
        return s;
    if (!is_type(dtype) || !pitch_ok(ldx, m->width))
        return HPACML_E_INVAL;
    if (m->rows == 0 || m->width == 0)
        return HPACML_OK;
    Operands o;
    add_matrix(&o, *m, false);
    o.add(x, m->rows, m->width, ldx, size_of(dtype), size_of(dtype), true);
    if (o.check() != HPACML_OK)
        return o.status;
    return status_of(f8::launch_load(matrix_of(*m), x, dtype, ldx, (hipStream_t)stream));
}

hpacml_status hpacmlt_product_scratch(int64_t p_rows, int64_t q_rows, int64_t width, size_t *bytes) {
    if (!bytes || p_rows < 0 || q_rows < 0 || width < 0)
        return HPACML_E_INVAL;
    if (p_rows > kMaxRows || q_rows > kMaxRows || width > kMaxRows)
        return HPACML_E_UNSUPPORTED;
    *bytes = (size_t)f8::product_partial_bytes(p_rows, q_rows, width);
    return HPACML_OK;
}

hpacml_status hpacmlt_product(const hpacmlt_matrix *p, const hpacmlt_matrix *q, const float *b, int32_t act, void *y, int32_t y_dtype, int64_t ldy,
                              int32_t accumulate, void *scratch, size_t scratch_bytes, void *stream) {
    hpacml_status s = matrix_status(p);
    if (s == HPACML_OK)
        s = matrix_status(q);
    if (s != HPACML_OK)
        return s;
    if (!is_type(y_dtype) || !is_act(act) || !pitch_ok(ldy, q->rows) ||
        (accumulate && (y_dtype != HPACML_F32 || b || act != HPACML_ACT_IDENTITY)))
        return HPACML_E_INVAL;
    if (p->width != q->width)
        return HPACML_E_SHAPE;
    if (p->rows == 0 || q->rows == 0)
        return HPACML_OK;
    const int64_t need = f8::product_partial_bytes(p->rows, q->rows, p->width);
    if ((int64_t)scratch_bytes < need)
        return HPACML_E_RANGE;
    Operands o;
    add_matrix(&o, *p, false);
    add_matrix(&o, *q, false);
    if (b)
        o.add(b, 1, q->rows, q->rows, 4, 4, false);
    o.add(y, p->rows, q->rows, ldy, size_of(y_dtype), size_of(y_dtype), true);
    o.add(scratch, need > 0, need, need, 1, 16, true);
    if (o.check() != HPACML_OK)
        return o.status;
    return status_of(f8::launch_product({matrix_of(*p), matrix_of(*q), b, y, ldy, act == HPACML_ACT_RELU, accumulate != 0, (float *)scratch},
                                        y_dtype, (hipStream_t)stream));
}

hpacml_status hpacmlt_linear_scratch(const hpacmlt_matrix *W, int64_t rows, size_t *bytes) {
    const hpacml_status s = matrix_status(W);
    if (s != HPACML_OK)
        return s;
    if (!bytes || rows < 0 || W->rows < 1 || W->width < 1)
        return HPACML_E_INVAL;
    if (rows > kMaxRows || f8::too_many_blocks(rows, W->width))
        return HPACML_E_UNSUPPORTED;
    *bytes = rows ? LinearLayout(rows, W->width, W->rows).bytes : 0;
    return HPACML_OK;
}

hpacml_status hpacmlt_linear_run(const hpacmlt_matrix *W, const float *b, const void *x, int32_t x_dtype, int64_t ldx, int64_t rows, void *y,
                                 int32_t y_dtype, int64_t ldy, int32_t act, const hpacmlt_matrix *keep, void *scratch, size_t scratch_bytes,
                                 void *stream) {
    hpacml_status s = matrix_status(W);
    if (s == HPACML_OK && keep)
        s = matrix_status(keep);
    if (s != HPACML_OK)
        return s;
    if (W->rows < 1 || W->width < 1 || !is_type(x_dtype) || !is_type(y_dtype) || !is_act(act) || rows < 0 || !pitch_ok(ldx, W->width) ||
        !pitch_ok(ldy, W->rows))
        return HPACML_E_INVAL;
    if (rows > kMaxRows || f8::too_many_blocks(rows, W->width))
        return HPACML_E_UNSUPPORTED;
    if (keep && (keep->rows != W->width || keep->width != rows))
        return HPACML_E_SHAPE;
    if (rows == 0)
        return HPACML_OK;
    const LinearLayout l(rows, W->width, W->rows);
    if (scratch_bytes < l.bytes)
        return HPACML_E_RANGE;
    Operands o;
    add_matrix(&o, *W, false);
    if (b)
        o.add(b, 1, W->rows, W->rows, 4, 4, false);
    o.add(x, rows, W->width, ldx, size_of(x_dtype), size_of(x_dtype), false);
    o.add(y, rows, W->rows, ldy, size_of(y_dtype), size_of(y_dtype), true);
    if (keep)
        add_matrix(&o, *keep, true);
    o.add(scratch, l.bytes > 0, (int64_t)l.bytes, (int64_t)l.bytes, 1, 16, true);
    if (o.check() != HPACML_OK)
        return o.status;
    hipStream_t st = (hipStream_t)stream;
    const Matrix kept = keep ? matrix_of(*keep) : Matrix{};
    f8::ProductArgs product = {{nullptr, nullptr, rows, W->width}, matrix_of(*W), b, y, ldy, act == HPACML_ACT_RELU, 0, nullptr};
    if (f8::few_rows(rows, W->rows, W->width)) {
        hipError_t e = keep ? f8::launch_quantize({x, nullptr, ldx, 0, rows, W->width, Matrix{}, kept, nullptr, 0}, x_dtype, st) : hipSuccess;
        return status_of(e == hipSuccess ? f8::launch_linear_few(product, x, x_dtype, ldx, y_dtype, st) : e);
    }
    product.p = l.x.in((char *)scratch, rows, W->width);
    product.partial = (float *)((char *)scratch + l.partial);
    hipError_t e = f8::launch_quantize({x, nullptr, ldx, 0, rows, W->width, product.p, kept, nullptr, 0}, x_dtype, st);
    return status_of(e == hipSuccess ? f8::launch_product(product, y_dtype, st) : e);
}

hpacml_status hpacmlt_backward_scratch(int64_t rows, int64_t n_in, int32_t n_out, int32_t want_dw, int32_t want_db, int32_t want_dx,
                                       size_t *bytes) {
    if (!bytes || rows < 0 || n_in < 1 || n_out < 1)
        return HPACML_E_INVAL;
    if (rows > kMaxRows || n_in > kMaxRows || f8::too_many_blocks(rows, n_out) || f8::too_many_blocks(rows, n_in))
        return HPACML_E_UNSUPPORTED;
    *bytes = rows ? BackwardLayout(rows, n_in, n_out, want_dw != 0, want_db != 0, want_dx != 0).bytes : 0;
    return HPACML_OK;
}

hpacml_status hpacmlt_backward(const hpacmlt_matrix *kept, const void *dy, const void *y, int32_t dtype, int64_t lddy, int64_t ldy, int32_t n_out,
                               const hpacmlt_matrix *Wt, float *dw, int64_t lddw, float *db, void *dx, int64_t lddx, int32_t accumulate,
                               void *scratch, size_t scratch_bytes, void *stream) {
    hpacml_status s = matrix_status(kept);
    if (s == HPACML_OK && dx)
        s = matrix_status(Wt);
    if (s != HPACML_OK)
        return s;
    const int64_t rows = kept->width, n_in = kept->rows;
    if (!is_type(dtype) || n_out < 1 || n_in < 1 || !pitch_ok(lddy, n_out) || (y && !pitch_ok(ldy, n_out)) || (!dw && !db && !dx) ||
        (dw && !pitch_ok(lddw, n_in)) || (dx && !pitch_ok(lddx, n_in)))
        return HPACML_E_INVAL;
    if (f8::too_many_blocks(rows, n_out))
        return HPACML_E_UNSUPPORTED;
    if (dx && (Wt->rows != n_in || Wt->width != n_out))
        return HPACML_E_SHAPE;
    const BackwardLayout l(rows, n_in, n_out, dw, db, dx);
    if (rows && scratch_bytes < l.bytes)
        return HPACML_E_RANGE;
    const int64_t es = size_of(dtype);
    Operands o;
    o.add(dy, rows, n_out, lddy, es, es, false);
    if (y)
        o.add(y, rows, n_out, ldy, es, es, false);
    if (dw) {
        add_matrix(&o, *kept, false);
        o.add(dw, n_out, n_in, lddw, 4, 4, true);
    }
    if (db)
        o.add(db, 1, n_out, n_out, 4, 4, true);
    if (dx) {
        add_matrix(&o, *Wt, false);
        o.add(dx, rows, n_in, lddx, es, es, true);
    }
    o.add(scratch, rows > 0, (int64_t)l.bytes, (int64_t)l.bytes, 1, 16, true);
    if (o.check() != HPACML_OK)
        return o.status;
    hipStream_t st = (hipStream_t)stream;
    if (rows == 0) {
        hipError_t e = hipSuccess;
        if (!accumulate && dw)
            e = f8::launch_product({{nullptr, nullptr, n_out, 0}, {nullptr, nullptr, n_in, 0}, nullptr, dw, lddw, 0, 0, nullptr}, HPACML_F32, st);
        if (!accumulate && db && e == hipSuccess)
            e = launch_column_sums({nullptr, 0, n_out, 0, db, nullptr, n_out, 0, nullptr}, st);
        return status_of(e);
    }
    char *at = (char *)scratch;
    const Matrix by_row = dx ? l.by_row.in(at, rows, n_out) : Matrix{}, by_column = dw ? l.by_column.in(at, n_out, rows) : Matrix{};
    float *sums = db ? (float *)(at + l.sums) : nullptr, *partial = (float *)(at + l.partial);
    hipError_t e = f8::launch_quantize({dy, y, lddy, ldy, rows, n_out, by_row, by_column, sums, 0}, dtype, st);
    if (e == hipSuccess && db)
        e = launch_column_sums({sums, f8::blocks_of(rows), n_out, n_out, db, nullptr, n_out, accumulate != 0, (float *)(at + l.room)}, st);
    if (e == hipSuccess && dx)
        e = f8::launch_product({by_row, matrix_of(*Wt), nullptr, dx, lddx, 0, 0, partial}, dtype, st);
    if (e == hipSuccess && dw)
        e = f8::launch_product({by_column, matrix_of(*kept), nullptr, dw, lddw, 0, accumulate != 0, partial}, HPACML_F32, st);
    return status_of(e);
}

hpacml_status hpacmlt_group_norm_scratch(int32_t dtype, int64_t images, int64_t points, int32_t channels, int32_t groups, int32_t backward,
                                         size_t *bytes) {
    const hpacml_status s = norm_status(dtype, images, points, channels, groups);
    if (s != HPACML_OK)
        return s;
    if (!bytes)
        return HPACML_E_INVAL;
    *bytes = (size_t)group_norm_scratch(dtype, images, points, channels, groups, backward != 0);
    return HPACML_OK;
}

hpacml_status hpacmlt_group_norm(const void *x, int32_t dtype, int64_t ldx, int64_t images, int64_t points, int32_t channels, int32_t groups,
                                 const float *gamma, const float *beta, float eps, int32_t act, void *y, int64_t ldy, float *mean, float *rstd,
                                 void *scratch, size_t scratch_bytes, void *stream) {
    const hpacml_status s = norm_status(dtype, images, points, channels, groups);
    if (s != HPACML_OK)
        return s;
    if (!pitch_ok(ldx, channels) || !pitch_ok(ldy, channels) || !(eps >= FLT_MIN) || std::isinf(eps) || !is_norm_act(act) || !mean != !rstd)
        return HPACML_E_INVAL;
    if (images == 0)
        return HPACML_OK;
    const int64_t need = group_norm_scratch(dtype, images, points, channels, groups, false), es = size_of(dtype), rows = images * points;
    if ((int64_t)scratch_bytes < need)
        return HPACML_E_RANGE;
    Operands o;
    o.add(x, rows, channels, ldx, es, es, false);
    if (gamma)
        o.add(gamma, 1, channels, channels, 4, 4, false);
    if (beta)
        o.add(beta, 1, channels, channels, 4, 4, false);
    o.add(y, rows, channels, ldy, es, es, true);
    if (mean) {
        o.add(mean, 1, images * groups, images * groups, 4, 4, true);
        o.add(rstd, 1, images * groups, images * groups, 4, 4, true);
    }
    o.add(scratch, need > 0, need, need, 1, 16, true);
    if (o.check() != HPACML_OK)
        return o.status;
    GroupNorm a = {x, ldx, images, points, channels, groups, gamma, beta, eps, act, mean, rstd, y, ldy};
    a.scratch = (char *)scratch;
    return status_of(launch_group_norm(a, dtype, (hipStream_t)stream));
}

hpacml_status hpacmlt_group_norm_backward(const void *x, int32_t dtype, int64_t ldx, int64_t images, int64_t points, int32_t channels,
                                          int32_t groups, const float *gamma, const float *beta, int32_t act, const float *mean, const float *rstd,
                                          const void *dy, int64_t lddy, void *dx, int64_t lddx, float *dgamma, float *dbeta, int32_t accumulate,
                                          void *scratch, size_t scratch_bytes, void *stream) {
    const hpacml_status s = norm_status(dtype, images, points, channels, groups);
    if (s != HPACML_OK)
        return s;
    if (!pitch_ok(ldx, channels) || !pitch_ok(lddy, channels) || !is_norm_act(act) || (!dx && !dgamma && !dbeta) || (dx && !pitch_ok(lddx, channels)))
        return HPACML_E_INVAL;
    const int64_t need = images ? group_norm_scratch(dtype, images, points, channels, groups, true) : 0, es = size_of(dtype), rows = images * points;
    if ((int64_t)scratch_bytes < need)
        return HPACML_E_RANGE;
    Operands o;
    o.add(x, rows, channels, ldx, es, es, false);
    if (gamma)
        o.add(gamma, 1, channels, channels, 4, 4, false);
    if (beta)
        o.add(beta, 1, channels, channels, 4, 4, false);
    o.add(mean, 1, images * groups, images * groups, 4, 4, false);
    o.add(rstd, 1, images * groups, images * groups, 4, 4, false);
    o.add(dy, rows, channels, lddy, es, es, false);
    if (dx)
        o.add(dx, rows, channels, lddx, es, es, true);
    if (dgamma)
        o.add(dgamma, 1, channels, channels, 4, 4, true);
    if (dbeta)
        o.add(dbeta, 1, channels, channels, 4, 4, true);
    o.add(scratch, need > 0, need, need, 1, 16, true);
    if (o.check() != HPACML_OK)
        return o.status;
    GroupNorm a = {x, ldx, images, points, channels, groups, gamma, beta, 0.f, act, const_cast<float *>(mean), const_cast<float *>(rstd), dx, lddx};
    a.dy = dy;
    a.lddy = lddy;
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.accumulate = accumulate != 0;
    a.scratch = (char *)scratch;
    return status_of(launch_group_norm_backward(a, dtype, (hipStream_t)stream));
}

hpacml_status hpacmlt_gradients_create(const hpacmlt_gradient *gradients, int64_t n, hpacmlt_gradients **out) {
    if (!out)
        return HPACML_E_INVAL;
    *out = nullptr;
    if (n < 0 || (n && !gradients))
        return HPACML_E_INVAL;
    int device = 0;
    if (hipGetDevice(&device) != hipSuccess) {
        (void)hipGetLastError();
        return HPACML_E_DEVICE;
    }
    hpacmlt_gradients *set = nullptr;
    try {
        std::vector<Extent> extents;
        std::vector<GradChunk> chunks;
        Allocations known;
        int64_t total = 0;
        for (int64_t i = 0; i < n; ++i) {
            const hpacmlt_gradient &g = gradients[i];
            if (g.count < 0 || !is_type(g.from_dtype) || !is_type(g.to_dtype))
                return HPACML_E_INVAL;
            if (g.count == 0)
                continue;
            if (g.from == g.to && g.from_dtype != g.to_dtype)
                return HPACML_E_INVAL;
            if (g.count > INT64_MAX / 8)
                return HPACML_E_RANGE;
            const int64_t from = g.count * size_of(g.from_dtype), to = g.count * size_of(g.to_dtype);
            if (((uintptr_t)g.from & (size_of(g.from_dtype) - 1)) || ((uintptr_t)g.to & (size_of(g.to_dtype) - 1)))
                return HPACML_E_INVAL;
            hpacml_status s = known.holds(g.from, from, device);
            if (s == HPACML_OK && g.to != g.from)
                s = known.holds(g.to, to, device);
            if (s != HPACML_OK)
                return s;
            if (g.to != g.from)
                extents.push_back({(const char *)g.from, (const char *)g.from + from, false});
            extents.push_back({(const char *)g.to, (const char *)g.to + to, true});
            total += g.count;
        }
        // nothing written meets anything else
        std::sort(extents.begin(), extents.end(), [](const Extent &a, const Extent &b) { return a.at < b.at; });
        const char *end = nullptr, *written = nullptr;
        for (const Extent &e : extents) {
            if (e.at < written || (e.written && e.at < end))
                return HPACML_E_ALIAS;
            end = std::max(end, e.end);
            if (e.written)
                written = std::max(written, e.end);
        }
        const int64_t per = grad_chunk(total);
        for (int64_t i = 0; i < n; ++i) {
            const hpacmlt_gradient &g = gradients[i];
            const int32_t types = (g.from_dtype == HPACML_BF16) | (g.to_dtype == HPACML_BF16) << 1;
            for (int64_t at = 0; at < g.count; at += per)
                chunks.push_back({(const char *)g.from + at * size_of(g.from_dtype), (char *)g.to + at * size_of(g.to_dtype),
                                  (int32_t)std::min(per, g.count - at), types});
        }
        set = new hpacmlt_gradients_s;
        set->device = device;
        set->n = (int64_t)chunks.size();
        set->extents = std::move(extents);
        hipError_t e = hipDeviceSynchronize();
        if (e == hipSuccess && set->n)
            e = hipMalloc((void **)&set->chunks, chunks.size() * sizeof(GradChunk));
        if (e == hipSuccess && set->n)
            e = hipMemcpy(set->chunks, chunks.data(), chunks.size() * sizeof(GradChunk), hipMemcpyHostToDevice);
        if (e != hipSuccess) {
            (void)hipGetLastError();
            hpacmlt_gradients_destroy(set);
            return status_of(e);
        }
    } catch (const std::exception &) {
        hpacmlt_gradients_destroy(set);
        return HPACML_E_NOMEM;
    }
    *out = set;
    return HPACML_OK;
}

void hpacmlt_gradients_destroy(hpacmlt_gradients *set) {
    if (!set)
        return;
    if (set->chunks)
        (void)hipFree(set->chunks);
    delete set;
}

hpacml_status hpacmlt_gradients_scratch(const hpacmlt_gradients *set, size_t *bytes) {
    if (!set || !bytes)
        return HPACML_E_INVAL;
    *bytes = kGradScratch;
    return HPACML_OK;
}

hpacml_status hpacmlt_gradients_norm(const hpacmlt_gradients *set, int32_t kind, float *norm, void *scratch, size_t scratch_bytes, void *stream) {
    const hpacml_status s = gradients_status(set, kind, norm, scratch, scratch_bytes);
    if (s != HPACML_OK)
        return s;
    return status_of(launch_grad_norm(set->chunks, set->n, kind, norm, scratch, (hipStream_t)stream));
}

hpacml_status hpacmlt_gradients_clip(const hpacmlt_gradients *set, int32_t kind, double most, float *norm, void *scratch, size_t scratch_bytes,
                                     void *stream) {
    if (!(most >= 0))
        return HPACML_E_INVAL;
    const hpacml_status s = gradients_status(set, kind, norm, scratch, scratch_bytes);
    if (s != HPACML_OK)
        return s;
    return status_of(launch_grad_clip(set->chunks, set->n, kind, most, norm, scratch, (hipStream_t)stream));
}

}  // extern "C"
