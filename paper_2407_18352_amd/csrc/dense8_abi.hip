// C entry points of the 8-bit dense layers: handles, validation, dispatch.
// The contract of every entry point is in include/hpacml8.h.
#include <hip/hip_runtime.h>

#include <new>

#include "dense8.hpp"
#include "operands.hpp"

using namespace hpacml;

struct hpacml8_linear_s {
    int device = 0;
    int32_t n_in = 0, n_out = 0;
    int32_t slabs = 0;
    char *buf = nullptr;      // codes, blocked, then scales and biases, each to a multiple of four
    int8_t *w = nullptr;
    float *t = nullptr, *b = nullptr;
};

namespace {

hpacml_status checkpoint_status(const hpacml8_checkpoint *c) {
    if (!c || !is_act(c->act) || c->rows < 0 || c->width < 1)
        return HPACML_E_INVAL;
    if (c->width > HPACML8_MAX_WIDTH || c->rows > kMaxRows)
        return HPACML_E_UNSUPPORTED;
    if (!pitch_ok(c->ld_codes, c->width) || c->ld_codes % HPACML8_BLOCK != 0 ||
        !pitch_ok(c->ld_exps, (c->width + HPACML8_BLOCK - 1) / HPACML8_BLOCK))
        return HPACML_E_INVAL;
    return HPACML_OK;
}

void add_checkpoint(Operands *o, const hpacml8_checkpoint &c, bool written) {
    const int64_t blocks = (c.width + HPACML8_BLOCK - 1) / HPACML8_BLOCK;
    o->add(c.codes, c.rows, blocks * HPACML8_BLOCK, c.ld_codes, 1, 16, written);
    o->add(c.exps, c.rows, blocks, c.ld_exps, 1, 1, written);
}

// A host or device array to be read once: in device memory it has to lie inside
// its allocation.  here (may be NULL): floats of device `device`, which its
// kernels can read where they are.
hpacml_status source_status(const void *p, int64_t bytes, int device, bool *here) {
    hipPointerAttribute_t attr;
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    if (hipPointerGetAttributes(&attr, p) != hipSuccess) {
        (void)hipGetLastError();       // host memory that the runtime does not know
        return HPACML_OK;
    }
    if (attr.type != hipMemoryTypeDevice)
        return HPACML_OK;
    if (hipMemGetAddressRange(&base, &size, (hipDeviceptr_t)p) != hipSuccess) {
        (void)hipGetLastError();
        return HPACML_E_INVAL;
    }
    if (here)
        *here = attr.device == device && ((uintptr_t)p & 3) == 0;
    return inside({(const char *)p, 1, bytes, bytes, false}, (const char *)base, size) ? HPACML_OK : HPACML_E_RANGE;
}

// scratch of hpacml8_linear_run: codes, then scales
int64_t linear_scratch_rows(const hpacml8_linear *l, int64_t rows) { return linear8_scratch_rows(rows, l->n_in, l->n_out); }
size_t linear_codes_bytes(const hpacml8_linear *l, int64_t rows) { return (size_t)blocked_bytes(linear_scratch_rows(l, rows), l->slabs); }
size_t linear_scratch_bytes(const hpacml8_linear *l, int64_t rows) {
    return linear_codes_bytes(l, rows) + (size_t)linear_scratch_rows(l, rows) * 4;
}

}  // namespace

extern "C" {

hpacml_status hpacml8_linear_create(int32_t n_in, int32_t n_out, const float *W, const float *b, hpacml8_linear **out) {
    if (!out)
        return HPACML_E_INVAL;
    *out = nullptr;
    if (n_in < 1 || n_out < 1 || !W)
        return HPACML_E_INVAL;
    if (n_in > HPACML8_MAX_WIDTH || n_out > HPACML8_MAX_WIDTH)
        return HPACML_E_UNSUPPORTED;
    int device = 0;
    bool w_here = false;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        return status_of(e);
    }
    hpacml_status source = source_status(W, (int64_t)n_out * n_in * 4, device, &w_here);
    if (source == HPACML_OK && b)
        source = source_status(b, (int64_t)n_out * 4, device, nullptr);
    if (source != HPACML_OK)
        return source;
    hpacml8_linear *l = new (std::nothrow) hpacml8_linear_s;
    if (!l)
        return HPACML_E_NOMEM;
    l->n_in = n_in;
    l->n_out = n_out;
    l->slabs = (int32_t)slabs_of(n_in);
    float *staged = nullptr;
    const size_t codes = (size_t)blocked_bytes(n_out, l->slabs), wbytes = (size_t)n_out * n_in * 4, outs = ((size_t)n_out + 3) / 4 * 4;
    l->device = device;
    e = hipDeviceSynchronize();
    if (e == hipSuccess)
        e = hipMalloc((void **)&l->buf, codes + outs * 8);
    if (e == hipSuccess && !w_here)
        e = hipMalloc((void **)&staged, wbytes);
    if (e == hipSuccess) {
        l->w = (int8_t *)l->buf;
        l->t = (float *)(l->buf + codes);
        l->b = l->t + outs;
        e = hipMemset(l->t, 0, outs * 8);
    }
    if (e == hipSuccess && !w_here)
        e = hipMemcpy(staged, W, wbytes, hipMemcpyDefault);
    if (e == hipSuccess && b)
        e = hipMemcpy(l->b, b, (size_t)n_out * 4, hipMemcpyDefault);
    if (e == hipSuccess)
        e = launch_codes_by_row(w_here ? W : staged, HPACML_F32, n_in, n_out, n_in, l->w, l->t, nullptr);
    if (e == hipSuccess)
        e = hipDeviceSynchronize();
    if (staged)
        (void)hipFree(staged);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        hpacml8_linear_destroy(l);
        return status_of(e);
    }
    *out = l;
    return HPACML_OK;
}

void hpacml8_linear_destroy(hpacml8_linear *l) {
    if (!l)
        return;
    if (l->buf)
        (void)hipFree(l->buf);
    delete l;
}

hpacml_status hpacml8_linear_scratch(const hpacml8_linear *l, int64_t n_rows, size_t *bytes) {
    if (!l || !bytes || n_rows < 0)
        return HPACML_E_INVAL;
    if (n_rows > kMaxRows)
        return HPACML_E_UNSUPPORTED;
    *bytes = linear_scratch_bytes(l, n_rows);
    return HPACML_OK;
}

hpacml_status hpacml8_linear_run(const hpacml8_linear *l, const void *x, int32_t x_dtype, int64_t ldx, int64_t n_rows,
                                 void *y, int32_t y_dtype, int64_t ldy, int32_t act, void *scratch,
                                 size_t scratch_bytes, void *stream) {
    if (!l || !is_type(x_dtype) || !is_type(y_dtype) || !is_act(act) || n_rows < 0 || !pitch_ok(ldx, l->n_in) ||
        !pitch_ok(ldy, l->n_out))
        return HPACML_E_INVAL;
    if (n_rows > kMaxRows)
        return HPACML_E_UNSUPPORTED;
    if (n_rows == 0)
        return HPACML_OK;
    const size_t need = linear_scratch_bytes(l, n_rows);
    if (scratch_bytes < need)
        return HPACML_E_RANGE;
    Operands o;
    o.add(x, n_rows, l->n_in, ldx, size_of(x_dtype), size_of(x_dtype), false);
    o.add(y, n_rows, l->n_out, ldy, size_of(y_dtype), size_of(y_dtype), true);
    o.add(scratch, 1, (int64_t)need, (int64_t)need, 1, 16, true);
    if (o.check() != HPACML_OK)
        return o.status;
    if (o.device != l->device)
        return HPACML_E_INVAL;
    hipStream_t st = (hipStream_t)stream;
    int8_t *q = (int8_t *)scratch;
    float *s = (float *)((char *)scratch + linear_codes_bytes(l, n_rows));
    return status_of(launch_linear8({x, ldx, q, s, l->w, l->t, l->b, y, n_rows, ldy, l->slabs, l->n_in, l->n_out, act == HPACML_ACT_RELU},
                                    x_dtype, y_dtype, st));
}

hpacml_status hpacml8_checkpoint_save(const hpacml8_checkpoint *c, const void *z, int32_t z_dtype, int64_t ldz, void *a,
                                      int32_t a_dtype, int64_t lda, void *stream) {
    const hpacml_status s = checkpoint_status(c);
    if (s != HPACML_OK)
        return s;
    if (!is_type(z_dtype) || !pitch_ok(ldz, c->width) || (a && (!is_type(a_dtype) || !pitch_ok(lda, c->width))))
        return HPACML_E_INVAL;
    if (c->rows == 0)
        return HPACML_OK;
    Operands o;
    const bool in_place = a == z && a_dtype == z_dtype && lda == ldz;
    o.add(z, c->rows, c->width, ldz, size_of(z_dtype), size_of(z_dtype), in_place);
    if (a && !in_place)
        o.add(a, c->rows, c->width, lda, size_of(a_dtype), size_of(a_dtype), true);
    add_checkpoint(&o, *c, true);
    if (o.check() != HPACML_OK)
        return o.status;
    return status_of(launch_checkpoint_save(*c, z, z_dtype, ldz, a, a_dtype, lda, (hipStream_t)stream));
}

hpacml_status hpacml8_checkpoint_load(const hpacml8_checkpoint *c, void *a, int32_t a_dtype, int64_t lda, void *stream) {
    const hpacml_status s = checkpoint_status(c);
    if (s != HPACML_OK)
        return s;
    if (!is_type(a_dtype) || !pitch_ok(lda, c->width))
        return HPACML_E_INVAL;
    if (c->rows == 0)
        return HPACML_OK;
    Operands o;
    o.add(a, c->rows, c->width, lda, size_of(a_dtype), size_of(a_dtype), true);
    add_checkpoint(&o, *c, false);
    if (o.check() != HPACML_OK)
        return o.status;
    return status_of(launch_checkpoint_load(*c, a, a_dtype, lda, (hipStream_t)stream));
}

hpacml_status hpacml8_backward_scratch(const hpacml8_checkpoint *c, const void *dy, int32_t dtype, int64_t lddy,
                                       int32_t n_out, int32_t want_dw, int32_t want_dx, size_t *bytes) {
    const hpacml_status s = checkpoint_status(c);
    if (s != HPACML_OK)
        return s;
    if (!bytes || !is_type(dtype) || n_out < 1 || !pitch_ok(lddy, n_out))
        return HPACML_E_INVAL;
    if (n_out > HPACML8_MAX_WIDTH)
        return HPACML_E_UNSUPPORTED;
    *bytes = backward8_plan(*c, dy, dtype, lddy, n_out, want_dw != 0, want_dx != 0).bytes;
    return HPACML_OK;
}

hpacml_status hpacml8_backward(const hpacml8_checkpoint *c, const void *dy, int32_t dtype, int64_t lddy, int32_t n_out,
                               const void *W, int64_t ldw, float *dw, int64_t lddw, float *db, void *dx, int64_t lddx,
                               int32_t accumulate, void *scratch, size_t scratch_bytes, void *stream) {
    const hpacml_status s = checkpoint_status(c);
    if (s != HPACML_OK)
        return s;
    if (!is_type(dtype) || n_out < 1 || !pitch_ok(lddy, n_out) || (!dw && !db && !dx) || (dw && !pitch_ok(lddw, c->width)) ||
        (dx && (!W || !pitch_ok(ldw, c->width) || !pitch_ok(lddx, c->width))))
        return HPACML_E_INVAL;
    if (n_out > HPACML8_MAX_WIDTH)
        return HPACML_E_UNSUPPORTED;
    const Backward8Plan plan = backward8_plan(*c, dy, dtype, lddy, n_out, dw || db, dx != nullptr);
    if (scratch_bytes < plan.bytes)
        return HPACML_E_RANGE;
    const int64_t es = size_of(dtype);
    Operands o;
    o.add(dy, c->rows, n_out, lddy, es, es, false);
    add_checkpoint(&o, *c, false);
    if (dw)
        o.add(dw, n_out, c->width, lddw, 4, 4, true);
    if (db)
        o.add(db, 1, n_out, n_out, 4, 4, true);
    if (dx) {
        o.add(W, n_out, c->width, ldw, es, es, false);
        o.add(dx, c->rows, c->width, lddx, es, es, true);
    }
    o.add(scratch, 1, (int64_t)plan.bytes, (int64_t)plan.bytes, 1, 16, true);
    if (o.check() != HPACML_OK)
        return o.status;
    return status_of(launch_backward8({*c, dy, dtype, lddy, n_out, W, ldw, dw, lddw, db, dx, lddx, accumulate, (char *)scratch},
                                      plan, (hipStream_t)stream));
}

}  // extern "C"
