/* The binding's way into the library for the calls that programs make in a loop.
 *
 * A small call is bound by its host side: of 4.9 us (bf16 64 x 64 x 64 through ctypes) the launch takes 2.9, the library 0.4 and
 * converting fifteen arguments the rest; through this it is 3.6.  make(name, address, ...) returns a callable that takes the binding's own arguments in
 * order - tensors or addresses, a workspace tensor or None, a stream or None - and calls the function at `address` without
 * the interpreter lock.  The three functions that find the current stream may be None: such an entry takes calls that name theirs.
 * Whatever is not plain (a subclass of int, a value out of range, an object without data_ptr) it
 * leaves to the caller by returning NotImplemented, so that there is one place that says what an argument may be. */
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stdint.h>

typedef struct {
    void *fn;
    PyObject *initialized, *device, *raw_stream;        /* torch's: is there a device context, which device, its current stream; or None */
} Entry;

static PyObject *data_ptr_name, *nbytes_name, *stream_name;

/* Each returns 0, or -1 where the argument is not plain (with or without an exception set). */
static int get_int(PyObject *o, int64_t lo, int64_t hi, int64_t *out)
{
    int overflow = 0;
    if (!PyLong_CheckExact(o) && !PyBool_Check(o))
        return -1;
    *out = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow || *out < lo || *out > hi ? -1 : 0;
}
static int get_i32(PyObject *o, int *out)
{
    int64_t v;
    if (get_int(o, INT32_MIN, INT32_MAX, &v))
        return -1;
    *out = (int)v;
    return 0;
}
static int get_i64(PyObject *o, int64_t *out) { return get_int(o, INT64_MIN, INT64_MAX, out); }
static int get_truth(PyObject *o, int *out) { return (*out = PyObject_IsTrue(o)) < 0 ? -1 : 0; }
static int get_float(PyObject *o, float *out)
{
    if (PyFloat_CheckExact(o)) {
        *out = (float)PyFloat_AS_DOUBLE(o);
        return 0;
    }
    int64_t v;
    if (get_int(o, -(1 << 24), 1 << 24, &v))
        return -1;
    *out = (float)v;
    return 0;
}
static int get_address(PyObject *o, void **out)
{
    int64_t v;
    if (get_int(o, 0, INT64_MAX, &v))
        return -1;
    *out = (void *)(intptr_t)v;
    return 0;
}
static int get_ptr(PyObject *o, void **out)
{
    if (o == Py_None) {
        *out = NULL;
        return 0;
    }
    if (PyLong_Check(o))
        return get_address(o, out);
    PyObject *p = PyObject_CallMethodNoArgs(o, data_ptr_name);
    if (!p)
        return -1;
    const int rc = get_address(p, out);
    Py_DECREF(p);
    return rc;
}
static int get_workspace(PyObject *o, void **ws, size_t *bytes)
{
    *ws = NULL;
    *bytes = 0;
    if (o == Py_None)
        return 0;
    if (PyLong_Check(o) || get_ptr(o, ws))
        return -1;
    PyObject *n = PyObject_GetAttr(o, nbytes_name);
    int64_t v;
    const int rc = n ? get_int(n, 0, INT64_MAX, &v) : -1;
    Py_XDECREF(n);
    if (rc == 0)
        *bytes = (size_t)v;
    return rc;
}
static int get_stream(const Entry *e, PyObject *o, void **out)
{
    if (o != Py_None) {
        if (PyLong_Check(o))
            return get_address(o, out);
        PyObject *s = PyObject_GetAttr(o, stream_name);
        const int rc = s ? get_address(s, out) : -1;
        Py_XDECREF(s);
        return rc;
    }
    if (e->initialized == Py_None)
        return -1;
    PyObject *yes = PyObject_CallNoArgs(e->initialized);
    const int is = yes ? PyObject_IsTrue(yes) : -1;
    Py_XDECREF(yes);
    if (is != 1)
        return -1;
    PyObject *dev = PyObject_CallNoArgs(e->device);
    PyObject *raw = dev ? PyObject_CallOneArg(e->raw_stream, dev) : NULL;
    const int rc = raw ? get_address(raw, out) : -1;
    Py_XDECREF(raw);
    Py_XDECREF(dev);
    return rc;
}

static PyObject *not_plain(void)
{
    PyErr_Clear();
    Py_RETURN_NOTIMPLEMENTED;
}

#define ENTRY(count)                                                          \
    const Entry *e = (const Entry *)PyCapsule_GetPointer(self, NULL);         \
    if (!e || n != (count))                                                   \
        return not_plain();
#define RETURN_CALL(...)                                                      \
    do {                                                                      \
        int rc_;                                                              \
        Py_BEGIN_ALLOW_THREADS                                                \
        rc_ = __VA_ARGS__;                                                    \
        Py_END_ALLOW_THREADS                                                  \
        return PyLong_FromLong(rc_);                                          \
    } while (0)

/* transA, transB, M, N, K, A, lda, B, ldb, beta, C, ldc, workspace, stream */
static PyObject *call_f32(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int tA, tB;
    int64_t M, N, K, lda, ldb, ldc;
    void *A, *B, *C, *ws, *st;
    size_t nb;
    float beta;
    ENTRY(14)
    if (get_i32(a[0], &tA) || get_i32(a[1], &tB) || get_i64(a[2], &M) || get_i64(a[3], &N) || get_i64(a[4], &K) || get_ptr(a[5], &A) ||
        get_i64(a[6], &lda) || get_ptr(a[7], &B) || get_i64(a[8], &ldb) || get_float(a[9], &beta) || get_ptr(a[10], &C) ||
        get_i64(a[11], &ldc) || get_workspace(a[12], &ws, &nb) || get_stream(e, a[13], &st))
        return not_plain();
    typedef int (*fn)(int, int, int64_t, int64_t, int64_t, const void *, int64_t, const void *, int64_t, float, void *, int64_t, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(tA, tB, M, N, K, A, lda, B, ldb, beta, C, ldc, ws, nb, st));
}

/* the same with c_is_f32 before the workspace */
static PyObject *call_half(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int tA, tB, c32;
    int64_t M, N, K, lda, ldb, ldc;
    void *A, *B, *C, *ws, *st;
    size_t nb;
    float beta;
    ENTRY(15)
    if (get_i32(a[0], &tA) || get_i32(a[1], &tB) || get_i64(a[2], &M) || get_i64(a[3], &N) || get_i64(a[4], &K) || get_ptr(a[5], &A) ||
        get_i64(a[6], &lda) || get_ptr(a[7], &B) || get_i64(a[8], &ldb) || get_float(a[9], &beta) || get_ptr(a[10], &C) ||
        get_i64(a[11], &ldc) || get_truth(a[12], &c32) || get_workspace(a[13], &ws, &nb) || get_stream(e, a[14], &st))
        return not_plain();
    typedef int (*fn)(int, int, int64_t, int64_t, int64_t, const void *, int64_t, const void *, int64_t, float, void *, int64_t, int, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(tA, tB, M, N, K, A, lda, B, ldb, beta, C, ldc, c32, ws, nb, st));
}

/* transA, transB, M, N, K, A, lda, B, ldb, accumulate, C, ldc, stream */
static PyObject *call_s8(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int tA, tB, acc;
    int64_t M, N, K, lda, ldb, ldc;
    void *A, *B, *C, *st;
    ENTRY(13)
    if (get_i32(a[0], &tA) || get_i32(a[1], &tB) || get_i64(a[2], &M) || get_i64(a[3], &N) || get_i64(a[4], &K) || get_ptr(a[5], &A) ||
        get_i64(a[6], &lda) || get_ptr(a[7], &B) || get_i64(a[8], &ldb) || get_truth(a[9], &acc) || get_ptr(a[10], &C) ||
        get_i64(a[11], &ldc) || get_stream(e, a[12], &st))
        return not_plain();
    typedef int (*fn)(int, int, int64_t, int64_t, int64_t, const void *, int64_t, const void *, int64_t, int, void *, int64_t, void *);
    RETURN_CALL(((fn)e->fn)(tA, tB, M, N, K, A, lda, B, ldb, acc, C, ldc, st));
}

/* transA, transB, M, N, K, batch, A, A_off, lda, B, B_off, ldb, beta, C, ldc, workspace, stream */
static PyObject *call_brgemm(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int tA, tB;
    int64_t M, N, K, batch, lda, ldb, ldc;
    void *A, *Ao, *B, *Bo, *C, *ws, *st;
    size_t nb;
    float beta;
    ENTRY(17)
    if (get_i32(a[0], &tA) || get_i32(a[1], &tB) || get_i64(a[2], &M) || get_i64(a[3], &N) || get_i64(a[4], &K) || get_i64(a[5], &batch) ||
        get_ptr(a[6], &A) || get_ptr(a[7], &Ao) || get_i64(a[8], &lda) || get_ptr(a[9], &B) || get_ptr(a[10], &Bo) || get_i64(a[11], &ldb) ||
        get_float(a[12], &beta) || get_ptr(a[13], &C) || get_i64(a[14], &ldc) || get_workspace(a[15], &ws, &nb) || get_stream(e, a[16], &st))
        return not_plain();
    typedef int (*fn)(int, int, int64_t, int64_t, int64_t, int64_t, const void *, const void *, int64_t, const void *, const void *, int64_t, float, void *,
                      int64_t, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(tA, tB, M, N, K, batch, A, Ao, lda, B, Bo, ldb, beta, C, ldc, ws, nb, st));
}

/* in_dtype, transA, transB, M, N, K, batch, A, A_off, lda, B, B_off, ldb, beta, C, ldc, c_is_f32, bias, epilogue, workspace, stream */
static PyObject *call_fused(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int dt, tA, tB, c32, epi;
    int64_t M, N, K, batch, lda, ldb, ldc;
    void *A, *Ao, *B, *Bo, *C, *bias, *ws, *st;
    size_t nb;
    float beta;
    ENTRY(21)
    if (get_i32(a[0], &dt) || get_i32(a[1], &tA) || get_i32(a[2], &tB) || get_i64(a[3], &M) || get_i64(a[4], &N) || get_i64(a[5], &K) ||
        get_i64(a[6], &batch) || get_ptr(a[7], &A) || get_ptr(a[8], &Ao) || get_i64(a[9], &lda) || get_ptr(a[10], &B) || get_ptr(a[11], &Bo) ||
        get_i64(a[12], &ldb) || get_float(a[13], &beta) || get_ptr(a[14], &C) || get_i64(a[15], &ldc) || get_truth(a[16], &c32) ||
        get_ptr(a[17], &bias) || get_i32(a[18], &epi) || get_workspace(a[19], &ws, &nb) || get_stream(e, a[20], &st))
        return not_plain();
    typedef int (*fn)(int, int, int, int64_t, int64_t, int64_t, int64_t, const void *, const void *, int64_t, const void *, const void *, int64_t, float,
                      void *, int64_t, int, const void *, int, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(dt, tA, tB, M, N, K, batch, A, Ao, lda, B, Bo, ldb, beta, C, ldc, c32, bias, epi, ws, nb, st));
}

/* transA, M, N, K, A, lda, packedB, beta, C, ldc, c_is_f32, bias, epilogue, workspace, stream */
static PyObject *call_packed(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int tA, c32, epi;
    int64_t M, N, K, lda, ldc;
    void *A, *B, *C, *bias, *ws, *st;
    size_t nb;
    float beta;
    ENTRY(15)
    if (get_i32(a[0], &tA) || get_i64(a[1], &M) || get_i64(a[2], &N) || get_i64(a[3], &K) || get_ptr(a[4], &A) || get_i64(a[5], &lda) ||
        get_ptr(a[6], &B) || get_float(a[7], &beta) || get_ptr(a[8], &C) || get_i64(a[9], &ldc) || get_truth(a[10], &c32) || get_ptr(a[11], &bias) ||
        get_i32(a[12], &epi) || get_workspace(a[13], &ws, &nb) || get_stream(e, a[14], &st))
        return not_plain();
    typedef int (*fn)(int, int64_t, int64_t, int64_t, const void *, int64_t, const void *, float, void *, int64_t, int, const void *, int, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(tA, M, N, K, A, lda, B, beta, C, ldc, c32, bias, epi, ws, nb, st));
}

/* transA, transB, M, N, K, nmat, A, lda, strideA, B, ldb, strideB, beta, C, ldc, strideC, [c_is_f32,] stream */
static PyObject *batched(PyObject *self, PyObject *const *a, Py_ssize_t n, int half)
{
    int tA, tB, c32 = 0;
    int64_t M, N, K, nmat, lda, sa, ldb, sb, ldc, sc;
    void *A, *B, *C, *st;
    float beta;
    ENTRY(17 + half)
    if (get_i32(a[0], &tA) || get_i32(a[1], &tB) || get_i64(a[2], &M) || get_i64(a[3], &N) || get_i64(a[4], &K) || get_i64(a[5], &nmat) ||
        get_ptr(a[6], &A) || get_i64(a[7], &lda) || get_i64(a[8], &sa) || get_ptr(a[9], &B) || get_i64(a[10], &ldb) || get_i64(a[11], &sb) ||
        get_float(a[12], &beta) || get_ptr(a[13], &C) || get_i64(a[14], &ldc) || get_i64(a[15], &sc) || (half && get_truth(a[16], &c32)) ||
        get_stream(e, a[16 + half], &st))
        return not_plain();
    if (half) {
        typedef int (*fn)(int, int, int64_t, int64_t, int64_t, int64_t, const void *, int64_t, int64_t, const void *, int64_t, int64_t, float, void *, int64_t,
                          int64_t, int, void *);
        RETURN_CALL(((fn)e->fn)(tA, tB, M, N, K, nmat, A, lda, sa, B, ldb, sb, beta, C, ldc, sc, c32, st));
    }
    typedef int (*fn)(int, int, int64_t, int64_t, int64_t, int64_t, const void *, int64_t, int64_t, const void *, int64_t, int64_t, float, void *, int64_t,
                      int64_t, void *);
    RETURN_CALL(((fn)e->fn)(tA, tB, M, N, K, nmat, A, lda, sa, B, ldb, sb, beta, C, ldc, sc, st));
}
static PyObject *call_batched_half(PyObject *self, PyObject *const *a, Py_ssize_t n) { return batched(self, a, n, 1); }
static PyObject *call_batched_f32(PyObject *self, PyObject *const *a, Py_ssize_t n) { return batched(self, a, n, 0); }

/* in_dtype, transB, M, N, K, groups, offsets, A, lda, B, ldb, strideB, beta, C, ldc, c_is_f32, bias, stride_bias, epilogue, workspace, stream */
static PyObject *call_grouped(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int dt, tB, c32, epi;
    int64_t M, N, K, groups, lda, ldb, sb, ldc, sbias;
    void *off, *A, *B, *C, *bias, *ws, *st;
    size_t nb;
    float beta;
    ENTRY(21)
    if (get_i32(a[0], &dt) || get_i32(a[1], &tB) || get_i64(a[2], &M) || get_i64(a[3], &N) || get_i64(a[4], &K) || get_i64(a[5], &groups) ||
        get_ptr(a[6], &off) || get_ptr(a[7], &A) || get_i64(a[8], &lda) || get_ptr(a[9], &B) || get_i64(a[10], &ldb) || get_i64(a[11], &sb) ||
        get_float(a[12], &beta) || get_ptr(a[13], &C) || get_i64(a[14], &ldc) || get_truth(a[15], &c32) || get_ptr(a[16], &bias) ||
        get_i64(a[17], &sbias) || get_i32(a[18], &epi) || get_workspace(a[19], &ws, &nb) || get_stream(e, a[20], &st))
        return not_plain();
    typedef int (*fn)(int, int, int64_t, int64_t, int64_t, int64_t, const void *, const void *, int64_t, const void *, int64_t, int64_t, float, void *,
                      int64_t, int, const void *, int64_t, int, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(dt, tB, M, N, K, groups, off, A, lda, B, ldb, sb, beta, C, ldc, c32, bias, sbias, epi, ws, nb, st));
}

/* in_dtype, M, N, K, groups, offsets, dY, ldy, X, ldx, beta, dW, ldw, strideW, c_is_f32, workspace, stream */
static PyObject *call_wgrad(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int dt, c32;
    int64_t M, N, K, groups, ldy, ldx, ldw, sw;
    void *off, *dY, *X, *dW, *ws, *st;
    size_t nb;
    float beta;
    ENTRY(17)
    if (get_i32(a[0], &dt) || get_i64(a[1], &M) || get_i64(a[2], &N) || get_i64(a[3], &K) || get_i64(a[4], &groups) || get_ptr(a[5], &off) ||
        get_ptr(a[6], &dY) || get_i64(a[7], &ldy) || get_ptr(a[8], &X) || get_i64(a[9], &ldx) || get_float(a[10], &beta) || get_ptr(a[11], &dW) ||
        get_i64(a[12], &ldw) || get_i64(a[13], &sw) || get_truth(a[14], &c32) || get_workspace(a[15], &ws, &nb) || get_stream(e, a[16], &st))
        return not_plain();
    typedef int (*fn)(int, int64_t, int64_t, int64_t, int64_t, const void *, const void *, int64_t, const void *, int64_t, float, void *, int64_t, int64_t,
                      int, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(dt, M, N, K, groups, off, dY, ldy, X, ldx, beta, dW, ldw, sw, c32, ws, nb, st));
}

/* in_dtype, transB, M, N, K, R, segments, offsets, ids, adapters, X, ldx, W, ldw, down, ld_down, stride_down, up, ld_up, stride_up, scale, beta, Y,
 * ldy, c_is_f32, bias, epilogue, H, ldh, workspace, stream */
static PyObject *call_adapters(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int dt, tB, c32, epi;
    int64_t M, N, K, R, segments, adapters, ldx, ldw, ldd, sd, ldu, su, ldy, ldh;
    void *off, *ids, *X, *W, *down, *up, *scale, *Y, *bias, *H, *ws, *st;
    size_t nb;
    float beta;
    ENTRY(31)
    if (get_i32(a[0], &dt) || get_i32(a[1], &tB) || get_i64(a[2], &M) || get_i64(a[3], &N) || get_i64(a[4], &K) || get_i64(a[5], &R) ||
        get_i64(a[6], &segments) || get_ptr(a[7], &off) || get_ptr(a[8], &ids) || get_i64(a[9], &adapters) || get_ptr(a[10], &X) ||
        get_i64(a[11], &ldx) || get_ptr(a[12], &W) || get_i64(a[13], &ldw) || get_ptr(a[14], &down) || get_i64(a[15], &ldd) || get_i64(a[16], &sd) ||
        get_ptr(a[17], &up) || get_i64(a[18], &ldu) || get_i64(a[19], &su) || get_ptr(a[20], &scale) || get_float(a[21], &beta) ||
        get_ptr(a[22], &Y) || get_i64(a[23], &ldy) || get_truth(a[24], &c32) || get_ptr(a[25], &bias) || get_i32(a[26], &epi) ||
        get_ptr(a[27], &H) || get_i64(a[28], &ldh) || get_workspace(a[29], &ws, &nb) || get_stream(e, a[30], &st))
        return not_plain();
    typedef int (*fn)(int, int, int64_t, int64_t, int64_t, int64_t, int64_t, const void *, const void *, int64_t, const void *, int64_t, const void *, int64_t,
                      const void *, int64_t, int64_t, const void *, int64_t, int64_t, const void *, float, void *, int64_t, int, const void *, int, void *,
                      int64_t, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(dt, tB, M, N, K, R, segments, off, ids, adapters, X, ldx, W, ldw, down, ldd, sd, up, ldu, su, scale, beta, Y, ldy, c32, bias, epi,
                            H, ldh, ws, nb, st));
}

/* in_dtype, trans, rows, K, X, ldx, x_rows, source, image, image_bytes or None, stream */
static PyObject *call_pack_mx4(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int dt, trans;
    int64_t rows, K, ldx, x_rows, bytes;
    void *X, *source, *image, *st;
    size_t nb;
    ENTRY(11)
    if (get_i32(a[0], &dt) || get_i32(a[1], &trans) || get_i64(a[2], &rows) || get_i64(a[3], &K) || get_ptr(a[4], &X) || get_i64(a[5], &ldx) ||
        get_i64(a[6], &x_rows) || get_ptr(a[7], &source) || get_stream(e, a[10], &st))
        return not_plain();
    if (a[9] == Py_None ? get_workspace(a[8], &image, &nb) : get_ptr(a[8], &image) || get_int(a[9], 0, INT64_MAX, &bytes))
        return not_plain();
    if (a[9] != Py_None)
        nb = (size_t)bytes;
    typedef int (*fn)(int, int, int64_t, int64_t, const void *, int64_t, int64_t, const void *, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(dt, trans, rows, K, X, ldx, x_rows, source, image, nb, st));
}

/* out_dtype, rows, K, image, out, ldo, stream */
static PyObject *call_unpack_mx4(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int dt;
    int64_t rows, K, ldo;
    void *image, *out, *st;
    ENTRY(7)
    if (get_i32(a[0], &dt) || get_i64(a[1], &rows) || get_i64(a[2], &K) || get_ptr(a[3], &image) || get_ptr(a[4], &out) ||
        get_i64(a[5], &ldo) || get_stream(e, a[6], &st))
        return not_plain();
    typedef int (*fn)(int, int64_t, int64_t, const void *, void *, int64_t, void *);
    RETURN_CALL(((fn)e->fn)(dt, rows, K, image, out, ldo, st));
}

/* a_dtype, M, N, K, A, lda, W, beta, C, ldc, c_is_f32, bias, epilogue, workspace, stream */
static PyObject *call_mx4(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int dt, c32, epi;
    int64_t M, N, K, lda, ldc;
    void *A, *W, *C, *bias, *ws, *st;
    size_t nb;
    float beta;
    ENTRY(15)
    if (get_i32(a[0], &dt) || get_i64(a[1], &M) || get_i64(a[2], &N) || get_i64(a[3], &K) || get_ptr(a[4], &A) || get_i64(a[5], &lda) ||
        get_ptr(a[6], &W) || get_float(a[7], &beta) || get_ptr(a[8], &C) || get_i64(a[9], &ldc) || get_truth(a[10], &c32) ||
        get_ptr(a[11], &bias) || get_i32(a[12], &epi) || get_workspace(a[13], &ws, &nb) || get_stream(e, a[14], &st))
        return not_plain();
    typedef int (*fn)(int, int64_t, int64_t, int64_t, const void *, int64_t, const void *, float, void *, int64_t, int, const void *, int, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(dt, M, N, K, A, lda, W, beta, C, ldc, c32, bias, epi, ws, nb, st));
}

/* a_dtype, M, N, K, groups, offsets, A, lda, W, strideW, beta, C, ldc, c_is_f32, bias, stride_bias, epilogue, workspace, stream */
static PyObject *call_grouped_mx4(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int dt, c32, epi;
    int64_t M, N, K, groups, lda, sw, ldc, sb;
    void *off, *A, *W, *C, *bias, *ws, *st;
    size_t nb;
    float beta;
    ENTRY(19)
    if (get_i32(a[0], &dt) || get_i64(a[1], &M) || get_i64(a[2], &N) || get_i64(a[3], &K) || get_i64(a[4], &groups) || get_ptr(a[5], &off) ||
        get_ptr(a[6], &A) || get_i64(a[7], &lda) || get_ptr(a[8], &W) || get_i64(a[9], &sw) || get_float(a[10], &beta) || get_ptr(a[11], &C) ||
        get_i64(a[12], &ldc) || get_truth(a[13], &c32) || get_ptr(a[14], &bias) || get_i64(a[15], &sb) || get_i32(a[16], &epi) ||
        get_workspace(a[17], &ws, &nb) || get_stream(e, a[18], &st))
        return not_plain();
    typedef int (*fn)(int, int64_t, int64_t, int64_t, int64_t, const void *, const void *, int64_t, const void *, int64_t, float, void *, int64_t, int,
                      const void *, int64_t, int, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(dt, M, N, K, groups, off, A, lda, W, sw, beta, C, ldc, c32, bias, sb, epi, ws, nb, st));
}

/* in_dtype, M, E, topk, logits, ld, valid, level, ids, gates, offsets, rows, place, balance, workspace, stream */
static PyObject *call_route(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int dt, level;
    int64_t M, E, top, ld;
    void *x, *valid, *ids, *gates, *off, *rows, *place, *balance, *ws, *st;
    size_t nb;
    ENTRY(16)
    if (get_i32(a[0], &dt) || get_i64(a[1], &M) || get_i64(a[2], &E) || get_i64(a[3], &top) || get_ptr(a[4], &x) || get_i64(a[5], &ld) ||
        get_ptr(a[6], &valid) || get_truth(a[7], &level) || get_ptr(a[8], &ids) || get_ptr(a[9], &gates) || get_ptr(a[10], &off) ||
        get_ptr(a[11], &rows) || get_ptr(a[12], &place) || get_ptr(a[13], &balance) || get_workspace(a[14], &ws, &nb) || get_stream(e, a[15], &st))
        return not_plain();
    typedef int (*fn)(int, int64_t, int64_t, int64_t, const void *, int64_t, const void *, int, void *, void *, void *, void *, void *, void *, void *, size_t, void *);
    RETURN_CALL(((fn)e->fn)(dt, M, E, top, x, ld, valid, level, ids, gates, off, rows, place, balance, ws, nb, st));
}

/* in_dtype, M, E, topk, logits, ld, level, ids, offsets, balance, dgates, dloss, dlogits, ldd, stream */
static PyObject *call_route_grad(PyObject *self, PyObject *const *a, Py_ssize_t n)
{
    int dt, level;
    int64_t M, E, top, ld, ldd;
    void *x, *ids, *off, *balance, *dgates, *dloss, *dx, *st;
    ENTRY(15)
    if (get_i32(a[0], &dt) || get_i64(a[1], &M) || get_i64(a[2], &E) || get_i64(a[3], &top) || get_ptr(a[4], &x) || get_i64(a[5], &ld) ||
        get_truth(a[6], &level) || get_ptr(a[7], &ids) || get_ptr(a[8], &off) || get_ptr(a[9], &balance) || get_ptr(a[10], &dgates) ||
        get_ptr(a[11], &dloss) || get_ptr(a[12], &dx) || get_i64(a[13], &ldd) || get_stream(e, a[14], &st))
        return not_plain();
    typedef int (*fn)(int, int64_t, int64_t, int64_t, const void *, int64_t, int, const void *, const void *, const void *, const void *, const void *, void *,
                      int64_t, void *);
    RETURN_CALL(((fn)e->fn)(dt, M, E, top, x, ld, level, ids, off, balance, dgates, dloss, dx, ldd, st));
}

#define DEF(name, fn) {name, (PyCFunction)(void (*)(void))fn, METH_FASTCALL, NULL}
static PyMethodDef entries[] = {
    DEF("gemm_f32", call_f32), DEF("gemm_bf16", call_half), DEF("gemm_f16", call_half), DEF("gemm_f8", call_half), DEF("gemm_bf8", call_half),
    DEF("gemm_s8", call_s8), DEF("brgemm_bf16", call_brgemm), DEF("brgemm_fused", call_fused), DEF("gemm_bf16_packed", call_packed),
    DEF("gemm_bf16_batched", call_batched_half), DEF("gemm_f32_batched", call_batched_f32),
    DEF("gemm_grouped", call_grouped), DEF("gemm_grouped_wgrad", call_wgrad), DEF("gemm_adapters", call_adapters),
    DEF("gemm_pack_mx4", call_pack_mx4), DEF("gemm_unpack_mx4", call_unpack_mx4), DEF("gemm_mx4", call_mx4),
    DEF("gemm_grouped_mx4", call_grouped_mx4), DEF("gemm_route", call_route), DEF("gemm_route_grad", call_route_grad)};

static PyObject *make(PyObject *self, PyObject *args)
{
    const char *name;
    unsigned long long address;
    PyObject *initialized, *device, *raw_stream;
    (void)self;
    if (!PyArg_ParseTuple(args, "sKOOO", &name, &address, &initialized, &device, &raw_stream))
        return NULL;
    for (size_t i = 0; i < sizeof entries / sizeof *entries; ++i) {
        if (strcmp(entries[i].ml_name, name))
            continue;
        Entry *e = (Entry *)PyMem_Malloc(sizeof *e);        /* as long as the process, like the library */
        if (!e)
            return PyErr_NoMemory();
        *e = (Entry){(void *)(uintptr_t)address, initialized, device, raw_stream};
        Py_INCREF(initialized);
        Py_INCREF(device);
        Py_INCREF(raw_stream);
        PyObject *capsule = PyCapsule_New(e, NULL, NULL);
        PyObject *f = capsule ? PyCFunction_New(&entries[i], capsule) : NULL;
        Py_XDECREF(capsule);
        return f;
    }
    return PyErr_Format(PyExc_KeyError, "%s", name);
}

static PyMethodDef methods[] = {{"make", make, METH_VARARGS, NULL}, {NULL, NULL, 0, NULL}};
static struct PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fastcall", NULL, -1, methods, NULL, NULL, NULL, NULL};

PyMODINIT_FUNC PyInit__fastcall(void)
{
    data_ptr_name = PyUnicode_InternFromString("data_ptr");
    nbytes_name = PyUnicode_InternFromString("nbytes");
    stream_name = PyUnicode_InternFromString("cuda_stream");
    return data_ptr_name && nbytes_name && stream_name ? PyModule_Create(&module) : NULL;
}
