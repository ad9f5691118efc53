// kt_fast.cpp -- argument marshalling of the training operators (the functions of binding.py with the same names):
// torch tensors in, one call of the C entry out.  A Python module of its own because their calls are short:
// checking and converting the arguments in Python takes as long as the kernels of a small batch.  No
// arithmetic, no state: the C entries' addresses are handed over by binding.py, which loads the module when the first
// operator is called.  KT_BELONGS (build.py) names the torch and Python whose binary interfaces it is built for.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/kaitian.h"

namespace {

// the C entries, in the order of ENTRIES below
decltype(&kt_ckpt_store) c_ckpt_store;
decltype(&kt_ckpt_restore) c_ckpt_restore;
decltype(&kt_norm_forward) c_norm_forward;
decltype(&kt_norm_backward) c_norm_backward;
decltype(&kt_act_forward) c_act_forward;
decltype(&kt_act_backward) c_act_backward;
decltype(&kt_attn_forward) c_attn_forward;
decltype(&kt_attn_backward) c_attn_backward;
decltype(&kt_embed_forward) c_embed_forward;
decltype(&kt_embed_backward) c_embed_backward;
decltype(&kt_xent_forward) c_xent_forward;
decltype(&kt_xent_backward) c_xent_backward;
decltype(&kt_orth_update) c_orth_update;
decltype(&kt_last_error) c_last_error;
PyObject *error_class;

struct Refused {};                              // a Python error is set

[[noreturn]] void refuse(int status, const char *fmt, ...) {
    char text[400];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(text, sizeof(text), fmt, ap);
    va_end(ap);
    PyObject *e = PyObject_CallFunction(error_class, "is", status, text);
    if (e != nullptr) {
        PyErr_SetObject(error_class, e);
        Py_DECREF(e);
    }
    throw Refused();
}

PyObject *done(int status) {
    if (status != KT_OK) refuse(status, "%s", c_last_error(nullptr));
    Py_RETURN_NONE;
}

int type_of(const at::Tensor &t) {              // kt_dtype, or -1
    return t.scalar_type() == at::kFloat ? KT_F32 : t.scalar_type() == at::kBFloat16 ? KT_BF16 : -1;
}

// The arguments of one call: what all its tensors have in common is seen to here.
struct Call {
    int device = -2;
    const at::Tensor *tensor(PyObject *o, const char *what, bool optional = false) {
        if (optional && o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) refuse(KT_ERR_INVALID, "%s: a tensor expected", what);
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda() && !t.is_cpu()) refuse(KT_ERR_INVALID, "%s: a tensor in device memory expected", what);
        const int on = t.is_cuda() ? t.device().index() : -1;
        if (device == -2) {
            // (without a device nothing can be started; arguments can still be refused)
            static const bool devices = c10::cuda::device_count() > 0;
            if (on < 0 && devices) refuse(KT_ERR_INVALID, "%s: a tensor in device memory expected", what);
            if (on >= 0 && on != c10::cuda::current_device()) refuse(KT_ERR_INVALID, "%s is on device %d, which is not the current one", what, on);
            device = on;
        }
        if (on != device) refuse(KT_ERR_INVALID, "%s is on another device than the tensors before it", what);
        return &t;
    }
};

void *stream_of(PyObject *o) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream().stream();
    PyObject *handle = PyLong_Check(o) ? (Py_INCREF(o), o) : PyObject_GetAttrString(o, "cuda_stream");
    if (handle == nullptr) throw Refused();
    void *s = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    if (PyErr_Occurred()) throw Refused();
    return s;
}

void *address(const at::Tensor *t) { return t == nullptr ? nullptr : t->data_ptr(); }

// (A workspace of any type and shape; an expanded or strided one would count bytes that are not its own.)
int64_t workspace_bytes(const at::Tensor *t) {
    if (t == nullptr) return 0;
    if (!t->is_contiguous()) refuse(KT_ERR_SHAPE, "workspace: a contiguous tensor expected");
    return static_cast<int64_t>(t->nbytes());
}

// ------------------------------------------------------------------------------- row operators
struct Matrix {
    void *at = nullptr;
    int64_t stride = 0, rows = 0, cols = 0;
    int type = KT_F32;
};
Matrix matrix(const at::Tensor *t, const char *what, const Matrix *like = nullptr) {
    Matrix m;
    if (t == nullptr) return m;
    if (t->dim() != 2 || (m.type = type_of(*t)) < 0 || (t->size(1) > 1 && t->stride(1) != 1))
        refuse(KT_ERR_SHAPE, "%s: a float32 or bfloat16 matrix with contiguous columns expected", what);
    m.at = t->data_ptr(), m.stride = t->stride(0), m.rows = t->size(0), m.cols = t->size(1);
    if (like != nullptr && (m.rows != like->rows || m.cols != like->cols || m.type != like->type)) refuse(KT_ERR_SHAPE, "%s: shape or dtype differs", what);
    return m;
}

bool is_shape(const at::Tensor &t, at::ScalarType type, int64_t rows, int64_t cols) {
    return t.scalar_type() == type && t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && t.is_contiguous();
}

void check_codes(const at::Tensor *codes, const at::Tensor *scales, int64_t rows, int64_t cols) {
    if (codes == nullptr && scales == nullptr) return;
    if (codes == nullptr || scales == nullptr) refuse(KT_ERR_INVALID, "a checkpoint has codes and scales: one of them is missing");
    if (!is_shape(*codes, at::kChar, rows, (cols + 15) / 16 * 16) || !is_shape(*scales, at::kFloat, rows, (cols + KT_CKPT_BLOCK - 1) / KT_CKPT_BLOCK))
        refuse(KT_ERR_SHAPE, "codes: int8 [rows, kt_ckpt_pitch(cols)], scales: float32 [rows, kt_ckpt_blocks(cols)], contiguous");
}

// Vectors over the columns, all of one type: that type (KT_F32 where there is none).
int check_params(int64_t cols, std::initializer_list<const at::Tensor *> all) {
    int type = -1;
    for (const at::Tensor *t : all) {
        if (t == nullptr) continue;
        if (type < 0) type = type_of(*t);
        if (type < 0 || type_of(*t) != type || t->dim() != 1 || t->size(0) != cols || !t->is_contiguous())
            refuse(KT_ERR_SHAPE, "weight, bias and their gradients: contiguous, [cols], all float32 or all bfloat16");
    }
    return type < 0 ? KT_F32 : type;
}

float *per_row(const at::Tensor *t, int64_t rows, const char *what) {
    if (t == nullptr) return nullptr;
    if (t->scalar_type() != at::kFloat || t->dim() != 1 || t->size(0) != rows || !t->is_contiguous()) refuse(KT_ERR_SHAPE, "%s: contiguous float32 [rows] expected", what);
    return static_cast<float *>(t->data_ptr());
}

PyObject *ckpt_store(PyObject *const *a) {      // x, codes, scales, stream
    Call c;
    const Matrix x = matrix(c.tensor(a[0], "x"), "x");
    const at::Tensor *codes = c.tensor(a[1], "codes", true), *scales = c.tensor(a[2], "scales", true);
    check_codes(codes, scales, x.rows, x.cols);
    return done(c_ckpt_store(x.at, x.stride, static_cast<int8_t *>(address(codes)), static_cast<float *>(address(scales)), x.rows, x.cols, x.type, stream_of(a[3])));
}

PyObject *ckpt_restore(PyObject *const *a) {    // codes, scales, out, weight, bias, stream
    Call c;
    const Matrix out = matrix(c.tensor(a[2], "out"), "out");
    const at::Tensor *codes = c.tensor(a[0], "codes", true), *scales = c.tensor(a[1], "scales", true), *weight = c.tensor(a[3], "weight", true), *bias = c.tensor(a[4], "bias", true);
    check_codes(codes, scales, out.rows, out.cols);
    const int type = check_params(out.cols, {weight, bias});
    return done(c_ckpt_restore(static_cast<int8_t *>(address(codes)), static_cast<float *>(address(scales)), address(weight), address(bias), type, out.at, out.stride, out.rows, out.cols, out.type,
                               stream_of(a[5])));
}

PyObject *norm_forward(PyObject *const *a) {    // x, weight, bias, out, mean, rstd, eps, codes, scales, stream
    Call c;
    const Matrix x = matrix(c.tensor(a[0], "x"), "x"), out = matrix(c.tensor(a[3], "out"), "out", &x);
    const at::Tensor *weight = c.tensor(a[1], "weight", true), *bias = c.tensor(a[2], "bias", true), *mean = c.tensor(a[4], "mean", true), *rstd = c.tensor(a[5], "rstd", true),
                     *codes = c.tensor(a[7], "codes", true), *scales = c.tensor(a[8], "scales", true);
    const double eps = PyFloat_AsDouble(a[6]);
    if (eps == -1.0 && PyErr_Occurred()) throw Refused();
    const int type = check_params(x.cols, {weight, bias});
    float *const m = per_row(mean, x.rows, "mean"), *const r = per_row(rstd, x.rows, "rstd");
    check_codes(codes, scales, x.rows, x.cols);
    return done(c_norm_forward(x.at, x.stride, address(weight), address(bias), type, out.at, out.stride, m, r, static_cast<int8_t *>(address(codes)), static_cast<float *>(address(scales)), x.rows,
                               x.cols, x.type, static_cast<float>(eps), stream_of(a[9])));
}

PyObject *norm_backward(PyObject *const *a) {   // dout, weight, rstd, dx, dweight, dbias, workspace, x, mean, codes, scales, stream
    Call c;
    const Matrix dout = matrix(c.tensor(a[0], "dout"), "dout"), dx = matrix(c.tensor(a[3], "dx"), "dx", &dout), x = matrix(c.tensor(a[7], "x", true), "x", &dout);
    const at::Tensor *weight = c.tensor(a[1], "weight", true), *rstd = c.tensor(a[2], "rstd", true), *dweight = c.tensor(a[4], "dweight", true), *dbias = c.tensor(a[5], "dbias", true),
                     *workspace = c.tensor(a[6], "workspace", true), *mean = c.tensor(a[8], "mean", true), *codes = c.tensor(a[9], "codes", true), *scales = c.tensor(a[10], "scales", true);
    const int type = check_params(dout.cols, {weight, dweight, dbias});
    check_codes(codes, scales, dout.rows, dout.cols);
    const float *const m = per_row(mean, dout.rows, "mean"), *const r = per_row(rstd, dout.rows, "rstd");
    return done(c_norm_backward(dout.at, dout.stride, x.at, x.stride, m, static_cast<int8_t *>(address(codes)), static_cast<float *>(address(scales)), r, address(weight), type, dx.at, dx.stride,
                                address(dweight), address(dbias), address(workspace), workspace_bytes(workspace), dout.rows, dout.cols, dout.type,
                                stream_of(a[11])));
}

int kind_of(PyObject *o) {
    const long kind = PyLong_AsLong(o);
    if (kind == -1 && PyErr_Occurred()) throw Refused();
    return static_cast<int>(kind);
}

PyObject *act_forward(PyObject *const *a) {     // x, out, codes, scales, kind, stream
    Call c;
    const Matrix x = matrix(c.tensor(a[0], "x"), "x"), out = matrix(c.tensor(a[1], "out"), "out", &x);
    const at::Tensor *codes = c.tensor(a[2], "codes", true), *scales = c.tensor(a[3], "scales", true);
    check_codes(codes, scales, x.rows, x.cols);
    return done(c_act_forward(x.at, x.stride, out.at, out.stride, static_cast<int8_t *>(address(codes)), static_cast<float *>(address(scales)), x.rows, x.cols, x.type, kind_of(a[4]), stream_of(a[5])));
}

PyObject *act_backward(PyObject *const *a) {    // dout, codes, scales, dx, kind, x, stream
    Call c;
    const Matrix dout = matrix(c.tensor(a[0], "dout"), "dout"), dx = matrix(c.tensor(a[3], "dx"), "dx", &dout), x = matrix(c.tensor(a[5], "x", true), "x", &dout);
    const at::Tensor *codes = c.tensor(a[1], "codes", true), *scales = c.tensor(a[2], "scales", true);
    check_codes(codes, scales, dout.rows, dout.cols);
    return done(c_act_backward(dout.at, dout.stride, x.at, x.stride, static_cast<int8_t *>(address(codes)), static_cast<float *>(address(scales)), dx.at, dx.stride, dout.rows, dout.cols, dout.type,
                               kind_of(a[4]), stream_of(a[6])));
}

// ----------------------------------------------------------------------------------- attention
struct Heads {
    void *at;
    int64_t stride[3];                          // batch, token, head
};
Heads heads(const at::Tensor *t, const char *what, const at::Tensor *like) {
    if (t->scalar_type() != at::kBFloat16 || t->sizes() != like->sizes() || (t->size(3) > 1 && t->stride(3) != 1))
        refuse(KT_ERR_SHAPE, "%s: bfloat16 [%lld, %lld, %lld, %lld] with a contiguous last dimension expected", what, (long long)like->size(0), (long long)like->size(1), (long long)like->size(2),
               (long long)like->size(3));
    return {t->data_ptr(), {t->stride(0), t->stride(1), t->stride(2)}};
}

// kt_attn from the shapes of q and k, with lse seen to.
kt_attn describe(Call &c, const at::Tensor *q, const at::Tensor *k, const at::Tensor *lse, PyObject *scale, PyObject *causal, PyObject *used_q, PyObject *used_kv) {
    if (q->dim() != 4 || k->dim() != 4 || q->size(0) != k->size(0) || q->size(3) != k->size(3))
        refuse(KT_ERR_SHAPE, "q and k: [batch, tokens, heads, head_dim] with the same batch and head_dim expected");
    for (const at::Tensor *t : {q, k})
        for (int64_t n : t->sizes())
            if (n > INT32_MAX) refuse(KT_ERR_SHAPE, "a dimension of %lld", (long long)n);
    kt_attn d{};
    d.batch = static_cast<int32_t>(q->size(0)), d.len_q = static_cast<int32_t>(q->size(1)), d.heads = static_cast<int32_t>(q->size(2)), d.head_dim = static_cast<int32_t>(q->size(3));
    d.len_kv = static_cast<int32_t>(k->size(1)), d.heads_kv = static_cast<int32_t>(k->size(2)), d.dtype = KT_BF16;
    PyObject *const used[2] = {used_q, used_kv};
    const int32_t **const to[2] = {&d.used_q, &d.used_kv};
    for (int i = 0; i < 2; ++i) {
        const at::Tensor *u = c.tensor(used[i], i == 0 ? "used_q" : "used_kv", true);
        if (u == nullptr) continue;
        if (u->scalar_type() != at::kInt || u->dim() != 1 || u->size(0) != d.batch || !u->is_contiguous()) refuse(KT_ERR_SHAPE, "used_q, used_kv: contiguous int32 [batch] expected");
        *to[i] = static_cast<const int32_t *>(u->data_ptr());
    }
    if (lse->scalar_type() != at::kFloat || lse->dim() != 3 || lse->size(0) != d.batch || lse->size(1) != d.heads || lse->size(2) != d.len_q || !lse->is_contiguous())
        refuse(KT_ERR_SHAPE, "lse: contiguous float32 [batch, heads, tokens] expected");
    if (scale == Py_None) {
        d.scale = d.head_dim > 0 ? 1.0f / std::sqrt(static_cast<float>(d.head_dim)) : 1.0f;
    } else {
        const double s = PyFloat_AsDouble(scale);
        if (s == -1.0 && PyErr_Occurred()) throw Refused();
        d.scale = static_cast<float>(s);
    }
    const int yes = PyObject_IsTrue(causal);
    if (yes < 0) throw Refused();
    d.causal = yes;
    return d;
}

PyObject *attn_forward(PyObject *const *a) {    // q, k, v, out, lse, scale, causal, used_q, used_kv, stream
    Call c;
    const at::Tensor *q = c.tensor(a[0], "q"), *k = c.tensor(a[1], "k"), *v = c.tensor(a[2], "v"), *out = c.tensor(a[3], "out"), *lse = c.tensor(a[4], "lse");
    const kt_attn d = describe(c, q, k, lse, a[5], a[6], a[7], a[8]);
    const Heads hq = heads(q, "q", q), hk = heads(k, "k", k), hv = heads(v, "v", k), ho = heads(out, "out", q);
    return done(c_attn_forward(&d, hq.at, hq.stride, hk.at, hk.stride, hv.at, hv.stride, ho.at, ho.stride, static_cast<float *>(lse->data_ptr()), stream_of(a[9])));
}

PyObject *attn_backward(PyObject *const *a) {   // dout, q, k, v, out, lse, dq, dk, dv, workspace, scale, causal, used_q, used_kv, stream
    Call c;
    const at::Tensor *dout = c.tensor(a[0], "dout"), *q = c.tensor(a[1], "q"), *k = c.tensor(a[2], "k"), *v = c.tensor(a[3], "v"), *out = c.tensor(a[4], "out"), *lse = c.tensor(a[5], "lse"),
                     *dq = c.tensor(a[6], "dq"), *dk = c.tensor(a[7], "dk"), *dv = c.tensor(a[8], "dv"), *workspace = c.tensor(a[9], "workspace");
    const kt_attn d = describe(c, q, k, lse, a[10], a[11], a[12], a[13]);
    const Heads hg = heads(dout, "dout", q), hq = heads(q, "q", q), hk = heads(k, "k", k), hv = heads(v, "v", k), ho = heads(out, "out", q), hdq = heads(dq, "dq", q), hdk = heads(dk, "dk", k),
                hdv = heads(dv, "dv", k);
    return done(c_attn_backward(&d, hg.at, hg.stride, hq.at, hq.stride, hk.at, hk.stride, hv.at, hv.stride, ho.at, ho.stride, static_cast<float *>(lse->data_ptr()), hdq.at, hdq.stride, hdk.at,
                                hdk.stride, hdv.at, hdv.stride, workspace->data_ptr(), workspace_bytes(workspace), stream_of(a[14])));
}

// ------------------------------------------------------------- embedding, loss and matrix updates
const int64_t *indices(const at::Tensor *t, const char *what, int64_t rows) {
    if (t->scalar_type() != at::kLong || t->dim() != 1 || (rows >= 0 && t->size(0) != rows) || !t->is_contiguous()) refuse(KT_ERR_SHAPE, "%s: contiguous int64, one to a row, expected", what);
    return static_cast<const int64_t *>(t->data_ptr());
}
float number(PyObject *o) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Refused();
    return static_cast<float>(x);
}
void check_cols(const Matrix &m, const char *what, int64_t cols) {
    if (m.cols != cols) refuse(KT_ERR_SHAPE, "%s: %lld columns expected", what, (long long)cols);
}

PyObject *embed_forward(PyObject *const *a) {   // ids, weight, out, scale, stream
    Call c;
    const at::Tensor *ids = c.tensor(a[0], "ids");
    const Matrix weight = matrix(c.tensor(a[1], "weight"), "weight"), out = matrix(c.tensor(a[2], "out"), "out");
    check_cols(weight, "weight", out.cols);
    return done(c_embed_forward(indices(ids, "ids", out.rows), weight.at, weight.stride, weight.type, out.at, out.stride, out.rows, out.cols, weight.rows, out.type, number(a[3]), stream_of(a[4])));
}

PyObject *embed_backward(PyObject *const *a) {  // dout, ids, dweight, workspace, scale, base, stream
    Call c;
    const Matrix dout = matrix(c.tensor(a[0], "dout"), "dout");
    const at::Tensor *ids = c.tensor(a[1], "ids"), *workspace = c.tensor(a[3], "workspace", true);
    const Matrix dweight = matrix(c.tensor(a[2], "dweight"), "dweight"), base = matrix(c.tensor(a[5], "base", true), "base", &dweight);
    check_cols(dweight, "dweight", dout.cols);
    return done(c_embed_backward(dout.at, dout.stride, indices(ids, "ids", dout.rows), base.at, base.stride, dweight.at, dweight.stride, dweight.type, address(workspace), workspace_bytes(workspace), dout.rows,
                                 dout.cols, dweight.rows, dout.type, number(a[4]), stream_of(a[6])));
}

PyObject *xent_forward(PyObject *const *a) {    // hidden, weight, targets, loss, lse, workspace, scale, stream
    Call c;
    const Matrix hidden = matrix(c.tensor(a[0], "hidden"), "hidden"), weight = matrix(c.tensor(a[1], "weight"), "weight");
    const at::Tensor *targets = c.tensor(a[2], "targets"), *loss = c.tensor(a[3], "loss"), *lse = c.tensor(a[4], "lse"), *workspace = c.tensor(a[5], "workspace", true);
    check_cols(weight, "weight", hidden.cols);
    if (hidden.type != weight.type) refuse(KT_ERR_SHAPE, "hidden and weight: one dtype expected");
    const int64_t *const t = indices(targets, "targets", hidden.rows);
    float *const to_loss = per_row(loss, hidden.rows, "loss"), *const to_lse = per_row(lse, hidden.rows, "lse");
    return done(c_xent_forward(hidden.at, hidden.stride, weight.at, weight.stride, t, to_loss, to_lse, address(workspace), workspace_bytes(workspace), hidden.rows, hidden.cols, weight.rows, hidden.type,
                               number(a[6]), stream_of(a[7])));
}

PyObject *xent_backward(PyObject *const *a) {   // dloss, hidden, weight, targets, lse, dhidden, dweight, workspace, scale, dlse, stream
    Call c;
    const at::Tensor *dloss = c.tensor(a[0], "dloss");
    const Matrix hidden = matrix(c.tensor(a[1], "hidden"), "hidden"), weight = matrix(c.tensor(a[2], "weight"), "weight");
    const at::Tensor *targets = c.tensor(a[3], "targets"), *lse = c.tensor(a[4], "lse"), *workspace = c.tensor(a[7], "workspace", true), *dlse = c.tensor(a[9], "dlse", true);
    const Matrix dhidden = matrix(c.tensor(a[5], "dhidden", true), "dhidden", &hidden), dweight = matrix(c.tensor(a[6], "dweight", true), "dweight", &weight);
    check_cols(weight, "weight", hidden.cols);
    if (hidden.type != weight.type) refuse(KT_ERR_SHAPE, "hidden and weight: one dtype expected");
    const int64_t *const t = indices(targets, "targets", hidden.rows);
    const float *const g = per_row(dloss, hidden.rows, "dloss"), *const z = per_row(dlse, hidden.rows, "dlse"), *const l = per_row(lse, hidden.rows, "lse");
    return done(c_xent_backward(g, z, hidden.at, hidden.stride, weight.at, weight.stride, t, l, dhidden.at, dhidden.stride, dweight.at, dweight.stride, address(workspace), workspace_bytes(workspace),
                                hidden.rows, hidden.cols, weight.rows, hidden.type, number(a[8]), stream_of(a[10])));
}

// Matrices of two or three dimensions.
struct Matrices {
    void *at;
    int64_t stride[2], size[3];
    int type;
};
Matrices matrices(const at::Tensor *t, const char *what) {
    const int64_t d = t->dim();
    Matrices m{};
    if ((d != 2 && d != 3) || (m.type = type_of(*t)) < 0 || (t->size(d - 1) > 1 && t->stride(d - 1) != 1))
        refuse(KT_ERR_SHAPE, "%s: float32 or bfloat16 [rows, cols] or [batch, rows, cols] with contiguous columns expected", what);
    m.at = t->data_ptr();
    m.size[0] = d == 3 ? t->size(0) : 1, m.size[1] = t->size(d - 2), m.size[2] = t->size(d - 1);
    m.stride[0] = d == 3 ? t->stride(0) : 0, m.stride[1] = t->stride(d - 2);
    return m;
}

PyObject *orth_update(PyObject *const *a) {     // x, out, workspace, steps, a, b, c, scale, stream
    Call c;
    const at::Tensor *tx = c.tensor(a[0], "x"), *tout = c.tensor(a[1], "out"), *workspace = c.tensor(a[2], "workspace", true);
    const Matrices x = matrices(tx, "x"), out = matrices(tout, "out");
    if (tx->sizes() != tout->sizes() || out.type != KT_BF16) refuse(KT_ERR_SHAPE, "out: bfloat16 of x's shape expected");
    const long steps = PyLong_AsLong(a[3]);
    if (steps == -1 && PyErr_Occurred()) throw Refused();
    const float coefficients[3] = {number(a[4]), number(a[5]), number(a[6])};
    return done(c_orth_update(x.at, x.stride, x.type, out.at, out.stride, address(workspace), workspace_bytes(workspace), x.size[0], x.size[1], x.size[2],
                              static_cast<int>(steps < -1 ? -1 : steps > 1000 ? 1000 : steps), coefficients, number(a[7]), stream_of(a[8])));
}

// ---------------------------------------------------------------------------------- the module
// No C++ exception leaves a call: torch's own become Python errors too.
template <PyObject *(*FN)(PyObject *const *), int N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != N) return PyErr_Format(PyExc_TypeError, "%d arguments expected, %zd given", N, n);
    try {
        return FN(args);
    } catch (const Refused &) {
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
        return nullptr;
    }
}

PyObject *bind(PyObject *, PyObject *const *args, Py_ssize_t n) {         // the error class, then the addresses of the C entries
    void **const to[] = {reinterpret_cast<void **>(&c_ckpt_store), reinterpret_cast<void **>(&c_ckpt_restore), reinterpret_cast<void **>(&c_norm_forward),
                         reinterpret_cast<void **>(&c_norm_backward), reinterpret_cast<void **>(&c_act_forward), reinterpret_cast<void **>(&c_act_backward),
                         reinterpret_cast<void **>(&c_attn_forward), reinterpret_cast<void **>(&c_attn_backward), reinterpret_cast<void **>(&c_embed_forward), reinterpret_cast<void **>(&c_embed_backward),
                         reinterpret_cast<void **>(&c_xent_forward), reinterpret_cast<void **>(&c_xent_backward), reinterpret_cast<void **>(&c_orth_update),
                         reinterpret_cast<void **>(&c_last_error)};
    constexpr Py_ssize_t ENTRIES = sizeof(to) / sizeof(to[0]);
    if (n != ENTRIES + 1) return PyErr_Format(PyExc_TypeError, "%zd arguments expected, %zd given", ENTRIES + 1, n);
    for (Py_ssize_t i = 0; i < ENTRIES; ++i) {
        *to[i] = PyLong_AsVoidPtr(args[i + 1]);
        if (PyErr_Occurred()) return nullptr;
    }
    Py_INCREF(args[0]);
    Py_XDECREF(error_class);
    error_class = args[0];
    Py_RETURN_NONE;
}

#define KT_METHOD(name, n) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(entry<name, n>)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(bind)), METH_FASTCALL, nullptr},
                         KT_METHOD(ckpt_store, 4),
                         KT_METHOD(ckpt_restore, 6),
                         KT_METHOD(norm_forward, 10),
                         KT_METHOD(norm_backward, 12),
                         KT_METHOD(act_forward, 6),
                         KT_METHOD(act_backward, 7),
                         KT_METHOD(attn_forward, 10),
                         KT_METHOD(attn_backward, 15),
                         KT_METHOD(embed_forward, 5),
                         KT_METHOD(embed_backward, 7),
                         KT_METHOD(xent_forward, 8),
                         KT_METHOD(xent_backward, 11),
                         KT_METHOD(orth_update, 9),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module_def = {PyModuleDef_HEAD_INIT, "_fast", KT_BELONGS, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fast() { return PyModule_Create(&module_def); }
