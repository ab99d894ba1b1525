// The native calls of the operators around the products: the same contract as in host_calls.cpp, arguments in the order of sp24.py's functions.
#include "host_args.hpp"

namespace {

// a matrix of exactly this shape and type, or (None) nothing
struct Matrix {
    void* p = nullptr;
    int64_t ld_ = 0;
    Matrix(Call& c, int i, int64_t rows, int64_t cols, at::ScalarType type)
    {
        if (!c.ok || c.none(i)) return;
        const at::Tensor* t = c.rowmajor(i);
        if (!c.ok) return;
        c.require(t->size(0) == rows && t->size(1) == cols && t->scalar_type() == type);
        p = t->data_ptr();
        ld_ = ld(*t);
    }
};

// a contiguous vector of n entries, or (None) nothing
template <typename T>
T* entries(Call& c, int i, int64_t n, at::ScalarType type)
{
    if (!c.ok || c.none(i)) return nullptr;
    const at::Tensor* t = c.contiguous(i);
    if (!c.ok) return nullptr;
    c.require(t->numel() == n && t->scalar_type() == type);
    return static_cast<T*>(t->data_ptr());
}
const float* floats(Call& c, int i, int64_t n) { return entries<const float>(c, i, n, at::kFloat); }

// the caller's workspace (argument i), or a new one where some is needed
struct Scratch {
    at::Tensor own;
    void* p = nullptr;
    size_t bytes = 0;
    Scratch(Call& c, int i, size_t need, const at::Tensor& like)
    {
        if (!c.ok) return;
        const at::Tensor* t = &own;
        if (!c.none(i)) t = c.contiguous(i);
        else if (need > 0) own = make({(int64_t)need}, at::kByte, like);
        else return;
        if (!c.ok) return;
        p = t->data_ptr();
        bytes = (size_t)t->numel() * t->element_size();
    }
};

sp24_act activation(Call& c, int i)
{
    if (c.text_is(i, "none")) return SP24_ACT_NONE;
    if (c.text_is(i, "gelu")) return SP24_ACT_GELU;
    if (c.text_is(i, "silu")) return SP24_ACT_SILU;
    c.require(c.text_is(i, "relu"));
    return SP24_ACT_RELU;
}

PyObject* wrap(at::Tensor& t)
{
    if (!t.defined()) Py_RETURN_NONE;
    return THPVariable_Wrap(std::move(t));
}
// a tuple of new references; none of them may be null
template <typename... O>
PyObject* tuple(O... objects)
{
    PyObject* items[] = {objects...};
    constexpr int n = sizeof...(O);
    PyObject* t = PyTuple_New(n);
    for (int i = 0; i < n; ++i) {
        if (t && items[i]) PyTuple_SET_ITEM(t, i, items[i]);
        else Py_XDECREF(items[i]);
    }
    return t;
}
PyObject* again(PyObject* o)
{
    Py_INCREF(o);
    return o;
}

// (X, weight, eps, residual, out_dtype, want_rstd, hidden, out) -> (y, scale, hidden, rstd)
PyObject* rmsnorm(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor* X = c.rowmajor(0);
    if (!c.ok) return not_handled();
    const int64_t N = X->size(0), H = X->size(1);
    const at::ScalarType type = X->scalar_type(), out = c.none(4) ? type : c.dtype(4);
    c.require(!c.none(1));
    const float* w = floats(c, 1, H);
    const float eps = c.real(2);
    const Matrix r(c, 3, N, H, type);
    const int want_rstd = c.truth(5);
    if (!c.ok) return not_handled();
    const sp24_dtype ti = type_of(type, c.ok), to = type_of(out, c.ok);
    const int64_t shape[2] = {N, H};
    const bool with_hidden = !c.none(3) || !c.none(6);
    at::Tensor scale, rstd, hidden;
    Matrix h(c, 6, N, H, type);
    Result y(c, 7, shape, out, X);
    if (!c.ok) return not_handled();
    if (with_hidden && c.none(6)) {
        hidden = make(shape, type, *X);
        h.p = hidden.data_ptr();
        h.ld_ = H;
    }
    if (to == SP24_I8 || to == SP24_F8) scale = make({N}, at::kFloat, *X);
    if (want_rstd) rstd = make({N}, at::kFloat, *X);
    const void* px = X->data_ptr();
    void *py = y.t->data_ptr(), *st = stream();
    float *ps = scale.defined() ? static_cast<float*>(scale.data_ptr()) : nullptr, *pr = rstd.defined() ? static_cast<float*>(rstd.data_ptr()) : nullptr;
    const int64_t ldx = ld(*X), ldy = ld(*y.t);
    const sp24_status s = without_gil([&] { return sp24_rmsnorm(px, r.p, w, eps, py, ps, h.p, pr, N, H, ldx, r.ld_, ldy, h.ld_, ti, to, st); });
    if (s != SP24_OK) return refused(self, s, "sp24_rmsnorm");
    return tuple(y.object(), wrap(scale), c.none(6) ? wrap(hidden) : again(args[6]), wrap(rstd));
}

// (X, out_dtype, out) -> (codes, scale)
PyObject* quantize_rows(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor* X = c.rowmajor(0);
    const at::ScalarType out = c.dtype(1);
    if (!c.ok) return not_handled();
    const int64_t N = X->size(0), H = X->size(1), shape[2] = {N, H};
    const sp24_dtype ti = type_of(X->scalar_type(), c.ok), to = type_of(out, c.ok);
    Result q(c, 2, shape, out, X);
    if (!c.ok) return not_handled();
    at::Tensor scale = make({N}, at::kFloat, *X);
    const void* px = X->data_ptr();
    void *pq = q.t->data_ptr(), *st = stream();
    float* ps = static_cast<float*>(scale.data_ptr());
    const int64_t ldx = ld(*X), ldq = ld(*q.t);
    const sp24_status s = without_gil([&] { return sp24_quantize_rows(px, pq, ps, N, H, ldx, ldq, ti, to, st); });
    return s == SP24_OK ? tuple(q.object(), wrap(scale)) : refused(self, s, "sp24_quantize_rows");
}

// (dY, hidden, weight, rstd, dhidden, workspace, out) -> (dX, dweight)
PyObject* rmsnorm_backward(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor* dY = c.rowmajor(0);
    if (!c.ok) return not_handled();
    const int64_t N = dY->size(0), H = dY->size(1), shape[2] = {N, H};
    const at::ScalarType type = dY->scalar_type();
    c.require(!c.none(1) && !c.none(2) && !c.none(3));
    const Matrix h(c, 1, N, H, type), dh(c, 4, N, H, type);
    const float *w = floats(c, 2, H), *rstd = floats(c, 3, N);
    if (!c.ok) return not_handled();
    const sp24_dtype t = type_of(type, c.ok);
    Result dX(c, 6, shape, type, dY);
    Scratch ws(c, 5, sp24_rmsnorm_backward_workspace_bytes(N, H), *dY);
    if (!c.ok) return not_handled();
    at::Tensor dw = make({H}, at::kFloat, *dY);
    const void* pd = dY->data_ptr();
    void *px = dX.t->data_ptr(), *st = stream();
    float* pw = static_cast<float*>(dw.data_ptr());
    const int64_t lddy = ld(*dY), lddx = ld(*dX.t);
    const sp24_status s = without_gil([&] { return sp24_rmsnorm_backward(pd, h.p, w, rstd, dh.p, px, pw, N, H, lddy, h.ld_, dh.ld_, lddx, t, ws.p, ws.bytes, st); });
    return s == SP24_OK ? tuple(dX.object(), wrap(dw)) : refused(self, s, "sp24_rmsnorm_backward");
}

// the compressed pair (arguments 0 and 1) and its size
struct Weights {
    const at::Tensor *V = nullptr, *meta = nullptr;
    int64_t M = 0, K = 0;
    explicit Weights(Call& c)
    {
        V = c.contiguous(0);
        meta = c.contiguous(1);
        if (!c.ok) return;
        c.require(V->dim() == 2 && is_input(V->scalar_type()));
        if (!c.ok) return;
        M = V->size(0);
        K = V->size(1) * 2;
        c.require(meta->numel() * (int64_t)meta->element_size() == M * (K / 8));
    }
};

// (V, meta, X, out_dtype, w_scale, x_scale, bias, act, residual, preact, layout, out)
PyObject* linear(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const Weights a(c);
    const at::Tensor* X = c.rowmajor(2);
    const at::ScalarType out = c.dtype(3);
    const sp24_layout l = c.layout(10);
    if (!c.ok) return not_handled();
    const int64_t M = a.M, N = X->size(0), K = a.K, shape[2] = {N, M};
    c.require(X->size(1) == K && X->scalar_type() == a.V->scalar_type());
    const float *ws = floats(c, 4, M), *xs = floats(c, 5, N), *b = floats(c, 6, M);
    const sp24_act act = activation(c, 7);
    const Matrix r(c, 8, N, M, out), z(c, 9, N, M, out);
    Result y(c, 11, shape, out, a.V);
    if (!c.ok) return not_handled();
    const sp24_dtype ti = type_of(a.V->scalar_type(), c.ok), to = type_of(out, c.ok);
    if (!c.ok) return not_handled();
    const void *pv = a.V->data_ptr(), *pm = a.meta->data_ptr(), *px = X->data_ptr();
    void *py = y.t->data_ptr(), *st = stream();
    const int64_t ldx = ld(*X), ldy = ld(*y.t);
    const sp24_status s = without_gil([&] { return sp24_linear(pv, pm, px, py, M, N, K, ldx, ldy, ws, xs, b, act, r.p, r.ld_, z.p, z.ld_, ti, to, l, st); });
    return s == SP24_OK ? y.object() : refused(self, s, "sp24_linear");
}

// (V, meta, X, offsets, out_dtype, w_scale, x_scale, bias, act, preact, layout, out)
PyObject* linear_grouped(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const Weights a(c);
    const at::Tensor *X = c.rowmajor(2), *offsets = c.contiguous(3);
    const at::ScalarType out = c.dtype(4);
    const sp24_layout l = c.layout(10);
    if (!c.ok) return not_handled();
    const int64_t experts = offsets->numel() - 1, R = X->size(0), K = a.K;
    c.require(offsets->scalar_type() == at::kInt && experts >= 1 && experts <= SP24_MOST_EXPERTS && X->size(1) == K && X->scalar_type() == a.V->scalar_type());
    if (!c.ok || a.M % experts != 0) return not_handled();
    const int64_t M = a.M / experts, shape[2] = {R, M};
    const float *ws = floats(c, 5, a.M), *xs = floats(c, 6, R), *b = floats(c, 7, a.M);
    const sp24_act act = activation(c, 8);
    const Matrix z(c, 9, R, M, out);
    Result y(c, 11, shape, out, a.V);
    if (!c.ok) return not_handled();
    const sp24_dtype ti = type_of(a.V->scalar_type(), c.ok), to = type_of(out, c.ok);
    if (!c.ok) return not_handled();
    const void *pv = a.V->data_ptr(), *pm = a.meta->data_ptr(), *px = X->data_ptr();
    const int32_t* po = static_cast<const int32_t*>(offsets->data_ptr());
    void *py = y.t->data_ptr(), *st = stream();
    const int64_t ldx = ld(*X), ldy = ld(*y.t);
    const sp24_status s = without_gil([&] {
        return sp24_linear_grouped(pv, pm, px, py, po, (int)experts, M, R, K, ldx, ldy, ws, xs, b, act, z.p, z.ld_, ti, to, l, st);
    });
    return s == SP24_OK ? y.object() : refused(self, s, "sp24_linear_grouped");
}

// (A, B, offsets, out_dtype): a new result only
PyObject* gemm_dense_grouped(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor *A = c.rowmajor(0), *B = c.rowmajor(1), *offsets = c.contiguous(2);
    const at::ScalarType out = c.dtype(3);
    c.require(c.none(4));
    if (!c.ok) return not_handled();
    const int64_t experts = offsets->numel() - 1, M = A->size(0), R = A->size(1), N = B->size(1);
    c.require(offsets->scalar_type() == at::kInt && experts >= 1 && experts <= SP24_MOST_EXPERTS && B->size(0) == R && B->scalar_type() == A->scalar_type());
    const sp24_dtype ti = type_of(A->scalar_type(), c.ok), to = type_of(out, c.ok);
    if (!c.ok) return not_handled();
    at::Tensor D = make({experts, M, N}, out, *A);
    const void *pa = A->data_ptr(), *pb = B->data_ptr();
    const int32_t* po = static_cast<const int32_t*>(offsets->data_ptr());
    void *pd = D.data_ptr(), *st = stream();
    const int64_t lda = ld(*A), ldb = ld(*B);
    const sp24_status s = without_gil([&] { return sp24_gemm_dense_grouped(pa, pb, pd, po, (int)experts, M, N, R, lda, ldb, N, ti, to, st); });
    return s == SP24_OK ? wrap(D) : refused(self, s, "sp24_gemm_dense_grouped");
}

// (dY, preact, act, offsets, workspace) -> (dZ, dZt, dbias)
PyObject* linear_backward(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor* dY = c.rowmajor(0);
    const sp24_act act = activation(c, 2);
    if (!c.ok) return not_handled();
    const int64_t N = dY->size(0), M = dY->size(1);
    const at::ScalarType type = dY->scalar_type();
    const bool copy = act != SP24_ACT_NONE;
    Matrix z(c, copy ? 1 : 0, N, M, type);
    c.require(!copy || !c.none(1));
    const bool grouped = !c.none(3);
    int64_t experts = 0;
    const int32_t* po = nullptr;
    if (grouped) {
        const at::Tensor* offsets = c.contiguous(3);
        if (!c.ok) return not_handled();
        experts = offsets->numel() - 1;
        c.require(offsets->scalar_type() == at::kInt && experts >= 1 && experts <= SP24_MOST_EXPERTS);
        po = static_cast<const int32_t*>(offsets->data_ptr());
    }
    if (!c.ok) return not_handled();
    const sp24_dtype t = type_of(type, c.ok);
    Scratch ws(c, 4, sp24_linear_backward_workspace_bytes(M, N, grouped), *dY);
    if (!c.ok) return not_handled();
    const int64_t pitch = (N + 7) / 8 * 8;                     // 16-byte rows, which the weights' gradient asks for
    at::Tensor dZ, dZt = make({M, pitch}, type, *dY), db = grouped ? make({experts, M}, at::kFloat, *dY) : make({M}, at::kFloat, *dY);
    if (pitch != N) dZt = dZt.narrow(1, 0, N);
    if (copy) dZ = make({N, M}, type, *dY);
    const void* pd = dY->data_ptr();
    void *pz = copy ? dZ.data_ptr() : nullptr, *pt = dZt.data_ptr(), *st = stream();
    float* pb = static_cast<float*>(db.data_ptr());
    const int64_t lddy = ld(*dY);
    const sp24_status s = without_gil([&] {
        return sp24_linear_backward(pd, copy ? z.p : nullptr, pz, pt, pb, M, N, lddy, z.ld_, M, pitch, act, po, (int)experts, t, ws.p, ws.bytes, st);
    });
    if (s != SP24_OK) return refused(self, s, "sp24_linear_backward");
    return tuple(copy ? wrap(dZ) : again(args[0]), wrap(dZt), wrap(db));
}

// (ids, experts, workspace) -> (offsets, slots, rows)
PyObject* moe_sort(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor* ids = c.contiguous(0);
    const int64_t experts = c.integer(1);
    if (!c.ok) return not_handled();
    c.require(ids->scalar_type() == at::kInt && experts >= 1 && experts <= SP24_MOST_EXPERTS);
    if (!c.ok) return not_handled();
    const int64_t T = ids->numel(), R = sp24_moe_rows(T, (int)experts);
    Scratch ws(c, 2, sp24_moe_sort_workspace_bytes(T, (int)experts), *ids);
    if (!c.ok) return not_handled();
    at::Tensor offsets = make({experts + 1}, at::kInt, *ids), slots = make(ids->sizes(), at::kInt, *ids), rows = make({R}, at::kInt, *ids);
    const int32_t* pi = static_cast<const int32_t*>(ids->data_ptr());
    int32_t *po = static_cast<int32_t*>(offsets.data_ptr()), *ps = static_cast<int32_t*>(slots.data_ptr()), *pr = static_cast<int32_t*>(rows.data_ptr());
    void* st = stream();
    const sp24_status s = without_gil([&] { return sp24_moe_sort(pi, po, ps, pr, T, (int)experts, R, ws.p, ws.bytes, st); });
    return s == SP24_OK ? tuple(wrap(offsets), wrap(slots), wrap(rows)) : refused(self, s, "sp24_moe_sort");
}

// (X, rows, topk, scale, out)
PyObject* moe_gather(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor *X = c.rowmajor(0), *rows = c.contiguous(1);
    const int64_t topk = c.integer(2);
    if (!c.ok) return not_handled();
    c.require(rows->scalar_type() == at::kInt && topk >= 1 && topk <= INT32_MAX);
    const int64_t N = X->size(0), H = X->size(1), R = rows->numel(), shape[2] = {R, H};
    const float* scale = floats(c, 3, N);
    if (!c.ok) return not_handled();
    const sp24_dtype t = type_of(X->scalar_type(), c.ok);
    Result xs(c, 4, shape, X->scalar_type(), X);
    if (!c.ok) return not_handled();
    const bool scaled = !c.none(3);
    at::Tensor scales;
    if (scaled) scales = make({R}, at::kFloat, *X);
    const void* px = X->data_ptr();
    const int32_t* pr = static_cast<const int32_t*>(rows->data_ptr());
    void *po = xs.t->data_ptr(), *st = stream();
    float* ps = scaled ? static_cast<float*>(scales.data_ptr()) : nullptr;
    const int64_t ldx = ld(*X), ldxs = ld(*xs.t);
    const sp24_status s = without_gil([&] { return sp24_moe_gather(px, scale, pr, po, ps, N, R, (int)topk, H, ldx, ldxs, t, st); });
    if (s != SP24_OK) return refused(self, s, "sp24_moe_gather");
    return scaled ? tuple(xs.object(), wrap(scales)) : xs.object();
}

// (Y, slots, weights, residual, out)
PyObject* moe_combine(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor *Y = c.rowmajor(0), *slots = c.contiguous(1);
    if (!c.ok) return not_handled();
    c.require(slots->dim() == 2 && slots->scalar_type() == at::kInt);
    if (!c.ok) return not_handled();
    const int64_t N = slots->size(0), topk = slots->size(1), R = Y->size(0), H = Y->size(1), shape[2] = {N, H};
    c.require(topk <= INT32_MAX);
    const float* w = floats(c, 2, N * topk);
    const Matrix r(c, 3, N, H, Y->scalar_type());
    if (!c.ok) return not_handled();
    const sp24_dtype t = type_of(Y->scalar_type(), c.ok);
    Result out(c, 4, shape, Y->scalar_type(), Y);
    if (!c.ok) return not_handled();
    const void* py = Y->data_ptr();
    const int32_t* ps = static_cast<const int32_t*>(slots->data_ptr());
    void *po = out.t->data_ptr(), *st = stream();
    const int64_t ldy = ld(*Y), ldo = ld(*out.t);
    const sp24_status s = without_gil([&] { return sp24_moe_combine(py, ps, w, r.p, po, N, R, (int)topk, H, ldy, r.ld_, ldo, t, st); });
    return s == SP24_OK ? out.object() : refused(self, s, "sp24_moe_combine");
}

// (dout, Y, slots, rows, weights, out) -> (dY, dweights)
PyObject* moe_combine_backward(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor *Y = c.rowmajor(1), *slots = c.contiguous(2);
    if (!c.ok) return not_handled();
    c.require(slots->dim() == 2 && slots->scalar_type() == at::kInt && !c.none(0) && !c.none(3) && !c.none(4));
    if (!c.ok) return not_handled();
    const int64_t N = slots->size(0), topk = slots->size(1), R = Y->size(0), H = Y->size(1), shape[2] = {R, H};
    c.require(topk <= INT32_MAX);
    const Matrix d(c, 0, N, H, Y->scalar_type());
    const int32_t* pr = entries<const int32_t>(c, 3, R, at::kInt);
    const float* w = floats(c, 4, N * topk);
    if (!c.ok) return not_handled();
    const sp24_dtype t = type_of(Y->scalar_type(), c.ok);
    Result dY(c, 5, shape, Y->scalar_type(), Y);
    if (!c.ok) return not_handled();
    at::Tensor dw = make({N, topk}, at::kFloat, *Y);
    const void* py = Y->data_ptr();
    const int32_t* ps = static_cast<const int32_t*>(slots->data_ptr());
    void *po = dY.t->data_ptr(), *st = stream();
    float* pw = static_cast<float*>(dw.data_ptr());
    const int64_t ldy = ld(*Y), lddy = ld(*dY.t);
    const sp24_status s = without_gil([&] { return sp24_moe_combine_backward(d.p, py, pr, ps, w, po, pw, N, R, (int)topk, H, d.ld_, ldy, lddy, t, st); });
    return s == SP24_OK ? tuple(dY.object(), wrap(dw)) : refused(self, s, "sp24_moe_combine_backward");
}

// what a call of the functions below reads or writes has to be on the device whose stream it goes to
void here(Call& c, const at::Tensor* t)
{
    if (c.ok && t) c.require(t->device().index() == c10::hip::current_device());
}
template <typename T>
T* entries_here(Call& c, int i, int64_t n, at::ScalarType type)
{
    T* const p = entries<T>(c, i, n, type);
    if (c.ok && !c.none(i)) here(c, c.tensor(i));
    return p;
}

bool softmax_score(Call& c, int i)
{
    if (c.text_is(i, "softmax")) return true;
    c.require(c.text_is(i, "sigmoid"));
    return false;
}
int small(Call& c, int i)
{
    const int64_t v = c.integer(i);
    c.require(v >= 0 && v <= INT32_MAX);
    return c.ok ? (int)v : 0;
}
bool is_float_row(at::ScalarType t) { return t == at::kFloat || t == at::kHalf || t == at::kBFloat16; }
bool is_code_type(at::ScalarType t) { return t == at::kChar || t == at::kFloat8_e4m3fn; }

// rows kept in 8 bits (argument i, a pair of codes and scales)
struct Kept {
    PyObject* parts[2] = {nullptr, nullptr};
    const at::Tensor *codes = nullptr, *scale = nullptr;
    int64_t N = 0, H = 0, ld_ = 0;
    Kept(Call& c, int i)
    {
        if (!c.ok) return;
        c.require(PyTuple_Check(c.args[i]) && PyTuple_GET_SIZE(c.args[i]) == 2);
        if (!c.ok) return;
        for (int k = 0; k < 2; ++k) parts[k] = PyTuple_GET_ITEM(c.args[i], k);
        Call p{parts, true};
        codes = p.rowmajor(0);
        scale = p.contiguous(1);
        c.require(p.ok);
        if (!c.ok) return;
        N = codes->size(0);
        H = codes->size(1);
        ld_ = ld(*codes);
        c.require(is_code_type(codes->scalar_type()) && scale->scalar_type() == at::kFloat &&
                  scale->numel() == N * ((H + SP24_CHECKPOINT_BLOCK - 1) / SP24_CHECKPOINT_BLOCK));
        here(c, codes);
        here(c, scale);
    }
    const void* data() const { return codes->data_ptr(); }
    const float* scales() const { return static_cast<const float*>(scale->data_ptr()); }
};

// (logits, topk, score, bias, groups, groups_kept, group_best, renormalise, scale, want_scores, want_load) -> (ids, weights, scores, load)
PyObject* moe_route(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor* X = c.rowmajor(0);
    const int topk = small(c, 1);
    const bool softmax = softmax_score(c, 2);
    if (!c.ok) return not_handled();
    const int64_t N = X->size(0), E = X->size(1);
    here(c, X);
    c.require(is_float_row(X->scalar_type()) && topk >= 1 && topk <= SP24_MOST_CHOICES && E >= 1 && E <= SP24_MOST_EXPERTS);
    const float* bias = entries_here<const float>(c, 3, E, at::kFloat);
    const int groups = small(c, 4), kept = small(c, 5), best = small(c, 6), renormalise = c.truth(7);
    const float scale = c.real(8);
    const int want_scores = c.truth(9), want_load = c.truth(10);
    if (!c.ok) return not_handled();
    const sp24_dtype t = type_of(X->scalar_type(), c.ok);
    at::Tensor ids = make({N, topk}, at::kInt, *X), weights = make({N, topk}, at::kFloat, *X), scores, load;
    if (want_scores) scores = make({N, E}, at::kFloat, *X);
    if (want_load) load = make({E}, at::kInt, *X);
    const void* px = X->data_ptr();
    int32_t *pi = static_cast<int32_t*>(ids.data_ptr()), *pl = want_load ? static_cast<int32_t*>(load.data_ptr()) : nullptr;
    float *pw = static_cast<float*>(weights.data_ptr()), *ps = want_scores ? static_cast<float*>(scores.data_ptr()) : nullptr;
    void* st = stream();
    const int64_t ldx = ld(*X);
    const sp24_status s = without_gil([&] {
        return sp24_moe_route(px, bias, pi, pw, ps, pl, N, (int)E, topk, groups, kept, best, softmax ? SP24_SCORE_SOFTMAX : SP24_SCORE_SIGMOID, renormalise, scale,
                              ldx, t, st);
    });
    return s == SP24_OK ? tuple(wrap(ids), wrap(weights), wrap(scores), wrap(load)) : refused(self, s, "sp24_moe_route");
}

// (logits, ids, dweights, score, renormalise, scale, dscores, out)
PyObject* moe_route_backward(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor *X = c.rowmajor(0), *ids = c.contiguous(1);
    const bool softmax = softmax_score(c, 3);
    c.require(!c.none(2));
    if (!c.ok) return not_handled();
    c.require(ids->dim() == 2 && ids->scalar_type() == at::kInt && is_float_row(X->scalar_type()));
    if (!c.ok) return not_handled();
    const int64_t N = X->size(0), E = X->size(1), topk = ids->size(1), shape[2] = {N, E};
    here(c, X);
    here(c, ids);
    c.require(ids->size(0) == N && E >= 1 && E <= SP24_MOST_EXPERTS && topk >= 1 && topk <= SP24_MOST_CHOICES);
    if (!c.ok) return not_handled();
    const float *dw = entries_here<const float>(c, 2, N * topk, at::kFloat), *ds = entries_here<const float>(c, 6, N * E, at::kFloat);
    const int renormalise = c.truth(4);
    const float scale = c.real(5);
    if (!c.ok) return not_handled();
    const sp24_dtype t = type_of(X->scalar_type(), c.ok);
    Result d(c, 7, shape, X->scalar_type(), X);
    here(c, d.t);
    if (!c.ok) return not_handled();
    const void* px = X->data_ptr();
    const int32_t* pi = static_cast<const int32_t*>(ids->data_ptr());
    void *pd = d.t->data_ptr(), *st = stream();
    const int64_t ldx = ld(*X), ldd = ld(*d.t);
    const sp24_status s = without_gil([&] {
        return sp24_moe_route_backward(px, pi, dw, ds, pd, N, (int)E, (int)topk, softmax ? SP24_SCORE_SOFTMAX : SP24_SCORE_SIGMOID, renormalise, scale, ldx, ldd,
                                       t, st);
    });
    return s == SP24_OK ? d.object() : refused(self, s, "sp24_moe_route_backward");
}

// (X, dtype, out) -> (codes, scale)
PyObject* checkpoint_rows(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor* X = c.rowmajor(0);
    const at::ScalarType code = c.dtype(1);
    if (!c.ok) return not_handled();
    here(c, X);
    c.require(is_float_row(X->scalar_type()) && is_code_type(code));
    const int64_t N = X->size(0), H = X->size(1), shape[2] = {N, H};
    Result q(c, 2, shape, code, X);
    here(c, q.t);
    if (!c.ok) return not_handled();
    const sp24_dtype t = type_of(X->scalar_type(), c.ok), to = type_of(code, c.ok);
    at::Tensor scale = make({N, (H + SP24_CHECKPOINT_BLOCK - 1) / SP24_CHECKPOINT_BLOCK}, at::kFloat, *X);
    const void* px = X->data_ptr();
    void *pq = q.t->data_ptr(), *st = stream();
    float* ps = static_cast<float*>(scale.data_ptr());
    const int64_t ldx = ld(*X), ldq = ld(*q.t);
    const sp24_status s = without_gil([&] { return sp24_checkpoint_rows(px, pq, ps, N, H, ldx, ldq, t, to, st); });
    return s == SP24_OK ? tuple(q.object(), wrap(scale)) : refused(self, s, "sp24_checkpoint_rows");
}

// (checkpoint, out_dtype, act, rows, topk, out)
PyObject* restore_rows(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const Kept k(c, 0);
    const at::ScalarType out = c.dtype(1);
    const sp24_act act = activation(c, 2);
    if (!c.ok) return not_handled();
    int64_t R = k.N;
    if (!c.none(3)) {
        const at::Tensor* rows = c.contiguous(3);
        if (!c.ok) return not_handled();
        R = rows->numel();
    }
    const int32_t* rows = entries_here<const int32_t>(c, 3, R, at::kInt);
    const int topk = small(c, 4);
    c.require(is_float_row(out));
    const int64_t shape[2] = {R, k.H}, H = k.H, N = k.N, ldk = k.ld_;
    Result o(c, 5, shape, out, k.codes);
    here(c, o.t);
    if (!c.ok) return not_handled();
    const sp24_dtype code = type_of(k.codes->scalar_type(), c.ok), t = type_of(out, c.ok);
    const void* pc = k.data();
    const float* ps = k.scales();
    void *po = o.t->data_ptr(), *st = stream();
    const int64_t ldo = ld(*o.t);
    const sp24_status s = without_gil([&] { return sp24_restore_rows(pc, ps, rows, po, N, R, topk, H, ldk, ldo, act, code, t, st); });
    return s == SP24_OK ? o.object() : refused(self, s, "sp24_restore_rows");
}

// (dY, preact, act, offsets, workspace) -> (dZ, dZt, dbias)
PyObject* linear_backward_checkpoint(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const at::Tensor* dY = c.rowmajor(0);
    const sp24_act act = activation(c, 2);
    if (!c.ok) return not_handled();
    here(c, dY);
    const int64_t N = dY->size(0), M = dY->size(1);
    const at::ScalarType type = dY->scalar_type();
    const bool copy = act != SP24_ACT_NONE;
    const void* pz = nullptr;
    const float* ps = nullptr;
    int64_t ldz = 0;
    sp24_dtype code = SP24_I8;
    if (copy) {
        const Kept k(c, 1);
        c.require(c.ok && k.N == N && k.H == M);
        if (!c.ok) return not_handled();
        pz = k.data();
        ps = k.scales();
        ldz = k.ld_;
        code = type_of(k.codes->scalar_type(), c.ok);
    }
    const bool grouped = !c.none(3);
    int64_t experts = 0;
    const int32_t* po = nullptr;
    if (grouped) {
        const at::Tensor* offsets = c.contiguous(3);
        if (!c.ok) return not_handled();
        here(c, offsets);
        experts = offsets->numel() - 1;
        c.require(offsets->scalar_type() == at::kInt && experts >= 1 && experts <= SP24_MOST_EXPERTS);
        po = static_cast<const int32_t*>(offsets->data_ptr());
    }
    if (!c.ok) return not_handled();
    const sp24_dtype t = type_of(type, c.ok);
    Scratch ws(c, 4, sp24_linear_backward_workspace_bytes(M, N, grouped), *dY);
    if (c.ok && !c.none(4)) here(c, c.tensor(4));
    if (!c.ok) return not_handled();
    const int64_t pitch = (M + 7) / 8 * 8, lddy = ld(*dY);     // 16-byte rows, which the weights' gradient asks for
    const void* pd = dY->data_ptr();
    const bool own = copy || reinterpret_cast<uintptr_t>(pd) % 16 != 0 || lddy % 8 != 0;
    at::Tensor dZ = own ? make_pitched(N, M, pitch, type, *dY) : *dY, db = grouped ? make({experts, M}, at::kFloat, *dY) : make({M}, at::kFloat, *dY);
    void *pdz = own ? dZ.data_ptr() : nullptr, *st = stream();
    float* pb = static_cast<float*>(db.data_ptr());
    const sp24_status s = without_gil([&] {
        return sp24_linear_backward_checkpoint(pd, pz, ps, pdz, nullptr, pb, M, N, lddy, ldz, pitch, 0, act, po, (int)experts, code, t, ws.p, ws.bytes, st);
    });
    if (s != SP24_OK) return refused(self, s, "sp24_linear_backward_checkpoint");
    at::Tensor turned = dZ.t();
    return tuple(own ? wrap(dZ) : again(args[0]), wrap(turned), wrap(db));
}

// A matrix that is row-major or the transpose of one (argument 0): its order and row stride
struct Ordered {
    const at::Tensor* t = nullptr;
    sp24_aorder order = SP24_A_KMAJOR;
    int64_t ld_ = 0;
    explicit Ordered(Call& c)
    {
        t = c.tensor(0);
        c.require(c.ok && t->dim() == 2);
        if (!c.ok) return;
        here(c, t);
        const int64_t M = t->size(0), K = t->size(1);
        const int64_t by_row = M > 1 ? t->stride(0) : std::max(t->stride(0), K), by_column = K > 1 ? t->stride(1) : std::max(t->stride(1), M);
        if ((t->stride(1) == 1 || K <= 1) && by_row % 8 == 0) ld_ = by_row;
        else {
            c.require(t->stride(0) == 1 || M <= 1);
            order = SP24_A_MMAJOR;
            ld_ = by_column;
        }
    }
};

// (A, checkpoint, out_dtype, out, workspace)
PyObject* gemm_dense_checkpoint(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const Ordered a(c);
    const Kept k(c, 1);
    const at::ScalarType out = c.dtype(2);
    if (!c.ok) return not_handled();
    const int64_t M = a.t->size(0), K = k.N, N = k.H, shape[2] = {M, N};
    c.require(a.t->size(1) == K);
    const sp24_dtype ti = type_of(a.t->scalar_type(), c.ok), to = type_of(out, c.ok), code = type_of(k.codes->scalar_type(), c.ok);
    Result d(c, 3, shape, out, a.t);
    here(c, d.t);
    Scratch ws(c, 4, sp24_gemm_dense_checkpoint_workspace_bytes(M, N, K, 0), *a.t);
    if (c.ok && !c.none(4)) here(c, c.tensor(4));
    if (!c.ok) return not_handled();
    const void *pa = a.t->data_ptr(), *pc = k.data();
    const float* ps = k.scales();
    void *pd = d.t->data_ptr(), *st = stream();
    const int64_t ldd = ld(*d.t);
    const sp24_status s = without_gil([&] { return sp24_gemm_dense_checkpoint(pa, a.order, pc, ps, pd, M, N, K, a.ld_, k.ld_, ldd, ti, code, to, ws.p, ws.bytes, st); });
    return s == SP24_OK ? d.object() : refused(self, s, "sp24_gemm_dense_checkpoint");
}

// (A, checkpoint, offsets, out_dtype, rows, topk, out, workspace): a new result only
PyObject* gemm_dense_grouped_checkpoint(PyObject* self, PyObject* const* args, Py_ssize_t)
{
    Call c{args, true};
    const Ordered a(c);
    const Kept k(c, 1);
    const at::Tensor* offsets = c.contiguous(2);
    const at::ScalarType out = c.dtype(3);
    const int topk = small(c, 5);
    c.require(c.none(6));
    if (!c.ok) return not_handled();
    here(c, offsets);
    const int64_t experts = offsets->numel() - 1, M = a.t->size(0), R = a.t->size(1), N = k.H, tokens = k.N;
    c.require(offsets->scalar_type() == at::kInt && experts >= 1 && experts <= SP24_MOST_EXPERTS && (!c.none(4) || tokens == R));
    const int32_t* rows = entries_here<const int32_t>(c, 4, R, at::kInt);
    Scratch ws(c, 7, sp24_gemm_dense_checkpoint_workspace_bytes(M, N, R, 1), *a.t);
    if (c.ok && !c.none(7)) here(c, c.tensor(7));
    const sp24_dtype ti = type_of(a.t->scalar_type(), c.ok), to = type_of(out, c.ok), code = c.ok ? type_of(k.codes->scalar_type(), c.ok) : SP24_I8;
    if (!c.ok) return not_handled();
    at::Tensor D = make({experts, M, N}, out, *a.t);
    const void *pa = a.t->data_ptr(), *pc = k.data();
    const float* ps = k.scales();
    const int32_t* po = static_cast<const int32_t*>(offsets->data_ptr());
    void *pd = D.data_ptr(), *st = stream();
    const sp24_status s = without_gil([&] {
        return sp24_gemm_dense_grouped_checkpoint(pa, a.order, pc, ps, rows, pd, po, (int)experts, M, N, R, tokens, topk, a.ld_, k.ld_, N, ti, code, to, ws.p, ws.bytes, st);
    });
    return s == SP24_OK ? wrap(D) : refused(self, s, "sp24_gemm_dense_grouped_checkpoint");
}

} // namespace

PyMethodDef sp24_layer_methods[] = {
    SP24_METHOD("sp24_rmsnorm", rmsnorm),
    SP24_METHOD("sp24_quantize_rows", quantize_rows),
    SP24_METHOD("sp24_rmsnorm_backward", rmsnorm_backward),
    SP24_METHOD("sp24_linear", linear),
    SP24_METHOD("sp24_linear_backward", linear_backward),
    SP24_METHOD("sp24_linear_grouped", linear_grouped),
    SP24_METHOD("sp24_gemm_dense_grouped", gemm_dense_grouped),
    SP24_METHOD("sp24_moe_sort", moe_sort),
    SP24_METHOD("sp24_moe_gather", moe_gather),
    SP24_METHOD("sp24_moe_combine", moe_combine),
    SP24_METHOD("sp24_moe_combine_backward", moe_combine_backward),
    SP24_METHOD("sp24_moe_route", moe_route),
    SP24_METHOD("sp24_moe_route_backward", moe_route_backward),
    SP24_METHOD("sp24_checkpoint_rows", checkpoint_rows),
    SP24_METHOD("sp24_restore_rows", restore_rows),
    SP24_METHOD("sp24_linear_backward_checkpoint", linear_backward_checkpoint),
    SP24_METHOD("sp24_gemm_dense_checkpoint", gemm_dense_checkpoint),
    SP24_METHOD("sp24_gemm_dense_grouped_checkpoint", gemm_dense_grouped_checkpoint),
    {nullptr, nullptr, 0, nullptr}};
