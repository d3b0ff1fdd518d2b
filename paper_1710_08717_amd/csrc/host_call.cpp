// The binding's plain calls without Python in between: checks, output and workspace tensors and the library call of one operator in one C function.
//
// An operator on small matrices takes 2 to 10 us on the GPU; the same steps in
// Python take 8 to 10 us of host time a call, here 4.3 to 5, 3 of them the launch (16 matrices of 32 x 32).  A function
// here answers None, having done nothing, for everything but a plain call -- torch.Tensor arguments on the current device, dense, contiguous, of one
// precision, of shapes that fit, no mode or transform of torch active, flags and numbers of the usual types, sizes the library accepts -- and
// the Python code then runs as it would without it, errors included.
#include <Python.h>
#include <dlfcn.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <initializer_list>
#include <mutex>
#include <stdexcept>
#include <tuple>
#include <unordered_map>

#include "la.h"

namespace {

struct Lib {
    decltype(&la_workspace_bytes) workspace_bytes;
    decltype(&la_gp_workspace_bytes) gp_workspace_bytes;
    decltype(&la_potrf_batched_ws) potrf;
    decltype(&la_potrf_backward_ws) potrf_backward;
    decltype(&la_trsm_batched_ws) trsm, trmm;
    decltype(&la_trsm_backward_ws) trsm_backward, trmm_backward;
    decltype(&la_syrk_batched_ws) syrk;
    decltype(&la_syrk_backward_ws) syrk_backward;
    decltype(&la_gemm2_batched_ws) gemm2;
    decltype(&la_gemm2_backward_ws) gemm2_backward;
    decltype(&la_potri_ws) potri;
    decltype(&la_potri_backward_ws) potri_backward;
    decltype(&la_sumlogdiag) sumlogdiag;
    decltype(&la_gp_criterion) gp_criterion;
    decltype(&la_delta_rule_step) delta_rule_step;
    decltype(&la_layer_norm) layer_norm;
    decltype(&la_layer_norm_backward_workspace_bytes) layer_norm_backward_workspace_bytes;
    decltype(&la_layer_norm_backward) layer_norm_backward;
    decltype(&la_clip_gradients_workspace_bytes) clip_gradients_workspace_bytes;
    decltype(&la_clip_gradients) clip_gradients;
} lib;
bool bound = false;

// Dense tensors of ordinary autograd; anything that wraps or records them (vmap, functionalisation, fake tensors, subclasses) goes by the Python code.
const c10::DispatchKeySet plain_keys({c10::DispatchKey::CUDA, c10::DispatchKey::AutogradCUDA, c10::DispatchKey::ADInplaceOrView,
                                      c10::DispatchKey::AutocastCUDA});

bool plain(const at::Tensor &t) { return (t.key_set() | plain_keys) == plain_keys; }

// A result or scratch tensor: plain as well, or the call is none of this file's.
at::Tensor fresh(at::IntArrayRef sizes, const at::TensorOptions &options)
{
    at::Tensor t = at::empty(sizes, options.requires_grad(false));
    if (!plain(t))
        throw std::runtime_error("not a plain tensor");
    return t;
}

// One call's tensors.
struct Call {
    const at::Tensor *first = nullptr;
    la_dtype dt = LA_F32;
    int device = -1;
    int64_t batch = 0;
    at::Tensor workspace;  // kept until the call is enqueued
    void *wp = nullptr;
    size_t wb = 0;

    // the tensor behind `o`, or null where the call is not a plain one
    const at::Tensor *tensor(PyObject *o)
    {
        if (!THPVariable_CheckExact(o))
            return nullptr;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.defined() || !t.is_cuda() || t.layout() != c10::kStrided || !plain(t) || !t.is_contiguous() ||
            t.dim() > 8)
            return nullptr;
        if (!first) {
            if (t.scalar_type() == at::kFloat)
                dt = LA_F32;
            else if (t.scalar_type() == at::kDouble)
                dt = LA_F64;
            else
                return nullptr;
            device = t.get_device();
            first = &t;
        } else if (t.scalar_type() != first->scalar_type() || t.get_device() != device) {
            return nullptr;
        }
        return &t;
    }
    // plain circumstances: asked once the tensors are there.  (A mode or a transform -- grad, jvp, vmap, functionalisation, tracing -- wraps what is
    // allocated inside it, whatever the arguments are: its key is among the included ones.)
    bool here() const
    {
        return bound && device == c10::hip::current_device() && !c10::impl::TorchDispatchModeTLS::any_modes_set() &&
               !at::impl::torch_function_mode_enabled() &&
               (c10::impl::tls_local_dispatch_key_set().included_ | c10::default_included_set) == c10::default_included_set;
    }
    void scratch(size_t need)
    {
        if (!need)
            return;
        workspace = fresh({(int64_t)need}, first->options().dtype(at::kByte));
        wp = workspace.data_ptr();
        wb = need;
    }
    // bytes of an operator's workspace; the answers are remembered, they depend on the sizes only
    void scratch(la_op op, int n, int m, int k)
    {
        using Key = std::tuple<int, int, int64_t, int, int, int>;
        struct Hash {
            size_t operator()(const Key &x) const
            {
                size_t h = (size_t)std::get<2>(x);
                for (size_t v : {(size_t)std::get<0>(x), (size_t)std::get<1>(x), (size_t)std::get<3>(x), (size_t)std::get<4>(x), (size_t)std::get<5>(x)})
                    h = h * 1000003u + v;
                return h;
            }
        };
        static std::mutex mutex;
        static std::unordered_map<Key, size_t, Hash> sizes;
        const Key key{(int)op, (int)dt, batch, n, m, k};
        size_t need;
        {
            std::lock_guard<std::mutex> lock(mutex);
            const auto it = sizes.find(key);
            if (it != sizes.end()) {
                need = it->second;
            } else {
                need = lib.workspace_bytes(op, dt, batch, n, m, k);
                if (sizes.size() >= 4096)  // (a program with that many sizes asks again)
                    sizes.clear();
                sizes.emplace(key, need);
            }
        }
        scratch(need);
    }
    void *stream() const { return (void *)c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(device).stream(); }
};

int64_t leading(const at::Tensor &t, int trailing)
{
    int64_t b = 1;
    for (int64_t i = 0; i < t.dim() - trailing; ++i)
        b *= t.size(i);
    return b;
}

bool small(int64_t x) { return x >= 0 && x <= (1 << 20); }
bool flag(PyObject *o, int &v)
{
    if (!PyBool_Check(o))
        return false;
    v = o == Py_True;
    return true;
}
bool number(PyObject *o, double &v)
{
    if (!PyFloat_CheckExact(o))
        return false;
    v = PyFloat_AS_DOUBLE(o);
    return true;
}

// Allocations and the library's call, without the GIL, as torch makes its own: an allocation may wait for the GPU, and the GPU for a callback in
// Python.  An exception does not leave with the GIL released.  (Only std::exception is caught, here and below: a thread that meets the end of the
// interpreter where it takes the GIL back is unwound, which must not be held up.)
template <class F>
la_status unlocked(F &&f)
{
    la_status s = LA_ERR_RUNTIME;
    PyThreadState *state = PyEval_SaveThread();
    try {
        s = f();
    } catch (const std::exception &) {
    }
    PyEval_RestoreThread(state);
    return s;
}

PyObject *wrap(const at::Tensor &t) { return THPVariable_Wrap(t); }
PyObject *pair(const at::Tensor &a, const at::Tensor &b)
{
    PyObject *x = wrap(a), *y = x ? wrap(b) : nullptr, *r = y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return r;
}
PyObject *none()
{
    Py_INCREF(Py_None);
    return Py_None;
}
// takes its references over; null where one is
PyObject *triple(PyObject *x, PyObject *y, PyObject *z)
{
    PyObject *r = x && y && z ? PyTuple_Pack(3, x, y, z) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    Py_XDECREF(z);
    return r;
}
at::Tensor like(const at::Tensor &t) { return fresh(t.sizes(), t.options()); }
at::Tensor shaped(const at::Tensor &t, int drop, std::initializer_list<int64_t> last)
{
    std::vector<int64_t> s(t.sizes().begin(), t.sizes().end() - drop);
    s.insert(s.end(), last);
    return fresh(s, t.options());
}

// A C++ exception (no memory, say) leaves the call to the Python code, which meets it again and reports it as ever.
#define LA_FUNCTION(name, count)                                                       \
    PyObject *name##_call(PyObject *const *a);                                         \
    PyObject *name(PyObject *, PyObject *const *a, Py_ssize_t n)                       \
    {                                                                                  \
        if (n == (count)) {                                                            \
            try {                                                                      \
                if (PyObject *r = name##_call(a))                                      \
                    return r;                                                          \
            } catch (const std::exception &) {                                         \
            }                                                                          \
            if (PyErr_Occurred())                                                      \
                PyErr_Clear();                                                         \
        }                                                                              \
        Py_RETURN_NONE;                                                                \
    }                                                                                  \
    PyObject *name##_call(PyObject *const *a)

// a batch of square matrices
bool square(const at::Tensor *t, int64_t &n)
{
    if (!t || t->dim() < 2)
        return false;
    n = t->size(-1);
    return t->size(-2) == n && small(n);
}

LA_FUNCTION(potrf, 2)
{
    Call c;
    int64_t n;
    int lower;
    const at::Tensor *A = c.tensor(a[0]);
    if (!square(A, n) || !flag(a[1], lower) || !c.here())
        return nullptr;
    c.batch = leading(*A, 2);
    at::Tensor L;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        L = like(*A);
        c.scratch(LA_OP_POTRF, (int)n, 0, 0);
        return lib.potrf(c.dt, lower, c.batch, (int)n, A->data_ptr(), L.data_ptr(), nullptr, c.wp, c.wb, st);
    });
    return s == LA_OK ? wrap(L) : nullptr;
}

LA_FUNCTION(potrf_backward, 3)
{
    Call c;
    int64_t n;
    int lower;
    const at::Tensor *L = c.tensor(a[0]), *G = L ? c.tensor(a[1]) : nullptr;
    if (!square(L, n) || !G || G->sizes() != L->sizes() || !flag(a[2], lower) || !c.here())
        return nullptr;
    c.batch = leading(*L, 2);
    at::Tensor W;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        W = like(*G);
        c.scratch(LA_OP_POTRF_BACKWARD, (int)n, 0, 0);
        return lib.potrf_backward(c.dt, lower, c.batch, (int)n, L->data_ptr(), G->data_ptr(), W.data_ptr(), c.wp, c.wb, st);
    });
    return s == LA_OK ? wrap(W) : nullptr;
}

// the vectors of trsm / trmm: m of them, or -1
int64_t vectors(const at::Tensor &L, const at::Tensor *X, int64_t n, int right)
{
    if (!X || X->dim() < 2 || X->size(right ? -1 : -2) != n || leading(*X, 2) != leading(L, 2))
        return -1;
    return X->size(right ? -2 : -1);
}

// (solve, L, A, lower, trans, rightside, alpha)
LA_FUNCTION(tri, 7)
{
    Call c;
    int64_t n;
    int solve, lower, trans, right;
    double alpha;
    const at::Tensor *L = c.tensor(a[1]), *A = L ? c.tensor(a[2]) : nullptr;
    if (!square(L, n) || !flag(a[0], solve) || !flag(a[3], lower) || !flag(a[4], trans) || !flag(a[5], right) || !number(a[6], alpha))
        return nullptr;
    const int64_t m = vectors(*L, A, n, right);
    if (m < 0 || m > INT32_MAX || !c.here())
        return nullptr;
    c.batch = leading(*L, 2);
    at::Tensor B;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        B = like(*A);
        c.scratch(solve ? LA_OP_TRSM : LA_OP_TRMM, (int)n, (int)m, 0);
        return (solve ? lib.trsm : lib.trmm)(c.dt, lower, trans, right, alpha, c.batch, (int)n, (int)m, L->data_ptr(), A->data_ptr(), B.data_ptr(),
                                             c.wp, c.wb, st);
    });
    return s == LA_OK ? wrap(B) : nullptr;
}

// (solve, L, X, Bbar, lower, trans, rightside, alpha)
LA_FUNCTION(tri_backward, 8)
{
    Call c;
    int64_t n;
    int solve, lower, trans, right;
    double alpha;
    const at::Tensor *L = c.tensor(a[1]), *X = L ? c.tensor(a[2]) : nullptr, *G = X ? c.tensor(a[3]) : nullptr;
    if (!square(L, n) || !G || !flag(a[0], solve) || !flag(a[4], lower) || !flag(a[5], trans) || !flag(a[6], right) || !number(a[7], alpha) ||
        X->sizes() != G->sizes())
        return nullptr;
    const int64_t m = vectors(*L, X, n, right);
    if (m < 0 || m > INT32_MAX || !c.here())
        return nullptr;
    c.batch = leading(*L, 2);
    at::Tensor Ab, Lb;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        Ab = like(*G);
        Lb = like(*L);
        c.scratch(solve ? LA_OP_TRSM_BACKWARD : LA_OP_TRMM_BACKWARD, (int)n, (int)m, 0);
        return (solve ? lib.trsm_backward : lib.trmm_backward)(c.dt, lower, trans, right, alpha, c.batch, (int)n, (int)m, L->data_ptr(),
                                                               X->data_ptr(), G->data_ptr(), Ab.data_ptr(), Lb.data_ptr(), c.wp, c.wb, st);
    });
    return s == LA_OK ? pair(Ab, Lb) : nullptr;
}

LA_FUNCTION(syrk, 3)
{
    Call c;
    int trans;
    double alpha;
    const at::Tensor *A = c.tensor(a[0]);
    if (!A || A->dim() < 2 || !flag(a[1], trans) || !number(a[2], alpha))
        return nullptr;
    const int64_t n = A->size(trans ? -1 : -2), k = A->size(trans ? -2 : -1);
    if (!small(n) || k > INT32_MAX || !c.here())
        return nullptr;
    c.batch = leading(*A, 2);
    at::Tensor B;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        B = shaped(*A, 2, {n, n});
        c.scratch(LA_OP_SYRK, (int)n, 0, (int)k);
        return lib.syrk(c.dt, trans, alpha, c.batch, (int)n, (int)k, A->data_ptr(), B.data_ptr(), c.wp, c.wb, st);
    });
    return s == LA_OK ? wrap(B) : nullptr;
}

LA_FUNCTION(syrk_backward, 4)
{
    Call c;
    int trans;
    double alpha;
    const at::Tensor *A = c.tensor(a[0]), *G = A ? c.tensor(a[1]) : nullptr;
    if (!G || A->dim() < 2 || G->dim() < 2 || !flag(a[2], trans) || !number(a[3], alpha))
        return nullptr;
    const int64_t n = A->size(trans ? -1 : -2), k = A->size(trans ? -2 : -1);
    if (G->size(-1) != n || G->size(-2) != n || leading(*A, 2) != leading(*G, 2) || !small(n) || k > INT32_MAX || !c.here())
        return nullptr;
    c.batch = leading(*A, 2);
    at::Tensor B;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        B = like(*A);
        c.scratch(LA_OP_SYRK_BACKWARD, (int)n, 0, (int)k);
        return lib.syrk_backward(c.dt, trans, alpha, c.batch, (int)n, (int)k, A->data_ptr(), G->data_ptr(), B.data_ptr(), c.wp, c.wb, st);
    });
    return s == LA_OK ? wrap(B) : nullptr;
}

// sizes of C = t_a(A) t_b(B)
bool product(const at::Tensor *A, const at::Tensor *B, int ta, int tb, int64_t &m, int64_t &n, int64_t &k)
{
    if (!A || !B || A->dim() < 2 || B->dim() < 2)
        return false;
    m = A->size(ta ? -1 : -2);
    k = A->size(ta ? -2 : -1);
    n = B->size(tb ? -2 : -1);
    return B->size(tb ? -1 : -2) == k && leading(*A, 2) == leading(*B, 2) && m <= INT32_MAX && n <= INT32_MAX && k <= INT32_MAX;
}

LA_FUNCTION(gemm2, 5)
{
    Call c;
    int ta, tb;
    double alpha;
    int64_t m, n, k;
    const at::Tensor *A = c.tensor(a[0]), *B = A ? c.tensor(a[1]) : nullptr;
    if (!flag(a[2], ta) || !flag(a[3], tb) || !number(a[4], alpha) || !product(A, B, ta, tb, m, n, k) || !c.here())
        return nullptr;
    c.batch = leading(*A, 2);
    at::Tensor C;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        C = shaped(*A, 2, {m, n});
        c.scratch(LA_OP_GEMM2, (int)n, (int)m, (int)k);
        return lib.gemm2(c.dt, ta, tb, alpha, c.batch, (int)m, (int)n, (int)k, A->data_ptr(), B->data_ptr(), C.data_ptr(), c.wp, c.wb, st);
    });
    return s == LA_OK ? wrap(C) : nullptr;
}

LA_FUNCTION(gemm2_backward, 6)
{
    Call c;
    int ta, tb;
    double alpha;
    int64_t m, n, k;
    const at::Tensor *A = c.tensor(a[0]), *B = A ? c.tensor(a[1]) : nullptr, *G = B ? c.tensor(a[2]) : nullptr;
    if (!G || !flag(a[3], ta) || !flag(a[4], tb) || !number(a[5], alpha) || !product(A, B, ta, tb, m, n, k) || G->dim() < 2 || G->size(-2) != m ||
        G->size(-1) != n || leading(*G, 2) != leading(*A, 2) || !c.here())
        return nullptr;
    c.batch = leading(*A, 2);
    at::Tensor Ab, Bb;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        Ab = like(*A);
        Bb = like(*B);
        c.scratch(LA_OP_GEMM2_BACKWARD, (int)n, (int)m, (int)k);
        return lib.gemm2_backward(c.dt, ta, tb, alpha, c.batch, (int)m, (int)n, (int)k, A->data_ptr(), B->data_ptr(), G->data_ptr(), Ab.data_ptr(),
                                  Bb.data_ptr(), c.wp, c.wb, st);
    });
    return s == LA_OK ? pair(Ab, Bb) : nullptr;
}

LA_FUNCTION(potri, 2)
{
    Call c;
    int64_t n;
    int lower;
    const at::Tensor *L = c.tensor(a[0]);
    if (!square(L, n) || !flag(a[1], lower) || !c.here())
        return nullptr;
    c.batch = leading(*L, 2);
    at::Tensor B;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        B = like(*L);
        c.scratch(LA_OP_POTRI, (int)n, 0, 0);
        return lib.potri(c.dt, lower, c.batch, (int)n, L->data_ptr(), B.data_ptr(), c.wp, c.wb, st);
    });
    return s == LA_OK ? wrap(B) : nullptr;
}

LA_FUNCTION(potri_backward, 4)
{
    Call c;
    int64_t n;
    int lower;
    const at::Tensor *L = c.tensor(a[0]), *B = L ? c.tensor(a[1]) : nullptr, *G = B ? c.tensor(a[2]) : nullptr;
    if (!square(L, n) || !G || B->sizes() != L->sizes() || G->sizes() != L->sizes() || !flag(a[3], lower) || !c.here())
        return nullptr;
    c.batch = leading(*L, 2);
    at::Tensor X;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        X = like(*L);
        c.scratch(LA_OP_POTRI_BACKWARD, (int)n, 0, 0);
        return lib.potri_backward(c.dt, lower, c.batch, (int)n, L->data_ptr(), B->data_ptr(), G->data_ptr(), X.data_ptr(), c.wp, c.wb, st);
    });
    return s == LA_OK ? wrap(X) : nullptr;
}

LA_FUNCTION(sumlogdiag, 1)
{
    Call c;
    const at::Tensor *L = c.tensor(a[0]);
    int64_t n;
    if (!square(L, n) || !c.here())
        return nullptr;
    at::Tensor o;
    void *st = c.stream();
    const int64_t batch = leading(*L, 2);
    const la_status s = unlocked([&] {
        o = shaped(*L, 2, {});
        return lib.sumlogdiag(c.dt, batch, (int)n, L->data_ptr(), o.data_ptr(), st);
    });
    return s == LA_OK ? wrap(o) : nullptr;
}

LA_FUNCTION(gp_criterion, 2)
{
    Call c;
    int64_t n;
    const at::Tensor *A = c.tensor(a[0]), *y = A ? c.tensor(a[1]) : nullptr;
    if (!square(A, n) || !y || y->dim() < 1 || y->size(-1) != n || leading(*y, 1) != leading(*A, 2) || !c.here())
        return nullptr;
    c.batch = leading(*A, 2);
    at::Tensor Ab, loss;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        Ab = like(*A);
        loss = shaped(*A, 2, {});
        c.scratch(lib.gp_workspace_bytes(c.dt, c.batch, (int)n));
        return lib.gp_criterion(c.dt, c.batch, (int)n, A->data_ptr(), y->data_ptr(), loss.data_ptr(), Ab.data_ptr(), nullptr, c.wp, c.wb, st);
    });
    return s == LA_OK ? pair(loss, Ab) : nullptr;
}

// The sequence-layer operators.  Their tensors are float32, bfloat16 or float16 (float64 too for layer norm and clipping) with gates, states and statistics
// in float32: each has its type asked for.
bool layer_type(const at::Tensor &t, la_dtype &dt)
{
    switch (t.scalar_type()) {
    case at::kFloat: dt = LA_F32; return true;
    case at::kDouble: dt = LA_F64; return true;
    case at::kBFloat16: dt = LA_BF16; return true;
    case at::kHalf: dt = LA_F16; return true;
    default: return false;
    }
}

struct LayerCall : Call {
    // a plain dense tensor on the call's device (the first one's), or null
    const at::Tensor *dense(PyObject *o, bool contiguous = true)
    {
        if (!THPVariable_CheckExact(o))
            return nullptr;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.defined() || !t.is_cuda() || t.layout() != c10::kStrided || !plain(t) || (contiguous && !t.is_contiguous()) || t.dim() > 8)
            return nullptr;
        if (!first) {
            device = t.get_device();
            first = &t;
        } else if (t.get_device() != device) {
            return nullptr;
        }
        return &t;
    }
    // None gives true and no tensor
    bool maybe(PyObject *o, const at::Tensor *&t)
    {
        t = o == Py_None ? nullptr : dense(o);
        return o == Py_None || t;
    }
};

// A tensor of the caller's that a call has written: autograd is told, as of torch's own operators in place.  (An inference tensor has no versions.)
void written(const at::Tensor &t)
{
    if (!t.is_inference())
        t.unsafeGetTensorImpl()->bump_version();
}

// [batch, heads, size] whose heads and elements are dense: elements from one sequence to the next, or -1
int64_t step_rows(const at::Tensor &t)
{
    const int64_t row = t.size(1) * t.size(2);
    if (t.numel() == 0 || (t.size(2) != 1 && t.stride(2) != 1) || (t.size(1) != 1 && t.stride(1) != t.size(2)))
        return -1;
    return t.size(0) == 1 ? row : t.stride(0) >= row ? t.stride(0) : -1;
}

// (q, k, v, g, beta, state, slots, scale)
LA_FUNCTION(delta_rule_step, 8)
{
    LayerCall c;
    la_dtype dt;
    const at::Tensor *q = c.dense(a[0], false), *k = q ? c.dense(a[1], false) : nullptr, *v = k ? c.dense(a[2], false) : nullptr;
    const at::Tensor *g = v ? c.dense(a[3]) : nullptr, *beta = g ? c.dense(a[4]) : nullptr, *state = beta ? c.dense(a[5]) : nullptr, *slots;
    double scale;
    if (!state || !c.maybe(a[6], slots) || !layer_type(*q, dt) || dt == LA_F64 || q->dim() != 3 || v->dim() != 3 || k->sizes() != q->sizes() ||
        k->scalar_type() != q->scalar_type() || v->scalar_type() != q->scalar_type() || state->dim() != 4)
        return nullptr;
    const int64_t batch = q->size(0), hk = q->size(1), dk = q->size(2), hv = v->size(1), dv = v->size(2);
    if (v->size(0) != batch || hk < 1 || hv < 1 || hv % hk || !small(hv) || !small(dk) || !small(dv))
        return nullptr;
    for (const at::Tensor *t : {g, beta})
        if (t->dim() != 2 || t->size(0) != batch || t->size(1) != hv || t->scalar_type() != at::kFloat)
            return nullptr;
    if (state->scalar_type() != at::kFloat || state->size(1) != hv || state->size(2) != dk || state->size(3) != dv ||
        (slots && (slots->scalar_type() != at::kInt || slots->dim() != 1 || slots->size(0) != batch)))
        return nullptr;
    if (a[7] == Py_None)
        scale = std::pow((double)dk, -0.5);
    else if (!number(a[7], scale))
        return nullptr;
    const int64_t lq = step_rows(*q), lk = step_rows(*k), lv = step_rows(*v);
    if (lq < 0 || lk < 0 || lv < 0 || !c.here())
        return nullptr;
    at::Tensor o;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        o = fresh({batch, hv, dv}, v->options());
        return lib.delta_rule_step(dt, batch, (int)hk, (int)hv, (int)dk, (int)dv, q->data_ptr(), lq, k->data_ptr(), lk, v->data_ptr(), lv,
                                   (const float *)g->data_ptr(), (const float *)beta->data_ptr(), scale, (float *)state->data_ptr(), state->size(0),
                                   slots ? (const int32_t *)slots->data_ptr() : nullptr, o.data_ptr(), st);
    });
    if (s != LA_OK)
        return nullptr;
    written(*state);
    return wrap(o);
}

// the type of weight and bias beside x: x's own, or float32 beside 16 bits
bool weights_fit(const at::Tensor &x, la_dtype dt, std::initializer_list<const at::Tensor *> w, la_dtype &wdt)
{
    wdt = dt;
    bool seen = false;
    for (const at::Tensor *t : w)
        if (t) {
            la_dtype own;
            if (t->dim() != 1 || t->size(0) != x.size(-1) || !layer_type(*t, own) || (seen && own != wdt) ||
                !(own == dt || (own == LA_F32 && (dt == LA_BF16 || dt == LA_F16))))
                return false;
            wdt = own;
            seen = true;
        }
    return true;
}

// (x, weight, bias, eps, want_stats): dense rows
LA_FUNCTION(layer_norm, 5)
{
    LayerCall c;
    la_dtype dt, wdt;
    const at::Tensor *x = c.dense(a[0]), *w, *b;
    double eps;
    int stats;
    if (!x || x->dim() < 1 || !c.maybe(a[1], w) || !c.maybe(a[2], b) || !number(a[3], eps) || !flag(a[4], stats) || !layer_type(*x, dt) ||
        !weights_fit(*x, dt, {w, b}, wdt) || x->size(-1) > INT32_MAX || !c.here())
        return nullptr;
    const int64_t rows = leading(*x, 1), n = x->size(-1);
    at::Tensor y, mean, rstd;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        y = like(*x);
        if (stats) {
            const at::IntArrayRef lead = x->sizes().slice(0, x->dim() - 1);
            const at::TensorOptions o = x->options().dtype(dt == LA_F64 ? at::kDouble : at::kFloat);
            mean = fresh(lead, o);
            rstd = fresh(lead, o);
        }
        return lib.layer_norm(dt, wdt, rows, (int)n, n, x->data_ptr(), w ? w->data_ptr() : nullptr, b ? b->data_ptr() : nullptr, eps, y.data_ptr(),
                              stats ? mean.data_ptr() : nullptr, stats ? rstd.data_ptr() : nullptr, st);
    });
    if (s != LA_OK)
        return nullptr;
    return stats ? triple(wrap(y), wrap(mean), wrap(rstd)) : triple(wrap(y), none(), none());
}

// (x, y_bar, mean, rstd, weight, want_weights): dense rows
LA_FUNCTION(layer_norm_backward, 6)
{
    LayerCall c;
    la_dtype dt, wdt;
    const at::Tensor *x = c.dense(a[0]), *yb = x ? c.dense(a[1]) : nullptr, *mean = yb ? c.dense(a[2]) : nullptr, *rstd = mean ? c.dense(a[3]) : nullptr, *w;
    int want;
    if (!rstd || x->dim() < 1 || !c.maybe(a[4], w) || !flag(a[5], want) || !layer_type(*x, dt) || !weights_fit(*x, dt, {w}, wdt) ||
        yb->sizes() != x->sizes() || yb->scalar_type() != x->scalar_type() || x->size(-1) > INT32_MAX)
        return nullptr;
    const at::IntArrayRef lead = x->sizes().slice(0, x->dim() - 1);
    for (const at::Tensor *t : {mean, rstd})
        if (t->sizes() != lead || t->scalar_type() != (dt == LA_F64 ? at::kDouble : at::kFloat))
            return nullptr;
    if (!c.here())
        return nullptr;
    const int64_t rows = leading(*x, 1), n = x->size(-1);
    at::Tensor xb, wb, bb;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        xb = like(*x);
        if (want) {
            const at::TensorOptions o = w ? w->options() : x->options();
            wb = fresh({n}, o);
            bb = fresh({n}, o);
        }
        c.scratch(lib.layer_norm_backward_workspace_bytes(dt, rows, (int)n));
        return lib.layer_norm_backward(dt, wdt, rows, (int)n, n, x->data_ptr(), yb->data_ptr(), mean->data_ptr(), rstd->data_ptr(),
                                       w ? w->data_ptr() : nullptr, xb.data_ptr(), want ? wb.data_ptr() : nullptr, want ? bb.data_ptr() : nullptr, c.wp,
                                       c.wb, st);
    });
    if (s != LA_OK)
        return nullptr;
    return want ? triple(wrap(xb), wrap(wb), wrap(bb)) : triple(wrap(xb), none(), none());
}

// (grads, max_norm, out or None): lists of tensors
LA_FUNCTION(clip_gradients, 3)
{
    LayerCall c;
    double limit;
    if (!PyList_CheckExact(a[0]) || !number(a[1], limit) || !(a[2] == Py_None || PyList_CheckExact(a[2])))
        return nullptr;
    const Py_ssize_t n = PyList_GET_SIZE(a[0]);
    if (n < 1 || n > INT32_MAX || (a[2] != Py_None && PyList_GET_SIZE(a[2]) != n))
        return nullptr;
    std::vector<la_dtype> types(n);
    std::vector<int64_t> sizes(n);
    std::vector<const void *> src(n);
    std::vector<void *> dst(n);
    std::vector<at::Tensor> held;  // (the lists may change while the GIL is released)
    held.reserve(2 * n);
    bool wide = false;
    for (Py_ssize_t i = 0; i < n; ++i) {
        const at::Tensor *x = c.dense(PyList_GET_ITEM(a[0], i)), *y = x && a[2] != Py_None ? c.dense(PyList_GET_ITEM(a[2], i)) : x;
        if (!x || !y || !layer_type(*x, types[i]) || (y != x && (y->sizes() != x->sizes() || y->scalar_type() != x->scalar_type())))
            return nullptr;
        sizes[i] = x->numel();
        src[i] = x->data_ptr();
        dst[i] = y->data_ptr();
        wide |= types[i] == LA_F64;
        held.push_back(*x);
        held.push_back(*y);
    }
    c.first = &held[0];
    if (!c.here())
        return nullptr;
    at::Tensor norm;
    void *st = c.stream();
    const la_status s = unlocked([&] {
        norm = fresh({}, held[0].options().dtype(wide ? at::kDouble : at::kFloat));
        c.scratch(lib.clip_gradients_workspace_bytes((int)n, sizes.data()));
        return lib.clip_gradients((int)n, types.data(), sizes.data(), src.data(), dst.data(), limit, wide ? LA_F64 : LA_F32, norm.data_ptr(), c.wp, c.wb, st);
    });
    if (s != LA_OK)
        return nullptr;
    for (size_t i = 1; i < held.size(); i += 2)  // (the outputs)
        written(held[i]);
    return wrap(norm);
}

// bind(path): the library whose functions are called
PyObject *bind(PyObject *, PyObject *path)
{
    const char *p = PyUnicode_AsUTF8(path);
    if (!p)
        return nullptr;
    void *h = dlopen(p, RTLD_NOW | RTLD_LOCAL);
    if (!h)
        return PyErr_Format(PyExc_OSError, "%s", dlerror());
#define LA_BIND(member, symbol)                                                         \
    if (!(lib.member = reinterpret_cast<decltype(lib.member)>(dlsym(h, #symbol))))      \
    return PyErr_Format(PyExc_OSError, "%s has no %s", p, #symbol)
    LA_BIND(workspace_bytes, la_workspace_bytes);
    LA_BIND(gp_workspace_bytes, la_gp_workspace_bytes);
    LA_BIND(potrf, la_potrf_batched_ws);
    LA_BIND(potrf_backward, la_potrf_backward_ws);
    LA_BIND(trsm, la_trsm_batched_ws);
    LA_BIND(trmm, la_trmm_batched_ws);
    LA_BIND(trsm_backward, la_trsm_backward_ws);
    LA_BIND(trmm_backward, la_trmm_backward_ws);
    LA_BIND(syrk, la_syrk_batched_ws);
    LA_BIND(syrk_backward, la_syrk_backward_ws);
    LA_BIND(gemm2, la_gemm2_batched_ws);
    LA_BIND(gemm2_backward, la_gemm2_backward_ws);
    LA_BIND(potri, la_potri_ws);
    LA_BIND(potri_backward, la_potri_backward_ws);
    LA_BIND(sumlogdiag, la_sumlogdiag);
    LA_BIND(gp_criterion, la_gp_criterion);
    LA_BIND(delta_rule_step, la_delta_rule_step);
    LA_BIND(layer_norm, la_layer_norm);
    LA_BIND(layer_norm_backward_workspace_bytes, la_layer_norm_backward_workspace_bytes);
    LA_BIND(layer_norm_backward, la_layer_norm_backward);
    LA_BIND(clip_gradients_workspace_bytes, la_clip_gradients_workspace_bytes);
    LA_BIND(clip_gradients, la_clip_gradients);
#undef LA_BIND
    bound = true;
    Py_RETURN_NONE;
}

#define LA_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {LA_METHOD(potrf), LA_METHOD(potrf_backward), LA_METHOD(tri), LA_METHOD(tri_backward), LA_METHOD(syrk), LA_METHOD(syrk_backward),
                         LA_METHOD(gemm2), LA_METHOD(gemm2_backward), LA_METHOD(potri), LA_METHOD(potri_backward), LA_METHOD(sumlogdiag),
                         LA_METHOD(gp_criterion), LA_METHOD(delta_rule_step), LA_METHOD(layer_norm), LA_METHOD(layer_norm_backward),
                         LA_METHOD(clip_gradients), {"bind", bind, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_la_host", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__la_host() { return PyModule_Create(&module); }
