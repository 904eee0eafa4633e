// _ddtorch: torch tensors to the C calls of dd_learner.h.  A parameter list of a model has hundreds
// of tensors; reading their addresses, sizes and types one by one from Python takes longer than
// the kernels (190 us for 5 x 192 tensors, against 12 us here).  Checks and marshalling only.
#include <cstdint>
#include <string>
#include <vector>

#include <torch/csrc/autograd/python_variable.h>

#include "dd_learner.h"

namespace {

struct Refused {
    std::string why;
};

[[noreturn]] void refuse(std::string why) { throw Refused{std::move(why)}; }

// Python's own error is set.
struct Raised {};

// Numbers.  One that does not convert ends the call before it starts: what stands for "error" in the
// conversions (-1, null) are arguments that the C calls would take.
void *pointer(PyObject *o)
{
    void *p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Raised{};
    return p;
}

double real(PyObject *o)
{
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) throw Raised{};
    return x;
}

long long integer(PyObject *o)
{
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) throw Raised{};
    return x;
}

bool truth(PyObject *o)
{
    const int x = PyObject_IsTrue(o);
    if (x < 0) throw Raised{};
    return x != 0;
}

dd_ctx *context(PyObject *o) { return static_cast<dd_ctx *>(pointer(o)); }

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) refuse(std::string(name) + ": want a tensor");
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda()) refuse(std::string(name) + ": want a CUDA tensor");
    return t;
}

// Address of a tensor with room for `bytes`, of an integer, or null for None.
void *address(PyObject *o, const char *name, size_t bytes)
{
    if (o == Py_None) return nullptr;
    if (PyLong_Check(o)) return pointer(o);
    const at::Tensor &t = tensor(o, name);
    if (!t.is_contiguous() || t.nbytes() < bytes) refuse(std::string(name) + ": want " + std::to_string(bytes) + " contiguous bytes");
    return t.data_ptr();
}

std::string shape_of(const at::Tensor &t)
{
    std::string s = c10::toString(t.scalar_type());
    for (int64_t i = 0; i < t.dim(); ++i)
        s += (i ? ", " : " (") + std::to_string(t.size(i)) + " by " + std::to_string(t.stride(i));
    return s + (t.dim() ? ")" : " ()");
}

// ---- lists --------------------------------------------------------------------------------

struct List {
    std::vector<void *> ptr;
    std::vector<uint64_t> n;
    std::vector<uint8_t> dtype;
    int count() const { return (int)ptr.size(); }
};

struct Sequence {
    PyObject *fast;
    explicit Sequence(PyObject *o, const char *name) : fast(PySequence_Fast(o, name)) { if (!fast) { PyErr_Clear(); refuse(std::string(name) + ": want a list of tensors"); } }
    ~Sequence() { Py_DECREF(fast); }
    Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(fast); }
    PyObject *operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(fast, i); }
};

List gradients(PyObject *o)
{
    const Sequence s(o, "grads");
    List l;
    l.ptr.resize(s.size());
    l.n.resize(s.size());
    l.dtype.resize(s.size());
    for (Py_ssize_t i = 0; i < s.size(); ++i) {
        const at::Tensor &t = tensor(s[i], "grads");
        const at::ScalarType k = t.scalar_type();
        if (k != at::kFloat && k != at::kBFloat16) refuse(std::string("gradients must be float32 or bfloat16, not ") + c10::toString(k));
        if (!t.is_contiguous()) refuse("gradients must be contiguous");
        l.ptr[i] = t.data_ptr();
        l.n[i] = (uint64_t)t.numel();
        l.dtype[i] = k == at::kBFloat16 ? DD_BF16 : DD_F32;
    }
    return l;
}

enum class Kind { kSame, kF32, kBF16 };

// A list that goes with the gradients tensor by tensor; entries may be None where `holes` says so.
std::vector<void *> matching(PyObject *o, const List &grads, const char *name, Kind kind, bool holes = false)
{
    const Sequence s(o, name);
    bool ok = s.size() == grads.count();
    std::vector<void *> p(s.size());
    for (Py_ssize_t i = 0; ok && i < s.size(); ++i) {
        if (holes && s[i] == Py_None) continue;
        const at::Tensor &t = tensor(s[i], name);
        const int want = kind == Kind::kSame ? grads.dtype[i] : kind == Kind::kF32 ? DD_F32 : DD_BF16;
        ok = t.scalar_type() == (want == DD_BF16 ? at::kBFloat16 : at::kFloat) && (uint64_t)t.numel() == grads.n[i] && t.is_contiguous();
        p[i] = t.data_ptr();
    }
    if (!ok)
        refuse(std::string(name) + " must match the gradients tensor by tensor: contiguous, same size, " +
               (kind == Kind::kSame ? "same dtype" : kind == Kind::kF32 ? "float32" : "bfloat16"));
    return p;
}

// (ctx, grads, max_norm, record, stream)
int grad_norm(PyObject *const *a)
{
    const List g = gradients(a[1]);
    return dd_grad_norm(context(a[0]), g.ptr.data(), g.n.data(), g.dtype.data(), g.count(),
                        (float)real(a[2]), (dd_grad_record *)address(a[3], "record", sizeof(dd_grad_record)),
                        pointer(a[4]));
}

// (ctx, grads, out, max_norm, record, stream)
int clip_gradients(PyObject *const *a)
{
    const List g = gradients(a[1]);
    std::vector<void *> out;
    if (a[2] != Py_None) out = matching(a[2], g, "out", Kind::kSame);
    return dd_clip_gradients(context(a[0]), g.ptr.data(), a[2] != Py_None ? out.data() : nullptr, g.n.data(),
                             g.dtype.data(), g.count(), (float)real(a[3]),
                             (dd_grad_record *)address(a[4], "record", sizeof(dd_grad_record)), pointer(a[5]));
}

// (ctx, params, grads, exp_avg, exp_avg_sq, copies, clip, step, lr, beta1, beta2, eps, weight_decay, stream)
int adamw_step(PyObject *const *a)
{
    const List g = gradients(a[2]);
    const std::vector<void *> p = matching(a[1], g, "params", Kind::kF32), m = matching(a[3], g, "exp_avg", Kind::kF32),
                              v = matching(a[4], g, "exp_avg_sq", Kind::kF32);
    std::vector<void *> copies;
    if (a[5] != Py_None) copies = matching(a[5], g, "copies", Kind::kBF16, true);
    const long long step = integer(a[7]);
    const dd_adamw opt = {real(a[8]), real(a[9]), real(a[10]), real(a[11]),
                          real(a[12]), step > 0 ? (uint64_t)step : 0};
    return dd_adamw_step(context(a[0]), &opt, (float *const *)p.data(), g.ptr.data(), (float *const *)m.data(),
                         (float *const *)v.data(), a[5] != Py_None ? copies.data() : nullptr, g.n.data(), g.dtype.data(),
                         g.count(), (const dd_grad_record *)address(a[6], "clip", sizeof(dd_grad_record)), pointer(a[13]));
}

// ---- matrices -------------------------------------------------------------------------------

// Checks a rows x cols matrix with contiguous rows and joins its row stride to `ld` (0: none yet).
void *matrix(PyObject *o, const char *name, uint64_t rows, uint64_t cols, uint64_t &ld, at::ScalarType kind = at::kBFloat16)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, name);
    if (t.dim() != 2 || (uint64_t)t.size(0) != rows || (uint64_t)t.size(1) != cols || t.scalar_type() != kind ||
        (cols > 1 && t.stride(1) != 1))
        refuse(std::string(name) + ": want " + c10::toString(kind) + " [" + std::to_string(rows) + ", " + std::to_string(cols) +
               "] with contiguous rows, got (size by stride) " + shape_of(t));
    // an expanded matrix has stride 0, which the C calls take as "the row length itself"
    if (rows > 1 && (uint64_t)t.stride(0) < cols)
        refuse(std::string(name) + ": rows overlap, got (size by stride) " + shape_of(t));
    if (rows > 1 || ld == 0) {            // a single row takes whatever stride its partners have
        const uint64_t s = rows > 1 ? (uint64_t)t.stride(0) : (cols + 7) / 8 * 8;
        if (ld && s != ld) refuse(std::string(name) + ": row stride " + std::to_string(s) + " differs from " + std::to_string(ld));
        ld = s;
    }
    return t.data_ptr();
}

// (x, w_gate, w_up, w_down) -> block and x
const void *block_of(PyObject *const *a, PyObject *act, PyObject *flags, dd_gated_ffn &b)
{
    const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "w_gate");
    if (x.dim() != 2 || w.dim() != 2) refuse("x and the weights are matrices");
    b = dd_gated_ffn{};
    b.tokens = x.size(0);
    b.d = x.size(1);
    b.f = w.size(0);
    const long long kind = integer(act), bits = integer(flags);
    b.activation = kind == (int32_t)kind ? (int32_t)kind : -1;
    b.flags = bits == (uint32_t)bits ? (uint32_t)bits : ~0u;
    const void *px = matrix(a[0], "x", b.tokens, b.d, b.ld_x);
    b.w_gate = matrix(a[1], "w_gate", b.f, b.d, b.ld_in);
    b.w_up = matrix(a[2], "w_up", b.f, b.d, b.ld_in);
    b.w_down = matrix(a[3], "w_down", b.d, b.f, b.ld_down);
    return px;
}

size_t hidden_bytes(const dd_gated_ffn &b) { return (size_t)b.tokens * ((b.f + 7) / 8 * 8) * 2; }

// (ctx, x, w_gate, w_up, w_down, y, residual, gate, up, activation, hidden, status, stream, flags)
int gated_ffn_forward(PyObject *const *a)
{
    dd_gated_ffn b;
    const void *x = block_of(a + 1, a[9], a[13], b);
    void *y = matrix(a[5], "y", b.tokens, b.d, b.ld_y), *res = matrix(a[6], "residual", b.tokens, b.d, b.ld_y);
    void *gate = matrix(a[7], "gate", b.tokens, b.f, b.ld_gate), *up = matrix(a[8], "up", b.tokens, b.f, b.ld_gate);
    return dd_gated_ffn_forward(context(a[0]), &b, x, res, gate, up, address(a[10], "hidden", hidden_bytes(b)), y,
                                (int32_t *)address(a[11], "status", 4), pointer(a[12]));
}

// (ctx, x, w_gate, w_up, w_down, gate, up, dy, dx, dw_gate, dw_up, dw_down, activation, accumulate, scratch, status, stream, flags)
int gated_ffn_backward(PyObject *const *a)
{
    dd_gated_ffn b;
    const void *x = block_of(a + 1, a[12], a[17], b);
    const void *gate = matrix(a[5], "gate", b.tokens, b.f, b.ld_gate), *up = matrix(a[6], "up", b.tokens, b.f, b.ld_gate);
    const void *dy = matrix(a[7], "dy", b.tokens, b.d, b.ld_y);
    void *dx = matrix(a[8], "dx", b.tokens, b.d, b.ld_x);
    const at::ScalarType kind = tensor(a[11], "dw_down").scalar_type();
    if (kind != at::kFloat && kind != at::kBFloat16) refuse("the weights' gradients must be float32 or bfloat16");
    void *dwg = matrix(a[9], "dw_gate", b.f, b.d, b.ld_in, kind), *dwu = matrix(a[10], "dw_up", b.f, b.d, b.ld_in, kind);
    void *dwd = matrix(a[11], "dw_down", b.d, b.f, b.ld_down, kind);
    return dd_gated_ffn_backward(context(a[0]), &b, x, gate, up, dy, dx, dwg, dwu, dwd,
                                 kind == at::kBFloat16 ? DD_BF16 : DD_F32, truth(a[13]),
                                 address(a[14], "scratch", 3 * hidden_bytes(b)), (int32_t *)address(a[15], "status", 4),
                                 pointer(a[16]));
}

// Runs a call: refusals become ValueError, numbers that do not convert raise what Python raised.  Either
// way nothing has been launched.
template <int (*CALL)(PyObject *const *), int NARGS>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    if (n != NARGS) return PyErr_Format(PyExc_TypeError, "want %d arguments, got %zd", NARGS, n);
    try {
        return PyLong_FromLong(CALL(args));
    } catch (const Raised &) {
    } catch (const Refused &r) {
        PyErr_SetString(PyExc_ValueError, r.why.c_str());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

#define ENTRY(name, n) {#name, (PyCFunction)(void (*)(void))entry<name, n>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {ENTRY(grad_norm, 5), ENTRY(clip_gradients, 6), ENTRY(adamw_step, 14), ENTRY(gated_ffn_forward, 14),
                         ENTRY(gated_ffn_backward, 18), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ddtorch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ddtorch() { return PyModule_Create(&module); }
