// _ddtorch: torch tensors to the C calls of dd_learner.h and dd_decoder.h.  A parameter list of a model has hundreds
// of tensors; reading their addresses, sizes and types one by one from Python takes longer than
// the kernels (190 us for 5 x 192 tensors, against 12 us here).  Checks and marshalling only.
#include <cmath>
#include <cstdint>
#include <string>
#include <vector>

#include <torch/csrc/autograd/python_variable.h>

#include "dd_decoder.h"

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

// ---- the decoder's operators ------------------------------------------------------------------

// A contiguous vector of `n` elements, or null for None.
void *vector(PyObject *o, const char *name, uint64_t n, at::ScalarType kind)
{
    if (o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, name);
    if (t.scalar_type() != kind || (uint64_t)t.numel() != n || !t.is_contiguous())
        refuse(std::string(name) + ": want " + std::to_string(n) + " contiguous " + c10::toString(kind) + ", got (size by stride) " + shape_of(t));
    return t.data_ptr();
}

// [tokens, heads, dim] with contiguous heads; None: no tensor.
dd_heads heads_of(PyObject *o, const char *name, uint64_t tokens, uint64_t heads, uint64_t dim, at::ScalarType kind = at::kBFloat16)
{
    if (o == Py_None) return dd_heads{};
    const at::Tensor &t = tensor(o, name);
    if (t.dim() != 3 || (uint64_t)t.size(0) != tokens || (uint64_t)t.size(1) != heads || (uint64_t)t.size(2) != dim || t.scalar_type() != kind ||
        (dim > 1 && t.stride(2) != 1))
        refuse(std::string(name) + ": want " + c10::toString(kind) + " [" + std::to_string(tokens) + ", " + std::to_string(heads) + ", " +
               std::to_string(dim) + "] with contiguous heads, got (size by stride) " + shape_of(t));
    // an expanded tensor has stride 0, which the C calls take as a contiguous tensor's
    if ((tokens > 1 && t.stride(0) < (int64_t)dim) || (heads > 1 && t.stride(1) < (int64_t)dim))
        refuse(std::string(name) + ": rows overlap, got (size by stride) " + shape_of(t));
    return dd_heads{t.data_ptr(), tokens > 1 ? (uint64_t)t.stride(0) : 0, heads > 1 ? (uint64_t)t.stride(1) : 0};
}

// (ctx, q, k, positions, frequencies, q_out, k_out, magnitude, interleaved, inverse, stream)
int rotary_apply(PyObject *const *a)
{
    const at::Tensor &q = tensor(a[1], "q"), &f = tensor(a[4], "frequencies"), &p = tensor(a[3], "positions");
    if (q.dim() != 3) refuse("q: want [tokens, heads, dim]");
    const at::ScalarType kind = q.scalar_type();
    if (kind != at::kFloat && kind != at::kBFloat16) refuse(std::string("q must be float32 or bfloat16, not ") + c10::toString(kind));
    if (p.scalar_type() != at::kInt && p.scalar_type() != at::kLong) refuse(std::string("positions must be int32 or int64, not ") + c10::toString(p.scalar_type()));
    dd_rotary r{};
    r.tokens = q.size(0);
    r.heads = q.size(1);
    r.dim = q.size(2);
    r.rotary_dim = 2 * (uint64_t)f.numel();
    if (a[2] != Py_None) {
        const at::Tensor &k = tensor(a[2], "k");
        if (k.dim() != 3) refuse("k: want [tokens, heads, dim]");
        r.kv_heads = k.size(1);
    }
    r.dtype = kind == at::kBFloat16 ? DD_BF16 : DD_F32;
    r.interleaved = truth(a[8]);
    r.inverse = truth(a[9]);
    r.positions_64 = p.scalar_type() == at::kLong;
    r.magnitude = (float)real(a[7]);
    if ((a[6] == Py_None) != (a[2] == Py_None)) refuse("k and k_out: want both or neither");
    const dd_heads x = heads_of(a[1], "q", r.tokens, r.heads, r.dim, kind), y = heads_of(a[2], "k", r.tokens, r.kv_heads, r.dim, kind),
                   xo = heads_of(a[5], "q_out", r.tokens, r.heads, r.dim, kind), yo = heads_of(a[6], "k_out", r.tokens, r.kv_heads, r.dim, kind);
    return dd_rotary_apply(context(a[0]), &r, &x, &y, &xo, &yo, vector(a[3], "positions", r.tokens, p.scalar_type()),
                           (const double *)vector(a[4], "frequencies", f.numel(), at::kDouble), pointer(a[10]));
}

// (q, k) and the settings -> attention
dd_attention attention_of(PyObject *q_, PyObject *k_, PyObject *offsets, PyObject *scale, PyObject *causal, PyObject *flags)
{
    const at::Tensor &q = tensor(q_, "q"), &k = tensor(k_, "k");
    if (q.dim() != 3 || k.dim() != 3) refuse("q and k: want [tokens, heads, dim]");
    dd_attention b{};
    b.tokens = q.size(0);
    b.heads = q.size(1);
    b.dim = q.size(2);
    b.kv_heads = k.size(1);
    if (offsets != Py_None) {
        const at::Tensor &o = tensor(offsets, "offsets");
        if (o.numel() < 1) refuse("offsets: want one more than there are sequences");
        b.sequences = o.numel() - 1;
        b.offsets = (const int32_t *)vector(offsets, "offsets", o.numel(), at::kInt);
    }
    b.scale = scale == Py_None ? 1.0f / std::sqrt((float)b.dim) : (float)real(scale);
    b.causal = truth(causal);
    const long long bits = integer(flags);
    b.flags = bits == (uint32_t)bits ? (uint32_t)bits : ~0u;
    return b;
}

// (ctx, q, k, v, o, lse, offsets, scale, causal, scratch, status, stream, flags)
int attention_forward(PyObject *const *a)
{
    const dd_attention b = attention_of(a[1], a[2], a[6], a[7], a[8], a[12]);
    const dd_heads q = heads_of(a[1], "q", b.tokens, b.heads, b.dim), k = heads_of(a[2], "k", b.tokens, b.kv_heads, b.dim),
                   v = heads_of(a[3], "v", b.tokens, b.kv_heads, b.dim), o = heads_of(a[4], "o", b.tokens, b.heads, b.dim);
    return dd_attention_forward(context(a[0]), &b, &q, &k, &v, &o, (float *)vector(a[5], "lse", b.heads * b.tokens, at::kFloat),
                                address(a[9], "scratch", dd_attention_scratch_bytes(&b, 0)), (int32_t *)address(a[10], "status", 4), pointer(a[11]));
}

// (ctx, q, k, v, o, lse, d_o, dq, dk, dv, offsets, scale, causal, scratch, status, stream, flags)
int attention_backward(PyObject *const *a)
{
    const dd_attention b = attention_of(a[1], a[2], a[10], a[11], a[12], a[16]);
    const dd_heads q = heads_of(a[1], "q", b.tokens, b.heads, b.dim), k = heads_of(a[2], "k", b.tokens, b.kv_heads, b.dim),
                   v = heads_of(a[3], "v", b.tokens, b.kv_heads, b.dim), o = heads_of(a[4], "o", b.tokens, b.heads, b.dim),
                   d_o = heads_of(a[6], "d_o", b.tokens, b.heads, b.dim), dq = heads_of(a[7], "dq", b.tokens, b.heads, b.dim),
                   dk = heads_of(a[8], "dk", b.tokens, b.kv_heads, b.dim), dv = heads_of(a[9], "dv", b.tokens, b.kv_heads, b.dim);
    return dd_attention_backward(context(a[0]), &b, &q, &k, &v, &o, (const float *)vector(a[5], "lse", b.heads * b.tokens, at::kFloat), &d_o, &dq,
                                 &dk, &dv, address(a[13], "scratch", dd_attention_scratch_bytes(&b, 1)), (int32_t *)address(a[14], "status", 4),
                                 pointer(a[15]));
}

// (hidden, weight, targets) -> loss and hidden
const void *loss_of(PyObject *hidden, PyObject *weight, PyObject *targets, PyObject *flags, dd_vocab_loss &l)
{
    const at::Tensor &h = tensor(hidden, "hidden"), &w = tensor(weight, "weight");
    if (h.dim() != 2 || w.dim() != 2) refuse("hidden and weight are matrices");
    l = dd_vocab_loss{};
    l.tokens = h.size(0);
    l.d = h.size(1);
    l.vocab = w.size(0);
    const long long bits = integer(flags);
    l.flags = bits == (uint32_t)bits ? (uint32_t)bits : ~0u;
    const void *x = matrix(hidden, "hidden", l.tokens, l.d, l.ld_hidden);
    l.weight = matrix(weight, "weight", l.vocab, l.d, l.ld_weight);
    l.targets = (const int64_t *)vector(targets, "targets", l.tokens, at::kLong);
    return x;
}

// (ctx, hidden, weight, targets, loss, lse, scratch, status, stream, flags)
int vocab_loss_forward(PyObject *const *a)
{
    dd_vocab_loss l;
    const void *x = loss_of(a[1], a[2], a[3], a[9], l);
    dd_ctx *ctx = context(a[0]);
    return dd_vocab_loss_forward(ctx, &l, x, (float *)vector(a[4], "loss", l.tokens, at::kFloat), (float *)vector(a[5], "lse", l.tokens, at::kFloat),
                                 address(a[6], "scratch", dd_vocab_loss_scratch_bytes(ctx, &l, 0)), (int32_t *)address(a[7], "status", 4), pointer(a[8]));
}

// (ctx, hidden, weight, targets, lse, dloss, dhidden, dweight, accumulate, scratch, status, stream, flags)
int vocab_loss_backward(PyObject *const *a)
{
    dd_vocab_loss l;
    const void *x = loss_of(a[1], a[2], a[3], a[12], l);
    dd_ctx *ctx = context(a[0]);
    const at::ScalarType kind = tensor(a[7], "dweight").scalar_type();
    if (kind != at::kFloat && kind != at::kBFloat16) refuse("dweight must be float32 or bfloat16");
    void *dx = matrix(a[6], "dhidden", l.tokens, l.d, l.ld_hidden), *dw = matrix(a[7], "dweight", l.vocab, l.d, l.ld_weight, kind);
    return dd_vocab_loss_backward(ctx, &l, x, (const float *)vector(a[4], "lse", l.tokens, at::kFloat),
                                  (const float *)vector(a[5], "dloss", l.tokens, at::kFloat), dx, dw, kind == at::kBFloat16 ? DD_BF16 : DD_F32,
                                  truth(a[8]), address(a[9], "scratch", dd_vocab_loss_scratch_bytes(ctx, &l, 1)), (int32_t *)address(a[10], "status", 4),
                                  pointer(a[11]));
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
                         ENTRY(gated_ffn_backward, 18), ENTRY(rotary_apply, 11), ENTRY(attention_forward, 13), ENTRY(attention_backward, 17),
                         ENTRY(vocab_loss_forward, 10), ENTRY(vocab_loss_backward, 13), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ddtorch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ddtorch() { return PyModule_Create(&module); }
