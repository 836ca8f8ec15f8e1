// The plain call of layer norm, rotary positions and distillation without the interpreter in between: every argument a tensor on the current device, the current stream,
// no gradient asked for.  Checks, allocation of the outputs and the call of the C entry point take 5 to 9 us here and 13 to 24 in Python, more than the kernels of a
// small call.  Anything else (another stream or device, no rows, an operand to copy, an argument to refuse, a graph that would be lost) is answered by None before
// anything happened, and layers.py and training.py do what it calls for; they own the documentation and the errors.  An int is the library's error code.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/psgd.h"

// What this was compiled against: build.py looks for it in the file, since nothing compiled against one torch may be loaded into another.
extern "C" __attribute__((used, visibility("default"))) const char psgd_call_built_for[] = PSGD_CALL_BUILT_FOR;

namespace {

using at::Tensor;

// nullptr where `o` is not a tensor of torch's own (None included: `present` says whether it is that)
const Tensor* tensor(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

struct Here {
    int device;
    bool grad;
    Here() : device(c10::cuda::current_device()), grad(at::GradMode::is_enabled()) {}
    // a tensor of the two types on this device; `watch`: whose gradient must not be asked for
    bool takes(const Tensor& t, bool watch) const {
        return t.is_cuda() && t.get_device() == device && t.layout() == at::kStrided && (t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16) &&
               !(watch && grad && t.requires_grad());
    }
};
int code(const Tensor& t) { return t.scalar_type() == at::kFloat ? PSGD_DT_F32 : PSGD_DT_BF16; }
bool vector(const Tensor& t, int64_t n, at::ScalarType type, int device) {
    return t.is_cuda() && t.get_device() == device && t.scalar_type() == type && t.dim() == 1 && t.size(0) == n && t.is_contiguous();
}
// rows of unit column stride that do not overlap; their stride
bool matrix(const Tensor& t, int64_t T, int64_t F, int64_t& ld) {
    if (t.dim() != 2 || t.size(0) != T || t.size(1) != F) return false;
    ld = T > 1 ? t.stride(0) : F;
    return ld >= F && (F == 1 || t.stride(1) == 1);
}
Tensor matrix_like(const Tensor& t, int64_t T, int64_t F) { return at::empty({T, F}, t.options()); }
PyObject* none() { Py_RETURN_NONE; }
// without the interpreter's lock while the outputs are allocated and the kernels launched (and with it again where the allocator throws)
struct Unlocked {
    PyThreadState* state;
    Unlocked() : state(PyEval_SaveThread()) {}
    ~Unlocked() { PyEval_RestoreThread(state); }
};
PyObject* wrap(const Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : none(); }
PyObject* tuple(std::initializer_list<PyObject*> items) {          // takes the references over
    PyObject* r = PyTuple_New((Py_ssize_t)items.size());
    Py_ssize_t i = 0;
    bool whole = r != nullptr;
    for (PyObject* o : items) {
        whole = whole && o;
        if (r) PyTuple_SET_ITEM(r, i++, o);
        else Py_XDECREF(o);
    }
    if (!whole) { Py_XDECREF(r); return nullptr; }
    return r;
}

// (x, weight, bias, residual, eps, center, keep) -> (y, x, mean, rstd, buffer of the checkpoint)
PyObject* norm_forward(PyObject*, PyObject* const* o, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    if (count != 7) return none();
    const Tensor *x = tensor(o[0]), *w = tensor(o[1]), *b = tensor(o[2]), *r = tensor(o[3]);
    if (!x || !w || (!b && o[2] != Py_None) || (!r && o[3] != Py_None) || !PyFloat_CheckExact(o[4]) || !PyBool_Check(o[5]) || !PyBool_Check(o[6]) || !x->is_cuda()) return none();
    const Here here;
    const double eps = PyFloat_AS_DOUBLE(o[4]);
    const bool center = o[5] == Py_True, keep = o[6] == Py_True;
    if (!here.takes(*x, true) || x->dim() != 2 || x->size(0) < 1 || x->size(1) < 1 || !(eps >= 0)) return none();
    const int64_t T = x->size(0), F = x->size(1);
    int64_t ldx, ldr = 0;
    if (!matrix(*x, T, F, ldx) || !here.takes(*w, true) || !vector(*w, F, w->scalar_type(), here.device)) return none();
    if (b && (!here.takes(*b, true) || !vector(*b, F, w->scalar_type(), here.device))) return none();
    if (r && (!here.takes(*r, true) || r->scalar_type() != x->scalar_type() || !matrix(*r, T, F, ldr))) return none();
    Tensor y, s, mean, rstd, kept;
    psgd_status e;
    {
        const Unlocked unlocked;
        const auto stats = x->options().dtype(at::kFloat);
        const int64_t groups = (F + 31) / 32;
        y = matrix_like(*x, T, F);
        if (r) s = matrix_like(*x, T, F);
        rstd = at::empty({T}, stats);
        if (center) mean = at::empty({T}, stats);
        if (keep) kept = at::empty({T * groups * 33}, stats.dtype(at::kByte));
        int8_t* q = keep ? (int8_t*)kept.data_ptr() : nullptr;
        e = psgd_norm_forward(x->data_ptr(), ldx, code(*x), r ? r->data_ptr() : nullptr, ldr, w->data_ptr(), b ? b->data_ptr() : nullptr, code(*w), (float)eps, center, T, F,
                              r ? s.data_ptr() : nullptr, F, y.data_ptr(), F, code(y), center ? (float*)mean.data_ptr() : nullptr, (float*)rstd.data_ptr(), q,
                              keep ? (uint8_t*)q + T * groups * 32 : nullptr, c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)here.device).stream());
    }
    if (e != PSGD_OK) return PyLong_FromLong(e);
    PyObject* sum = r ? wrap(s) : o[0];
    if (!r) Py_INCREF(sum);
    return tuple({wrap(y), sum, wrap(mean), wrap(rstd), wrap(kept)});
    END_HANDLE_TH_ERRORS
}

// (dy, x, weight, mean, rstd, d_x, bias) -> (d_x, d_weight, d_bias)
PyObject* norm_backward(PyObject*, PyObject* const* o, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    if (count != 7) return none();
    const Tensor *dy = tensor(o[0]), *x = tensor(o[1]), *w = tensor(o[2]), *mean = tensor(o[3]), *rstd = tensor(o[4]), *add = tensor(o[5]);
    if (!dy || !x || !w || (!mean && o[3] != Py_None) || !rstd || (!add && o[5] != Py_None) || !PyBool_Check(o[6]) || !x->is_cuda()) return none();
    const Here here;
    const bool bias = o[6] == Py_True;
    if (!here.takes(*x, false) || x->dim() != 2 || x->size(0) < 1 || x->size(1) < 1) return none();
    const int64_t T = x->size(0), F = x->size(1);
    int64_t ldx, lddy, lda = 0;
    if (!matrix(*x, T, F, ldx) || !here.takes(*dy, false) || !matrix(*dy, T, F, lddy) || (dy->scalar_type() != x->scalar_type() && x->scalar_type() != at::kFloat)) return none();
    if (!here.takes(*w, false) || !vector(*w, F, w->scalar_type(), here.device) || !vector(*rstd, T, at::kFloat, here.device)) return none();
    if ((mean && !vector(*mean, T, at::kFloat, here.device)) || (add && (!here.takes(*add, false) || add->scalar_type() != x->scalar_type() || !matrix(*add, T, F, lda)))) return none();
    Tensor dx, dw, db, ws;
    psgd_status e;
    {
        const Unlocked unlocked;
        // (what the query answers depends on these alone: the last answer of this thread)
        thread_local struct { int64_t T, F; int device; size_t bytes; } asked = {-1, -1, -1, 0};
        e = PSGD_OK;
        if (asked.T != T || asked.F != F || asked.device != here.device) {
            e = psgd_norm_workspace(T, F, &asked.bytes);
            asked.T = e == PSGD_OK ? T : -1;
            asked.F = F;
            asked.device = here.device;
        }
        if (e == PSGD_OK) {
            const auto sums = x->options().dtype(at::kFloat);
            ws = at::empty({(int64_t)asked.bytes}, sums.dtype(at::kByte));
            dx = matrix_like(*x, T, F);
            dw = at::empty({F}, sums);
            if (bias) db = at::empty({F}, sums);
            e = psgd_norm_backward(dy->data_ptr(), lddy, code(*dy), x->data_ptr(), ldx, code(*x), w->data_ptr(), code(*w), mean ? (const float*)mean->data_ptr() : nullptr,
                                   (const float*)rstd->data_ptr(), add ? add->data_ptr() : nullptr, lda, T, F, dx.data_ptr(), F, (float*)dw.data_ptr(),
                                   bias ? (float*)db.data_ptr() : nullptr, ws.data_ptr(), asked.bytes, c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)here.device).stream());
        }
    }
    if (e != PSGD_OK) return PyLong_FromLong(e);
    return tuple({wrap(dx), wrap(dw), wrap(db)});
    END_HANDLE_TH_ERRORS
}

bool heads(const Tensor& t, const Tensor* like) {
    return t.dim() == 3 && t.size(2) >= 2 && t.stride(2) == 1 && (!like || (t.scalar_type() == like->scalar_type() && t.size(0) == like->size(0) && t.size(2) == like->size(2)));
}
// tokens and heads in t's order, without gaps
Tensor heads_like(const Tensor& t) {
    const int64_t T = t.size(0), H = t.size(1), D = t.size(2);
    const bool tokens_first = t.stride(0) >= t.stride(1) || T == 1 || H == 1;
    return tokens_first ? at::empty({T, H, D}, t.options()) : at::empty({H, T, D}, t.options()).transpose(0, 1);
}

// (backward, q, k, positions, frequencies, layout's code, scale, in_place) -> (q, k)
PyObject* rotary(PyObject*, PyObject* const* o, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    if (count != 8) return none();
    const Tensor *q = tensor(o[1]), *k = tensor(o[2]), *at = tensor(o[3]), *f = tensor(o[4]);
    if (!PyBool_Check(o[0]) || !q || (!k && o[2] != Py_None) || !at || !f || !PyLong_CheckExact(o[5]) || !PyFloat_CheckExact(o[6]) || !PyBool_Check(o[7]) || !q->is_cuda()) return none();
    const Here here;
    const bool backward = o[0] == Py_True, in_place = o[7] == Py_True;
    const long layout = PyLong_AsLong(o[5]);
    const double scale = PyFloat_AS_DOUBLE(o[6]);
    if (!here.takes(*q, !backward) || !heads(*q, nullptr) || (k && (!here.takes(*k, !backward) || !heads(*k, q)))) return none();
    const int64_t T = q->size(0), D = q->size(2), H = q->size(1), K = k ? k->size(1) : 0;
    if (T < 1 || H < 1 || (k && K < 1) || f->dim() != 1 || f->size(0) < 1 || 2 * f->size(0) > D) return none();
    if (!vector(*at, T, at::kLong, here.device) || !vector(*f, f->size(0), at::kDouble, here.device) || (!backward && here.grad && f->requires_grad())) return none();
    Tensor oq, ok;
    psgd_status e;
    {
        const Unlocked unlocked;
        oq = in_place ? *q : heads_like(*q);
        if (k) ok = in_place ? *k : heads_like(*k);
        e = psgd_rotary(q->data_ptr(), q->stride(0), q->stride(1), H, oq.data_ptr(), oq.stride(0), oq.stride(1), k ? k->data_ptr() : nullptr, k ? k->stride(0) : 0, k ? k->stride(1) : 0, K,
                        k ? ok.data_ptr() : nullptr, k ? ok.stride(0) : 0, k ? ok.stride(1) : 0, (const int64_t*)at->data_ptr(), (const double*)f->data_ptr(), T, D, 2 * f->size(0),
                        (int)layout, backward, (float)scale, code(*q), c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)here.device).stream());
    }
    if (e != PSGD_OK) return PyLong_FromLong(e);
    const auto given = [&](int i, const Tensor& t) -> PyObject* {
        if (!in_place) return wrap(t);
        if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();      // whoever has saved it for its gradients has to know
        Py_INCREF(o[i]);
        return o[i];
    };
    return tuple({given(1, oq), k ? given(2, ok) : none()});
    END_HANDLE_TH_ERRORS
}

// an operand that the tensor cores' loads can read in place
bool operand(const Tensor& t, int64_t rows, int64_t cols, int64_t& ld) {
    return t.scalar_type() == at::kBFloat16 && matrix(t, rows, cols, ld) && ((uintptr_t)t.data_ptr() & 15) == 0 && (rows == 1 || ld % 8 == 0);
}

// (grad, hidden, weight, logits, index, temperature, token_weight) -> (loss, token_loss, lse[, d_hidden, d_weight])
PyObject* distill(PyObject*, PyObject* const* o, Py_ssize_t count) {
    HANDLE_TH_ERRORS
    if (count != 7) return none();
    const Tensor *h = tensor(o[1]), *w = tensor(o[2]), *z = tensor(o[3]), *index = tensor(o[4]), *weight = tensor(o[6]);
    if (!PyBool_Check(o[0]) || !h || !w || !z || !index || !PyFloat_CheckExact(o[5]) || (!weight && o[6] != Py_None) || !h->is_cuda()) return none();
    const Here here;
    const bool grad = o[0] == Py_True;
    const double tau = PyFloat_AS_DOUBLE(o[5]);
    if (!here.takes(*h, !grad) || !here.takes(*w, !grad) || !here.takes(*z, !grad) || h->dim() != 2 || w->dim() != 2 || z->dim() != 2 || index->dim() != 2) return none();
    const int64_t T = h->size(0), D = h->size(1), V = w->size(0), K = z->size(1);
    int64_t ldh, ldw, ldl, ldi;
    if (T < 1 || D < 1 || V < 1 || K < 1 || K > 1024 || !(tau >= 1e-3 && tau <= 1e3) || !operand(*h, T, D, ldh) || !operand(*w, V, D, ldw)) return none();
    if (!matrix(*z, T, K, ldl) || !index->is_cuda() || index->get_device() != here.device || index->scalar_type() != at::kLong || !matrix(*index, T, K, ldi)) return none();
    if (weight && (!here.takes(*weight, !grad) || !vector(*weight, T, at::kFloat, here.device))) return none();
    Tensor loss, token_loss, lse, dh, dw, ws;
    psgd_status e;
    {
        const Unlocked unlocked;
        thread_local struct { int64_t T, V, D, K; int grad, device; size_t bytes; } asked = {-1, 0, 0, 0, 0, 0, 0};
        e = PSGD_OK;
        if (asked.T != T || asked.V != V || asked.D != D || asked.K != K || asked.grad != grad || asked.device != here.device) {
            asked.T = -1;
            e = psgd_distill_workspace(T, V, D, K, grad, &asked.bytes);
            if (e == PSGD_OK) asked = {T, V, D, K, grad, here.device, asked.bytes};
        }
        if (e == PSGD_OK) {
            const auto floats = h->options().dtype(at::kFloat);
            ws = at::empty({(int64_t)asked.bytes}, floats.dtype(at::kByte));
            loss = at::empty({}, floats);
            token_loss = at::empty({T}, floats);
            lse = at::empty({T}, floats);
            const auto st = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)here.device).stream();
            const int64_t* at_index = (const int64_t*)index->data_ptr();
            const float* at_weight = weight ? (const float*)weight->data_ptr() : nullptr;
            float *at_loss = (float*)loss.data_ptr(), *at_token = (float*)token_loss.data_ptr(), *at_lse = (float*)lse.data_ptr();
            if (grad) {
                dh = matrix_like(*h, T, D);
                dw = matrix_like(*w, V, D);
                e = psgd_distill_grad(h->data_ptr(), ldh, w->data_ptr(), ldw, z->data_ptr(), ldl, code(*z), at_index, ldi, K, (float)tau, at_weight, T, V, D, at_loss, at_token, at_lse,
                                      dh.data_ptr(), D, dw.data_ptr(), D, nullptr, ws.data_ptr(), asked.bytes, st);
            } else {
                e = psgd_distill_loss(h->data_ptr(), ldh, w->data_ptr(), ldw, z->data_ptr(), ldl, code(*z), at_index, ldi, K, (float)tau, at_weight, T, V, D, at_loss, at_token, at_lse,
                                      nullptr, ws.data_ptr(), asked.bytes, st);
            }
        }
    }
    if (e != PSGD_OK) return PyLong_FromLong(e);
    return grad ? tuple({wrap(loss), wrap(token_loss), wrap(lse), wrap(dh), wrap(dw)}) : tuple({wrap(loss), wrap(token_loss), wrap(lse)});
    END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"distill", (PyCFunction)(void (*)(void))distill, METH_FASTCALL, nullptr},
                         {"norm_forward", (PyCFunction)(void (*)(void))norm_forward, METH_FASTCALL, nullptr},
                         {"norm_backward", (PyCFunction)(void (*)(void))norm_backward, METH_FASTCALL, nullptr},
                         {"rotary", (PyCFunction)(void (*)(void))rotary, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call(void) { return PyModule_Create(&module); }
