// The calls that a program makes at every decode step, cfgzip_decode_step and cfgzip_engine_step, and those of the
// pre-computation as functions of a CPython extension: what the binding does for them in Python (a dozen attribute look-ups
// and checks of tensors, the conversion of as many arguments for ctypes) took 5 us of the 8 that a step on small logits
// takes, and the kernel 3; and of the 44 us of signatures and classes of 4,096 tokens, 157 of displacements and classes of
// 32,000 and 165 of relations and classes of 32,000 it took 5, 6 and 4, as the GPU has nothing to do before the first launch.
// The calls of the vocabulary projection, of what is read from its logits and of the layer in front of it are here for the same reason, with results and workspace of their own only.
//
// Marshalling only, and only of the plain case: exact torch.Tensor objects in GPU memory of the types and layouts the
// binding asks for, the current stream.  For anything else a function returns None and has done nothing; the binding then
// goes its general way, which also says what is wrong.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <limits>

namespace {

using DecodeStep = int (*)(void *, int32_t, int32_t, int32_t, int64_t, const int32_t *, const int32_t *, int32_t,
                           int32_t *, const int32_t *, const int32_t *, int32_t *, void *);
using EngineStep = int (*)(void *, int32_t, int32_t, int32_t, int64_t, const int32_t *, int32_t, int32_t,
                           const int32_t *, const uint16_t *, const int32_t *, const int32_t *, int32_t *, int32_t *,
                           void *);
using Signatures = int (*)(const uint8_t *, const int64_t *, int32_t, const uint16_t *, int32_t, uint16_t *, uint64_t *,
                           uint64_t, void *, size_t, void *);
using BuildClasses = int (*)(const uint8_t *, const int64_t *, int32_t, const uint16_t *, int32_t, const uint16_t *,
                             const uint64_t *, void *, int32_t *, int32_t *, int32_t *, int32_t *, int32_t *, void *,
                             size_t, void *);
using Displacements = int (*)(const uint8_t *, const int64_t *, int32_t, const uint16_t *, const uint8_t *, const int32_t *,
                              const uint16_t *, int32_t, int32_t, int32_t, uint16_t *, int32_t, uint64_t *, int32_t *,
                              uint64_t, void *, size_t, void *);
using NfaSignatures = int (*)(const uint8_t *, const int64_t *, int32_t, const int32_t *, int32_t, int32_t *, uint64_t *,
                              uint64_t, void *);
DecodeStep g_decode_step = nullptr;
EngineStep g_engine_step = nullptr;
Signatures g_signatures = nullptr;
BuildClasses g_build_classes = nullptr;
Displacements g_displacements = nullptr;
NfaSignatures g_nfa_signatures = nullptr;

using HeadLossBytes = size_t (*)(int32_t, int32_t, int32_t, int32_t);
using HeadLoss = int (*)(const void *, int64_t, const void *, int64_t, int32_t, int32_t, int32_t, int32_t, const int32_t *,
                         const int32_t *, int32_t, const int32_t *, int32_t, float *, float *, void *, size_t, void *);
using HeadLossGrad = int (*)(const void *, int64_t, const void *, int64_t, int32_t, int32_t, int32_t, int32_t, const int32_t *,
                             const int32_t *, int32_t, const int32_t *, int32_t, const float *, const float *, void *, int64_t,
                             void *, int64_t, void *, size_t, void *);
using Mx4Quantize = int (*)(const void *, int32_t, int64_t, int32_t, int64_t, uint8_t *, uint8_t *, void *);
using Mx4Values = int (*)(const uint8_t *, const uint8_t *, int64_t, int32_t, void *, int32_t, int64_t, void *);
using Mx4LogitsBytes = size_t (*)(int32_t, int32_t, int32_t, int32_t, int32_t);
using Mx4Logits = int (*)(const void *, int32_t, int64_t, const uint8_t *, const uint8_t *, const uint8_t *, int32_t, int32_t,
                          int32_t, const int32_t *, int32_t, const int32_t *, int32_t, void *, int32_t, int64_t, void *, size_t,
                          void *);
HeadLossBytes g_head_loss_bytes = nullptr, g_head_loss_grad_bytes = nullptr;
HeadLoss g_head_loss = nullptr;
HeadLossGrad g_head_loss_grad = nullptr;
Mx4Quantize g_mx4_quantize = nullptr;
Mx4Values g_mx4_values = nullptr;
Mx4LogitsBytes g_mx4_logits_bytes = nullptr;
Mx4Logits g_mx4_logits = nullptr;

using TokenLogprobsBytes = size_t (*)(int32_t, int32_t, int32_t);
using TokenLogprobs = int (*)(const void *, int32_t, int32_t, int32_t, int64_t, const int32_t *, int32_t, double, const int32_t *, int32_t,
                              const int32_t *, int32_t, float *, float *, float *, int32_t, int32_t *, float *, void *, size_t, void *);
using TokenLogprobsGrad = int (*)(const void *, int32_t, int32_t, int32_t, int64_t, const int32_t *, int32_t, double, const int32_t *, int32_t,
                                  const int32_t *, int32_t, const float *, const float *, const float *, const float *, const float *, void *,
                                  int64_t, void *);
using HeadLayerBytes = size_t (*)(int32_t, int32_t, int32_t);
using HeadLayer = int (*)(const void *, int64_t, const void *, int64_t, int32_t, int32_t, int32_t, int32_t, const void *, int32_t, const void *,
                          int64_t, void *, int32_t, int64_t, void *, int64_t, void *, size_t, void *);
using HeadLayerGrad = int (*)(const void *, int64_t, const void *, int64_t, int32_t, int32_t, int32_t, int32_t, const void *, int32_t, int64_t,
                              const void *, int64_t, void *, int64_t, void *, int64_t, void *, void *, size_t, void *);
TokenLogprobsBytes g_token_logprobs_bytes = nullptr;
TokenLogprobs g_token_logprobs = nullptr;
TokenLogprobsGrad g_token_logprobs_grad = nullptr;
HeadLayerBytes g_head_layer_bytes = nullptr, g_head_layer_grad_bytes = nullptr;
HeadLayer g_head_layer = nullptr;
HeadLayerGrad g_head_layer_grad = nullptr;

constexpr int64_t kMost = std::numeric_limits<int32_t>::max();

// The tensor in GPU memory that `o` is, nothing else around it, or null.  (A tensor that a transformation wraps has no
// storage.)
const at::Tensor *plain(PyObject *o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.defined() || !t.is_cuda() || t.layout() != at::kStrided || !t.has_storage()) return nullptr;
    return &t;
}
const at::Tensor *plain(PyObject *o, at::ScalarType type) {
    const at::Tensor *t = plain(o);
    return t && t->scalar_type() == type && t->is_contiguous() ? t : nullptr;
}
// The same where None stands for "none": false if it is something else.
template <typename T>
bool plain_or_none(PyObject *o, at::ScalarType type, T **out) {
    *out = nullptr;
    if (o == Py_None) return true;
    const at::Tensor *t = plain(o, type);
    if (!t) return false;
    *out = static_cast<T *>(t->data_ptr());
    return true;
}
// An exact int of 1 .. 2^31 - 1, or 0.
int64_t small_int(PyObject *o) {
    if (!PyLong_CheckExact(o)) return 0;
    int overflow = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow || v < 1 || v > kMost ? 0 : v;
}

struct Logits {
    void *data;
    int32_t type, B, V;
    int64_t stride;
};
bool logits_of(PyObject *o, PyObject *V, Logits *out) {
    const at::Tensor *t = plain(o);
    if (!t || t->dim() != 2 || t->stride(1) != 1) return false;
    if (t->scalar_type() == at::kFloat) out->type = 0;
    else if (t->scalar_type() == at::kBFloat16) out->type = 1;
    else return false;
    const int64_t columns = V == Py_None ? t->size(1) : small_int(V);
    if (columns < 1 || columns > kMost || t->size(0) > kMost) return false;
    out->data = t->data_ptr();
    out->B = (int32_t)t->size(0);
    out->V = (int32_t)columns;
    out->stride = t->stride(0);
    return true;
}

// What the call returns, made before the launch, behind which nothing can fail any more: the tensor handed in, or the new
// one around `made`.  Null: a Python error is set.
PyObject *result_of(PyObject *given, const at::Tensor &made) {
    if (given == Py_None) return THPVariable_Wrap(made);
    Py_INCREF(given);
    return given;
}
// The same, or the status of the launch if it is not 0.
PyObject *finish(int rc, PyObject *result) {
    if (rc == 0) return result;
    Py_DECREF(result);
    return PyLong_FromLong(rc);
}
// Nothing has been launched: the general way meets the same error (one that a dispatch mode raises is also set in the
// interpreter) and says so.
PyObject *leave_it() {
    PyErr_Clear();
    Py_RETURN_NONE;
}

// (logits, cls_bits, class_of_token, C, tok, rep_of_class, tok_bits_out, rep_out, V)
PyObject *decode_step(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 9 || !g_decode_step || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Logits l;
    int32_t C = 0, *tok_bits = nullptr, *rep_out = nullptr;
    const int32_t *bits_p = nullptr, *cls_p = nullptr, *tok_p = nullptr, *rep_p = nullptr;
    void *stream = nullptr;
    PyObject *result = nullptr;
    try {
        if (!logits_of(args[0], args[8], &l)) Py_RETURN_NONE;
        C = (int32_t)small_int(args[3]);
        const at::Tensor *bits = plain(args[1], at::kInt), *cls = plain(args[2], at::kInt),
                         *tok = plain(args[4], at::kInt), *rep = plain(args[5], at::kInt);
        if (!C || !bits || !cls || !tok || !rep || !plain_or_none(args[6], at::kInt, &tok_bits) ||
            !plain_or_none(args[7], at::kInt, &rep_out))
            Py_RETURN_NONE;
        if (bits->dim() != 2 || bits->size(0) != l.B || bits->size(1) != ((int64_t)C + 31) / 32 || tok->numel() != l.B ||
            rep->numel() != C || cls->numel() != l.V)
            Py_RETURN_NONE;
        at::Tensor made;
        if (args[7] == Py_None) {
            made = tok->dim() == 1 ? at::empty_like(*tok) : at::empty({l.B}, tok->options());
            rep_out = static_cast<int32_t *>(made.data_ptr());
        }
        bits_p = static_cast<const int32_t *>(bits->data_ptr());
        cls_p = static_cast<const int32_t *>(cls->data_ptr());
        tok_p = static_cast<const int32_t *>(tok->data_ptr());
        rep_p = static_cast<const int32_t *>(rep->data_ptr());
        stream = c10::hip::getCurrentHIPStream().stream();
        result = result_of(args[7], made);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_decode_step(l.data, l.type, l.B, l.V, l.stride, bits_p, cls_p, C, tok_bits, tok_p, rep_p, rep_out, stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// (logits, state_mask, C, class_of_token, sig_rep, tok_prev, states_in, states_out, tok_bits_out, V)
PyObject *engine_step(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 10 || !g_engine_step || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Logits l;
    int32_t S = 0, C = 0, *tok_prev = nullptr, *out = nullptr, *tok_bits = nullptr;
    uint16_t *sig_rep = nullptr;
    const int32_t *mask_p = nullptr, *cls_p = nullptr, *in_p = nullptr;
    void *stream = nullptr;
    PyObject *result = nullptr;
    try {
        if (!logits_of(args[0], args[9], &l)) Py_RETURN_NONE;
        C = (int32_t)small_int(args[2]);
        const at::Tensor *mask = plain(args[1], at::kInt), *cls = plain(args[3], at::kInt), *in = plain(args[6], at::kInt);
        if (!C || !mask || mask->dim() < 1 || mask->size(0) > kMost || !cls || !in ||
            !plain_or_none(args[4], at::kUInt16, &sig_rep) || !plain_or_none(args[5], at::kInt, &tok_prev) ||
            !plain_or_none(args[7], at::kInt, &out) || !plain_or_none(args[8], at::kInt, &tok_bits))
            Py_RETURN_NONE;
        at::Tensor made;
        if (args[7] == Py_None) {
            made = at::empty_like(*in);
            out = static_cast<int32_t *>(made.data_ptr());
        }
        mask_p = static_cast<const int32_t *>(mask->data_ptr());
        cls_p = static_cast<const int32_t *>(cls->data_ptr());
        in_p = static_cast<const int32_t *>(in->data_ptr());
        S = (int32_t)mask->size(0);
        stream = c10::hip::getCurrentHIPStream().stream();
        result = result_of(args[7], made);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_engine_step(l.data, l.type, l.B, l.V, l.stride, mask_p, S, C, cls_p, sig_rep, tok_prev, in_p, out, tok_bits, stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// A vocabulary as every call of the pre-computation takes it.
struct Vocabulary {
    const uint8_t *bytes;  // null where every token is empty
    const int64_t *off;
    int32_t V;
    const at::Tensor *off_tensor;
};
bool vocabulary_of(PyObject *bytes, PyObject *off, Vocabulary *out) {
    const at::Tensor *b = plain(bytes, at::kByte), *o = plain(off, at::kLong);
    if (!b || !o || o->numel() < 2 || o->numel() - 1 > kMost) return false;
    out->bytes = b->numel() ? static_cast<const uint8_t *>(b->data_ptr()) : nullptr;
    out->off = static_cast<const int64_t *>(o->data_ptr());
    out->V = (int32_t)(o->numel() - 1);
    out->off_tensor = o;
    return true;
}
bool seed_of(PyObject *o, uint64_t *out) {
    if (!PyLong_CheckExact(o)) return false;
    *out = PyLong_AsUnsignedLongLongMask(o);
    return !PyErr_Occurred();
}
bool bool_of(PyObject *o, bool *out) {
    *out = o == Py_True;
    return o == Py_True || o == Py_False;
}
at::Tensor new_tensor(at::IntArrayRef sizes, at::ScalarType type, const Vocabulary &v) {
    return at::empty(sizes, v.off_tensor->options().dtype(type));
}
// The tensor that a result is: the one handed in, else a new one.  False: not a plain one.
template <typename T>
bool result_in(PyObject *given, at::IntArrayRef sizes, at::ScalarType type, const Vocabulary &v, at::Tensor *made, T **data) {
    if (!plain_or_none(given, type, data)) return false;
    if (given == Py_None) {
        *made = new_tensor(sizes, type, v);
        *data = static_cast<T *>(made->data_ptr());
    }
    return true;
}
// References that are given up unless they are handed on.
struct Held {
    PyObject *o = nullptr;
    explicit Held(PyObject *x) : o(x) {}
    Held(const Held &) = delete;
    Held &operator=(const Held &) = delete;
    ~Held() { Py_XDECREF(o); }
};

// (tok_bytes, tok_off, table, want_sig, want_hash, hash_seed, sig_out, hash_out, workspace)
PyObject *signatures(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 9 || !g_signatures || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Vocabulary v;
    bool want_sig = false, want_hash = false;
    uint64_t seed = 0, *hash = nullptr;
    uint16_t *sig = nullptr;
    const uint16_t *table_p = nullptr;
    void *ws = nullptr, *stream = nullptr;
    int64_t S = 0, ws_bytes = 0;
    PyObject *result = nullptr;
    try {
        const at::Tensor *table = plain(args[2], at::kUInt16), *workspace = plain(args[8]);
        if (!vocabulary_of(args[0], args[1], &v) || !table || table->dim() < 1 || table->size(0) < 1 || table->size(0) > kMost ||
            !bool_of(args[3], &want_sig) || !bool_of(args[4], &want_hash) || !seed_of(args[5], &seed) || !workspace)
            return leave_it();
        S = table->size(0);
        at::Tensor made_sig, made_hash;
        if (want_sig ? !result_in(args[6], {v.V, S}, at::kUInt16, v, &made_sig, &sig) : !plain_or_none(args[6], at::kUInt16, &sig))
            Py_RETURN_NONE;
        if (want_hash ? !result_in(args[7], {v.V}, at::kLong, v, &made_hash, &hash) : !plain_or_none(args[7], at::kLong, &hash))
            Py_RETURN_NONE;
        table_p = static_cast<const uint16_t *>(table->data_ptr());
        ws = workspace->data_ptr();
        ws_bytes = workspace->numel();
        stream = c10::hip::getCurrentHIPStream().stream();
        const Held a(made_sig.defined() ? THPVariable_Wrap(made_sig) : Py_NewRef(args[6]));
        const Held b(made_hash.defined() ? THPVariable_Wrap(made_hash) : Py_NewRef(args[7]));
        if (a.o && b.o) result = PyTuple_Pack(2, a.o, b.o);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_signatures(v.bytes, v.off, v.V, table_p, (int32_t)S, sig, hash, seed, ws, (size_t)ws_bytes, stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// (tok_bytes, tok_off, table, sig, hash, class_of_token, rep_of_class, workspace, signatures_workspace): a tuple of the
// first two results, whole, and the two counts
PyObject *build_classes(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 9 || !g_build_classes || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Vocabulary v;
    uint16_t *table = nullptr, *sig = nullptr;
    uint8_t *sig_ws = nullptr;
    int32_t *cls = nullptr, *rep = nullptr;
    const uint64_t *hash = nullptr;
    void *ws = nullptr, *stream = nullptr;
    int64_t S = 0, ws_bytes = 0;
    PyObject *first = nullptr, *second = nullptr;
    try {
        const at::Tensor *h = plain(args[4], at::kLong), *workspace = plain(args[7]);
        if (!vocabulary_of(args[0], args[1], &v) || !plain_or_none(args[2], at::kUInt16, &table) ||
            !plain_or_none(args[3], at::kUInt16, &sig) || !h || !workspace || !plain_or_none(args[8], at::kByte, &sig_ws))
            Py_RETURN_NONE;
        if (args[2] != Py_None) {
            const at::Tensor &t = THPVariable_Unpack(args[2]);
            S = t.dim() >= 1 ? t.size(0) : 0;
        } else if (args[3] != Py_None) {
            const at::Tensor &t = THPVariable_Unpack(args[3]);
            S = t.dim() >= 2 ? t.size(1) : 0;
        }
        if (S < 1 || S > kMost) Py_RETURN_NONE;
        at::Tensor made_cls, made_rep;
        if (!result_in(args[5], {v.V}, at::kInt, v, &made_cls, &cls) || !result_in(args[6], {v.V}, at::kInt, v, &made_rep, &rep))
            Py_RETURN_NONE;
        hash = static_cast<const uint64_t *>(h->data_ptr());
        ws = workspace->data_ptr();
        ws_bytes = workspace->numel();
        stream = c10::hip::getCurrentHIPStream().stream();
        first = made_cls.defined() ? THPVariable_Wrap(made_cls) : Py_NewRef(args[5]);
        second = made_rep.defined() ? THPVariable_Wrap(made_rep) : Py_NewRef(args[6]);
    } catch (...) {
    }
    if (!first || !second) {
        Py_XDECREF(first);
        Py_XDECREF(second);
        return leave_it();
    }
    int rc = 0;
    int32_t C = 0, collisions = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_build_classes(v.bytes, v.off, v.V, table, (int32_t)S, sig, hash, sig_ws, cls, rep, nullptr, &C, &collisions, ws,
                         (size_t)ws_bytes, stream);
    Py_END_ALLOW_THREADS
    if (rc != 0) {
        Py_DECREF(first);
        Py_DECREF(second);
        return PyLong_FromLong(rc);
    }
    return Py_BuildValue("(NNii)", first, second, (int)C, (int)collisions);
}

// (tok_bytes, tok_off, prod_head, prod_byte, prod_body_off, prod_body, N, row_len, hash_seed, workspace)
PyObject *displacements(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 10 || !g_displacements || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Vocabulary v;
    uint64_t seed = 0, *hash = nullptr;
    const uint16_t *head_p = nullptr, *body_p = nullptr;
    const uint8_t *byte_p = nullptr;
    const int32_t *off_p = nullptr;
    uint16_t *rows = nullptr;
    int32_t *status = nullptr;
    void *ws = nullptr, *stream = nullptr;
    int64_t P = 0, total = 0, N = 0, row_len = 0, ws_bytes = 0;
    PyObject *result = nullptr;
    try {
        const at::Tensor *head = plain(args[2], at::kUInt16), *byte = plain(args[3], at::kByte), *off = plain(args[4], at::kInt),
                         *body = plain(args[5], at::kUInt16), *workspace = plain(args[9]);
        N = small_int(args[6]);
        row_len = small_int(args[7]);
        if (!vocabulary_of(args[0], args[1], &v) || !head || !byte || !off || !body || !workspace || !N || !row_len ||
            !seed_of(args[8], &seed) || head->numel() < 1 || head->numel() >= kMost || off->numel() != head->numel() + 1 ||
            body->numel() > kMost)
            return leave_it();
        P = head->numel();
        total = body->numel();
        const at::Tensor made_rows = new_tensor({v.V, row_len}, at::kUInt16, v), made_hash = new_tensor({v.V}, at::kLong, v),
                         made_status = new_tensor({v.V}, at::kInt, v);
        rows = static_cast<uint16_t *>(made_rows.data_ptr());
        hash = static_cast<uint64_t *>(made_hash.data_ptr());
        status = static_cast<int32_t *>(made_status.data_ptr());
        head_p = static_cast<const uint16_t *>(head->data_ptr());
        byte_p = static_cast<const uint8_t *>(byte->data_ptr());
        off_p = static_cast<const int32_t *>(off->data_ptr());
        body_p = total ? static_cast<const uint16_t *>(body->data_ptr()) : nullptr;
        ws = workspace->data_ptr();
        ws_bytes = workspace->numel();
        stream = c10::hip::getCurrentHIPStream().stream();
        const Held a(THPVariable_Wrap(made_rows)), b(THPVariable_Wrap(made_hash)), c(THPVariable_Wrap(made_status));
        if (a.o && b.o && c.o) result = PyTuple_Pack(3, a.o, b.o, c.o);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_displacements(v.bytes, v.off, v.V, head_p, byte_p, off_p, body_p, (int32_t)total, (int32_t)P, (int32_t)N, rows,
                         (int32_t)row_len, hash, status, seed, ws, (size_t)ws_bytes, stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// (tok_bytes, tok_off, nfa, want_hash, hash_seed)
PyObject *nfa_signatures(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 5 || !g_nfa_signatures || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Vocabulary v;
    bool want_hash = false;
    uint64_t seed = 0, *hash = nullptr;
    const int32_t *nfa_p = nullptr;
    int32_t *rel = nullptr;
    void *stream = nullptr;
    int64_t S = 0;
    PyObject *result = nullptr;
    try {
        const at::Tensor *nfa = plain(args[2], at::kInt);
        if (!vocabulary_of(args[0], args[1], &v) || !nfa || nfa->dim() != 3 || nfa->size(0) != 256 || nfa->size(1) < 1 ||
            nfa->size(1) > kMost - 31 || nfa->size(2) != (nfa->size(1) + 31) / 32 || !bool_of(args[3], &want_hash) ||
            !seed_of(args[4], &seed))
            return leave_it();
        S = nfa->size(1);
        const at::Tensor made_rel = new_tensor({v.V, S, nfa->size(2)}, at::kInt, v);
        const at::Tensor made_hash = want_hash ? new_tensor({v.V}, at::kLong, v) : at::Tensor();
        rel = static_cast<int32_t *>(made_rel.data_ptr());
        if (want_hash) hash = static_cast<uint64_t *>(made_hash.data_ptr());
        nfa_p = static_cast<const int32_t *>(nfa->data_ptr());
        stream = c10::hip::getCurrentHIPStream().stream();
        const Held a(THPVariable_Wrap(made_rel)), b(want_hash ? THPVariable_Wrap(made_hash) : Py_NewRef(Py_None));
        if (a.o && b.o) result = PyTuple_Pack(2, a.o, b.o);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_nfa_signatures(v.bytes, v.off, v.V, nfa_p, (int32_t)S, rel, hash, seed, stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// ---------------------------------------------------------------- the vocabulary projection

// A matrix whose rows are any distance apart, types by the library's numbers.
struct Matrix {
    const at::Tensor *t;
    void *data;
    int64_t stride;
    int32_t type, rows, columns;
};
constexpr at::ScalarType kTypes[] = {at::kFloat, at::kBFloat16, at::kHalf};
bool matrix_of(PyObject *o, Matrix *out) {
    const at::Tensor *t = plain(o);
    if (!t || t->dim() != 2) return false;
    out->type = -1;
    for (int i = 0; i < 3; ++i)
        if (t->scalar_type() == kTypes[i]) out->type = i;
    const int64_t rows = t->size(0), columns = t->size(1);
    if (out->type < 0 || rows > kMost || columns < 1 || columns > kMost || (columns > 1 && t->stride(1) != 1)) return false;
    out->stride = rows > 1 || t->stride(0) > columns ? t->stride(0) : columns;
    if (out->stride < columns) return false;
    out->t = t;
    out->data = t->data_ptr();
    out->rows = (int32_t)rows;
    out->columns = (int32_t)columns;
    return true;
}
// Codes and scales of rows of 4-bit values.
struct Blocks {
    const at::Tensor *t;
    const uint8_t *codes, *scales;
    int32_t rows, blocks;
};
bool blocks_of(PyObject *codes, PyObject *scales, Blocks *out) {
    const at::Tensor *c = plain(codes, at::kByte), *s = plain(scales, at::kByte);
    if (!c || !s || c->dim() != 2 || s->dim() != 2 || c->size(0) != s->size(0) || c->size(1) != 16 * s->size(1) || s->size(0) > kMost ||
        s->size(1) < 1 || s->size(1) > kMost / 32 || c->device() != s->device())
        return false;
    out->t = c;
    out->codes = static_cast<const uint8_t *>(c->data_ptr());
    out->scales = static_cast<const uint8_t *>(s->data_ptr());
    out->rows = (int32_t)s->size(0);
    out->blocks = (int32_t)s->size(1);
    return true;
}
// Masks of `rows` rows over V tokens: (bits, class_of_token, C), each None (C: 0) where there is none.
struct Masks {
    const int32_t *bits = nullptr, *class_of_token = nullptr;
    int32_t kind = 2, C = 0;
};
bool masks_of(PyObject *bits, PyObject *class_of_token, PyObject *C, int64_t rows, int64_t V, const at::Tensor &beside, Masks *out) {
    if (bits == Py_None) return class_of_token == Py_None && PyLong_CheckExact(C) && PyLong_AsLong(C) == 0;
    const at::Tensor *b = plain(bits, at::kInt);
    if (!b || b->dim() != 2 || b->size(0) != rows || b->device() != beside.device()) return false;
    out->kind = 0;
    int64_t n = V;
    if (class_of_token != Py_None) {
        const at::Tensor *c = plain(class_of_token, at::kInt);
        n = small_int(C);
        if (!c || !n || c->numel() != V || c->device() != beside.device()) return false;
        out->class_of_token = static_cast<const int32_t *>(c->data_ptr());
        out->kind = 1;
        out->C = (int32_t)n;
    }
    out->bits = static_cast<const int32_t *>(b->data_ptr());
    return b->size(1) == (n + 31) / 32;
}
// n values of `type` beside a tensor, in a row
void *vector_of(PyObject *o, at::ScalarType type, int64_t n, const at::Tensor &beside) {
    const at::Tensor *t = plain(o, type);
    return t && t->numel() == n && t->device() == beside.device() ? t->data_ptr() : nullptr;
}
at::Tensor workspace_of(size_t bytes, const at::Tensor &beside) {
    return at::empty({(int64_t)(bytes > 256 ? bytes : 256)}, beside.options().dtype(at::kByte));
}

// (hidden, weight, target, bits, class_of_token, C[, lse, grad_loss, want_hidden, want_weight]): what the loss and its gradients
// share.  No rows are left to the general way.
struct Head {
    Matrix hidden, weight;
    const int32_t *target;
    Masks masks;
};
bool head_of(PyObject *const *args, Head *out) {
    if (!matrix_of(args[0], &out->hidden) || !matrix_of(args[1], &out->weight) || out->weight.type == 0 ||
        out->hidden.type != out->weight.type || out->hidden.columns != out->weight.columns || out->hidden.rows < 1 ||
        out->hidden.t->device() != out->weight.t->device())
        return false;
    out->target = static_cast<const int32_t *>(vector_of(args[2], at::kInt, out->hidden.rows, *out->weight.t));
    return out->target && masks_of(args[3], args[4], args[5], out->hidden.rows, out->weight.rows, *out->weight.t, &out->masks);
}

PyObject *head_loss(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 6 || !g_head_loss || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Head h{};
    float *loss = nullptr, *lse = nullptr;
    void *ws = nullptr, *stream = nullptr;
    at::Tensor workspace;
    PyObject *result = nullptr;
    try {
        if (!head_of(args, &h)) return leave_it();
        const auto options = h.weight.t->options().dtype(at::kFloat);
        const at::Tensor made_loss = at::empty({h.hidden.rows}, options), made_lse = at::empty({h.hidden.rows}, options);
        workspace = workspace_of(g_head_loss_bytes(h.hidden.rows, h.weight.rows, h.weight.columns, h.masks.kind), *h.weight.t);
        loss = static_cast<float *>(made_loss.data_ptr());
        lse = static_cast<float *>(made_lse.data_ptr());
        ws = workspace.data_ptr();
        stream = c10::hip::getCurrentHIPStream().stream();
        const Held a(THPVariable_Wrap(made_loss)), b(THPVariable_Wrap(made_lse));
        if (a.o && b.o) result = PyTuple_Pack(2, a.o, b.o);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_head_loss(h.hidden.data, h.hidden.stride, h.weight.data, h.weight.stride, h.weight.type, h.hidden.rows, h.weight.rows,
                     h.weight.columns, h.target, h.masks.bits, h.masks.kind, h.masks.class_of_token, h.masks.C, loss, lse, ws,
                     (size_t)workspace.numel(), stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

PyObject *head_loss_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 10 || !g_head_loss_grad || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Head h{};
    const float *lse = nullptr, *grad_loss = nullptr;
    void *gh = nullptr, *gw = nullptr, *ws = nullptr, *stream = nullptr;
    bool want_hidden = false, want_weight = false;
    at::Tensor workspace;
    PyObject *result = nullptr;
    try {
        if (!head_of(args, &h) || !bool_of(args[8], &want_hidden) || !bool_of(args[9], &want_weight) || (!want_hidden && !want_weight))
            return leave_it();
        lse = static_cast<const float *>(vector_of(args[6], at::kFloat, h.hidden.rows, *h.weight.t));
        grad_loss = static_cast<const float *>(vector_of(args[7], at::kFloat, h.hidden.rows, *h.weight.t));
        if (!lse || !grad_loss) Py_RETURN_NONE;
        at::Tensor made_gh, made_gw;
        if (want_hidden) {
            made_gh = at::empty({h.hidden.rows, h.weight.columns}, h.weight.t->options());
            gh = made_gh.data_ptr();
        }
        if (want_weight) {
            made_gw = at::empty({h.weight.rows, h.weight.columns}, h.weight.t->options());
            gw = made_gw.data_ptr();
        }
        workspace = workspace_of(g_head_loss_grad_bytes(h.hidden.rows, h.weight.rows, h.weight.columns, h.masks.kind), *h.weight.t);
        ws = workspace.data_ptr();
        stream = c10::hip::getCurrentHIPStream().stream();
        const Held a(want_hidden ? THPVariable_Wrap(made_gh) : Py_NewRef(Py_None)), b(want_weight ? THPVariable_Wrap(made_gw) : Py_NewRef(Py_None));
        if (a.o && b.o) result = PyTuple_Pack(2, a.o, b.o);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_head_loss_grad(h.hidden.data, h.hidden.stride, h.weight.data, h.weight.stride, h.weight.type, h.hidden.rows, h.weight.rows,
                          h.weight.columns, h.target, h.masks.bits, h.masks.kind, h.masks.class_of_token, h.masks.C, lse, grad_loss, gh,
                          gh ? h.weight.columns : 0, gw, gw ? h.weight.columns : 0, ws, (size_t)workspace.numel(), stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// (x)
PyObject *mx4_quantize(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 1 || !g_mx4_quantize || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Matrix x{};
    uint8_t *codes = nullptr, *scales = nullptr;
    void *stream = nullptr;
    PyObject *result = nullptr;
    try {
        if (!matrix_of(args[0], &x)) Py_RETURN_NONE;
        const int64_t nb = ((int64_t)x.columns + 31) / 32;
        const auto options = x.t->options().dtype(at::kByte);
        const at::Tensor made_codes = at::empty({x.rows, 16 * nb}, options), made_scales = at::empty({x.rows, nb}, options);
        codes = static_cast<uint8_t *>(made_codes.data_ptr());
        scales = static_cast<uint8_t *>(made_scales.data_ptr());
        stream = c10::hip::getCurrentHIPStream().stream();
        const Held a(THPVariable_Wrap(made_codes)), b(THPVariable_Wrap(made_scales));
        if (a.o && b.o) result = PyTuple_Pack(2, a.o, b.o);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_mx4_quantize(x.data, x.type, x.rows, x.columns, x.stride, codes, scales, stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// The type that an argument names by the library's number, 0 .. last, or -1
int32_t type_of(PyObject *o, long last) {
    if (!PyLong_CheckExact(o)) return -1;
    const long v = PyLong_AsLong(o);
    return v < 0 || v > last ? -1 : (int32_t)v;
}

// (codes, scales, K, the result's type)
PyObject *mx4_values(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 4 || !g_mx4_values || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Blocks w{};
    int32_t K = 0, type = -1;
    void *out = nullptr, *stream = nullptr;
    PyObject *result = nullptr;
    try {
        K = (int32_t)small_int(args[2]);
        type = type_of(args[3], 2);
        if (!blocks_of(args[0], args[1], &w) || !K || type < 0 || ((int64_t)K + 31) / 32 != w.blocks) return leave_it();
        const at::Tensor made = at::empty({w.rows, K}, w.t->options().dtype(kTypes[type]));
        out = made.data_ptr();
        stream = c10::hip::getCurrentHIPStream().stream();
        result = THPVariable_Wrap(made);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_mx4_values(w.codes, w.scales, w.rows, K, out, type, K, stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// (hidden, codes, scales, hidden_scales, the result's type, bits, class_of_token, C)
PyObject *mx4_logits(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 8 || !g_mx4_logits || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Blocks w{}, x4{};
    Matrix x{};
    Masks m;
    const void *hidden = nullptr;
    int64_t stride = 0;
    int32_t kind = 3, B = 0, K = 0, type = -1;
    void *out = nullptr, *ws = nullptr, *stream = nullptr;
    size_t bytes = 0;
    at::Tensor workspace;
    PyObject *result = nullptr;
    try {
        type = type_of(args[4], 1);
        if (!blocks_of(args[1], args[2], &w) || type < 0 || w.rows < 1) return leave_it();
        if (args[3] == Py_None) {
            if (!matrix_of(args[0], &x) || x.type == 0 || ((int64_t)x.columns + 31) / 32 != w.blocks || x.t->device() != w.t->device())
                Py_RETURN_NONE;
            hidden = x.data, stride = x.stride, kind = x.type, B = x.rows, K = x.columns;
        } else {
            if (!blocks_of(args[0], args[3], &x4) || x4.blocks != w.blocks || x4.t->device() != w.t->device()) Py_RETURN_NONE;
            hidden = x4.codes, stride = 16 * (int64_t)w.blocks, B = x4.rows, K = 32 * w.blocks;
        }
        if (B < 1 || !masks_of(args[5], args[6], args[7], B, w.rows, *w.t, &m)) return leave_it();
        const at::Tensor made = at::empty({B, w.rows}, w.t->options().dtype(kTypes[type]));
        out = made.data_ptr();
        bytes = g_mx4_logits_bytes(kind, B, w.rows, K, m.kind);
        if (bytes) {
            workspace = workspace_of(bytes, *w.t);
            ws = workspace.data_ptr();
            bytes = (size_t)workspace.numel();
        }
        stream = c10::hip::getCurrentHIPStream().stream();
        result = THPVariable_Wrap(made);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_mx4_logits(hidden, kind, stride, x4.scales, w.codes, w.scales, B, w.rows, K, m.bits, m.kind, m.class_of_token, m.C, out, type,
                      w.rows, ws, bytes, stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// The addresses of the vocabulary projection's calls: cfgzip_head_loss_workspace_bytes, cfgzip_head_loss,
// cfgzip_head_loss_grad_workspace_bytes, cfgzip_head_loss_grad, cfgzip_mx4_quantize, cfgzip_mx4_values,
// cfgzip_mx4_logits_workspace_bytes and cfgzip_mx4_logits
PyObject *connect_head(PyObject *, PyObject *const *args, Py_ssize_t n) {
    void *at[8];
    if (n != 8) {
        PyErr_SetString(PyExc_TypeError, "connect_head takes eight addresses");
        return nullptr;
    }
    for (int i = 0; i < 8; ++i) at[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    g_head_loss_bytes = reinterpret_cast<HeadLossBytes>(at[0]);
    g_head_loss = reinterpret_cast<HeadLoss>(at[1]);
    g_head_loss_grad_bytes = reinterpret_cast<HeadLossBytes>(at[2]);
    g_head_loss_grad = reinterpret_cast<HeadLossGrad>(at[3]);
    g_mx4_quantize = reinterpret_cast<Mx4Quantize>(at[4]);
    g_mx4_values = reinterpret_cast<Mx4Values>(at[5]);
    g_mx4_logits_bytes = reinterpret_cast<Mx4LogitsBytes>(at[6]);
    g_mx4_logits = reinterpret_cast<Mx4Logits>(at[7]);
    Py_RETURN_NONE;
}

// ---------------------------------------------------------------- log probabilities, the layer in front of the projection

// On the device whose current stream a call takes; others are left to the general way.
bool here(const at::Tensor &t) { return t.device().index() == c10::hip::current_device(); }

// (logits, tokens, .., temperature, bits, class_of_token, C): what log probabilities and their gradient share.  No rows are left to the general way.
struct Score {
    Matrix logits;
    const at::Tensor *tokens = nullptr;  // none: null
    int32_t n = 0;
    double temperature = 0.0;
    Masks masks;
    const int32_t *ids() const { return tokens ? static_cast<const int32_t *>(tokens->data_ptr()) : nullptr; }
};
bool score_of(PyObject *logits, PyObject *tokens, PyObject *temperature, PyObject *const *masks, Score *out) {
    if (!matrix_of(logits, &out->logits) || out->logits.rows < 1 || !here(*out->logits.t) || !PyFloat_CheckExact(temperature)) return false;
    out->temperature = PyFloat_AS_DOUBLE(temperature);
    if (tokens != Py_None) {
        const at::Tensor *t = plain(tokens, at::kInt);
        if (!t || (t->dim() != 1 && t->dim() != 2) || t->size(0) != out->logits.rows || t->device() != out->logits.t->device()) return false;
        const int64_t n = t->dim() == 1 ? 1 : t->size(1);
        if (n < 1 || n > kMost) return false;
        out->tokens = t;
        out->n = (int32_t)n;
    }
    return masks_of(masks[0], masks[1], masks[2], out->logits.rows, out->logits.columns, *out->logits.t, &out->masks);
}
// n values beside a tensor, or None
bool vector_or_none(PyObject *o, int64_t n, const at::Tensor &beside, const float **out) {
    *out = nullptr;
    if (o == Py_None) return true;
    *out = static_cast<const float *>(vector_of(o, at::kFloat, n, beside));
    return *out != nullptr;
}

// (logits, tokens, top, temperature, bits, class_of_token, C)
PyObject *token_logprobs(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 7 || !g_token_logprobs || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Score s{};
    float *logprob = nullptr, *entropy = nullptr, *stats = nullptr, *top_logprobs = nullptr;
    int32_t *top_tokens = nullptr, top = 0;
    void *ws = nullptr, *stream = nullptr;
    size_t bytes = 0;
    at::Tensor workspace;
    PyObject *result = nullptr;
    try {
        if (!score_of(args[0], args[1], args[3], args + 4, &s) || !PyLong_CheckExact(args[2])) return leave_it();
        const long k = PyLong_AsLong(args[2]);
        if (k < 0 || k > 64) return leave_it();
        top = (int32_t)k;
        const auto floats = s.logits.t->options().dtype(at::kFloat), ints = s.logits.t->options().dtype(at::kInt);
        const int64_t N = s.logits.rows;
        at::Tensor made_logprob, made_tokens, made_top;
        const at::Tensor made_entropy = at::empty({N}, floats), made_stats = at::empty({N, 2}, floats);
        entropy = static_cast<float *>(made_entropy.data_ptr());
        stats = static_cast<float *>(made_stats.data_ptr());
        if (s.tokens) {
            made_logprob = at::empty(s.tokens->sizes(), floats);
            logprob = static_cast<float *>(made_logprob.data_ptr());
        }
        if (top) {
            made_tokens = at::empty({N, top}, ints);
            made_top = at::empty({N, top}, floats);
            top_tokens = static_cast<int32_t *>(made_tokens.data_ptr());
            top_logprobs = static_cast<float *>(made_top.data_ptr());
        }
        bytes = g_token_logprobs_bytes(s.logits.rows, s.logits.columns, top);
        if (bytes) {
            workspace = workspace_of(bytes, *s.logits.t);
            ws = workspace.data_ptr();
            bytes = (size_t)workspace.numel();
        }
        stream = c10::hip::getCurrentHIPStream().stream();
        const Held a(s.tokens ? THPVariable_Wrap(made_logprob) : Py_NewRef(Py_None)), b(THPVariable_Wrap(made_entropy)),
            c(THPVariable_Wrap(made_stats)), d(top ? THPVariable_Wrap(made_tokens) : Py_NewRef(Py_None)),
            e(top ? THPVariable_Wrap(made_top) : Py_NewRef(Py_None));
        if (a.o && b.o && c.o && d.o && e.o) result = PyTuple_Pack(5, a.o, b.o, c.o, d.o, e.o);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_token_logprobs(s.logits.data, s.logits.type, s.logits.rows, s.logits.columns, s.logits.stride, s.ids(), s.n, s.temperature,
                          s.masks.bits, s.masks.kind, s.masks.class_of_token, s.masks.C, logprob, entropy, stats, top, top_tokens, top_logprobs,
                          ws, bytes, stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// (logits, tokens, logprob, stats, grad_logprob, entropy, grad_entropy, temperature, bits, class_of_token, C)
PyObject *token_logprobs_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 11 || !g_token_logprobs_grad || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Score s{};
    const float *logprob = nullptr, *stats = nullptr, *grad_logprob = nullptr, *entropy = nullptr, *grad_entropy = nullptr;
    void *out = nullptr, *stream = nullptr;
    PyObject *result = nullptr;
    try {
        if (!score_of(args[0], args[1], args[7], args + 8, &s)) return leave_it();
        const at::Tensor &beside = *s.logits.t;
        const int64_t N = s.logits.rows;
        stats = static_cast<const float *>(vector_of(args[3], at::kFloat, 2 * N, beside));
        if (!stats || !vector_or_none(args[6], N, beside, &grad_entropy) ||
            !vector_or_none(grad_entropy ? args[5] : Py_None, N, beside, &entropy) || (grad_entropy && !entropy))
            return leave_it();
        if (s.tokens) {
            logprob = static_cast<const float *>(vector_of(args[2], at::kFloat, N * s.n, beside));
            grad_logprob = static_cast<const float *>(vector_of(args[4], at::kFloat, N * s.n, beside));
            if (!logprob || !grad_logprob || plain(args[2])->sizes() != s.tokens->sizes() || plain(args[4])->sizes() != s.tokens->sizes())
                return leave_it();
        }
        const at::Tensor made = at::empty({N, s.logits.columns}, beside.options());
        out = made.data_ptr();
        stream = c10::hip::getCurrentHIPStream().stream();
        result = THPVariable_Wrap(made);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_token_logprobs_grad(s.logits.data, s.logits.type, s.logits.rows, s.logits.columns, s.logits.stride, s.ids(), s.n, s.temperature,
                               s.masks.bits, s.masks.kind, s.masks.class_of_token, s.masks.C, logprob, stats, grad_logprob, entropy,
                               grad_entropy, out, s.logits.columns, stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// rows x columns values of `type` beside a tensor, rows any distance apart; for None `data` is null
struct Rows {
    const void *data = nullptr;
    int64_t stride = 0;
};
bool rows_of(PyObject *o, at::ScalarType type, int64_t rows, int64_t columns, const at::Tensor &beside, Rows *out) {
    if (o == Py_None) return true;
    const at::Tensor *t = plain(o);
    if (!t || t->scalar_type() != type || t->dim() != 2 || t->size(0) != rows || t->size(1) != columns || (columns > 1 && t->stride(1) != 1) ||
        t->device() != beside.device())
        return false;
    out->stride = rows > 1 || t->stride(0) > columns ? t->stride(0) : columns;
    out->data = t->data_ptr();
    return out->stride >= columns;
}
bool layer_of(PyObject *const *args, Matrix *hidden, Matrix *weight) {
    return matrix_of(args[0], hidden) && matrix_of(args[1], weight) && weight->type != 0 && hidden->type == weight->type &&
           hidden->columns == weight->columns && hidden->rows >= 1 && weight->rows >= 1 && hidden->t->device() == weight->t->device() &&
           here(*weight->t);
}

// (hidden, weight, bias, activation's number, residual, the result's type, want_slope)
PyObject *head_layer(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 7 || !g_head_layer || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Matrix x{}, w{};
    Rows residual;
    const void *bias = nullptr;
    int32_t activation = -1, type = -1;
    bool want_slope = false;
    void *out = nullptr, *slope = nullptr, *ws = nullptr, *stream = nullptr;
    size_t bytes = 0;
    at::Tensor workspace;
    PyObject *result = nullptr;
    try {
        if (!layer_of(args, &x, &w) || !bool_of(args[6], &want_slope)) return leave_it();
        activation = type_of(args[3], 4);
        type = args[5] == Py_None ? w.type : type_of(args[5], 2);
        if (activation < 0 || (type != 0 && type != w.type) || !rows_of(args[4], kTypes[w.type], x.rows, w.rows, *w.t, &residual)) return leave_it();
        if (args[2] != Py_None && !(bias = vector_of(args[2], kTypes[w.type], w.rows, *w.t))) return leave_it();
        const at::Tensor made = at::empty({x.rows, w.rows}, w.t->options().dtype(kTypes[type]));
        out = made.data_ptr();
        at::Tensor made_slope;
        if (want_slope) {
            made_slope = at::empty({x.rows, w.rows}, w.t->options().dtype(at::kShort));
            slope = made_slope.data_ptr();
        }
        bytes = g_head_layer_bytes(x.rows, w.rows, w.columns);
        if (bytes) {
            workspace = workspace_of(bytes, *w.t);
            ws = workspace.data_ptr();
            bytes = (size_t)workspace.numel();
        }
        stream = c10::hip::getCurrentHIPStream().stream();
        const Held a(THPVariable_Wrap(made)), b(want_slope ? THPVariable_Wrap(made_slope) : Py_NewRef(Py_None));
        if (a.o && b.o) result = PyTuple_Pack(2, a.o, b.o);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_head_layer(x.data, x.stride, w.data, w.stride, w.type, x.rows, w.rows, w.columns, bias, activation, residual.data, residual.stride,
                      out, type, w.rows, slope, slope ? w.rows : 0, ws, bytes, stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// (hidden, weight, grad_out, slope, want_hidden, want_weight, want_bias)
PyObject *head_layer_grad(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != 7 || !g_head_layer_grad || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    Matrix x{}, w{}, g{};
    Rows slope;
    bool want[3] = {false, false, false};
    void *out[3] = {nullptr, nullptr, nullptr}, *ws = nullptr, *stream = nullptr;
    at::Tensor workspace;
    PyObject *result = nullptr;
    try {
        if (!layer_of(args, &x, &w) || !matrix_of(args[2], &g) || g.rows != x.rows || g.columns != w.rows || (g.type != 0 && g.type != w.type) ||
            g.t->device() != w.t->device() || !rows_of(args[3], at::kShort, x.rows, w.rows, *w.t, &slope) || !bool_of(args[4], &want[0]) ||
            !bool_of(args[5], &want[1]) || !bool_of(args[6], &want[2]) || !(want[0] || want[1] || want[2]))
            return leave_it();
        at::Tensor made[3];
        if (want[0]) made[0] = at::empty({x.rows, w.columns}, w.t->options());
        if (want[1]) made[1] = at::empty({w.rows, w.columns}, w.t->options());
        if (want[2]) made[2] = at::empty({w.rows}, w.t->options());
        for (int i = 0; i < 3; ++i) out[i] = want[i] ? made[i].data_ptr() : nullptr;
        workspace = workspace_of(g_head_layer_grad_bytes(x.rows, w.rows, w.columns), *w.t);
        ws = workspace.data_ptr();
        stream = c10::hip::getCurrentHIPStream().stream();
        const Held a(want[0] ? THPVariable_Wrap(made[0]) : Py_NewRef(Py_None)), b(want[1] ? THPVariable_Wrap(made[1]) : Py_NewRef(Py_None)),
            c(want[2] ? THPVariable_Wrap(made[2]) : Py_NewRef(Py_None));
        if (a.o && b.o && c.o) result = PyTuple_Pack(3, a.o, b.o, c.o);
    } catch (...) {
    }
    if (!result) return leave_it();
    int rc = 0;
    Py_BEGIN_ALLOW_THREADS
    rc = g_head_layer_grad(x.data, x.stride, w.data, w.stride, w.type, x.rows, w.rows, w.columns, g.data, g.type, g.stride, slope.data,
                           slope.stride, out[0], out[0] ? w.columns : 0, out[1], out[1] ? w.columns : 0, out[2], ws,
                           (size_t)workspace.numel(), stream);
    Py_END_ALLOW_THREADS
    return finish(rc, result);
}

// The addresses of cfgzip_token_logprobs_workspace_bytes, cfgzip_token_logprobs, cfgzip_token_logprobs_grad, cfgzip_head_layer_workspace_bytes,
// cfgzip_head_layer, cfgzip_head_layer_grad_workspace_bytes and cfgzip_head_layer_grad
PyObject *connect_layer(PyObject *, PyObject *const *args, Py_ssize_t n) {
    void *at[7];
    if (n != 7) {
        PyErr_SetString(PyExc_TypeError, "connect_layer takes seven addresses");
        return nullptr;
    }
    for (int i = 0; i < 7; ++i) at[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    g_token_logprobs_bytes = reinterpret_cast<TokenLogprobsBytes>(at[0]);
    g_token_logprobs = reinterpret_cast<TokenLogprobs>(at[1]);
    g_token_logprobs_grad = reinterpret_cast<TokenLogprobsGrad>(at[2]);
    g_head_layer_bytes = reinterpret_cast<HeadLayerBytes>(at[3]);
    g_head_layer = reinterpret_cast<HeadLayer>(at[4]);
    g_head_layer_grad_bytes = reinterpret_cast<HeadLayerBytes>(at[5]);
    g_head_layer_grad = reinterpret_cast<HeadLayerGrad>(at[6]);
    Py_RETURN_NONE;
}

// The addresses of cfgzip_decode_step, cfgzip_engine_step, cfgzip_signatures, cfgzip_build_classes, cfgzip_displacements and
// cfgzip_nfa_signatures, of the library that the binding has loaded
PyObject *connect(PyObject *, PyObject *const *args, Py_ssize_t n) {
    void *at[6];
    if (n != 6) {
        PyErr_SetString(PyExc_TypeError, "connect takes six addresses");
        return nullptr;
    }
    for (int i = 0; i < 6; ++i) at[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    g_decode_step = reinterpret_cast<DecodeStep>(at[0]);
    g_engine_step = reinterpret_cast<EngineStep>(at[1]);
    g_signatures = reinterpret_cast<Signatures>(at[2]);
    g_build_classes = reinterpret_cast<BuildClasses>(at[3]);
    g_displacements = reinterpret_cast<Displacements>(at[4]);
    g_nfa_signatures = reinterpret_cast<NfaSignatures>(at[5]);
    Py_RETURN_NONE;
}

template <PyObject *(*F)(PyObject *, PyObject *const *, Py_ssize_t)>
PyCFunction fast() {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(F));
}
PyMethodDef g_methods[] = {{"decode_step", fast<decode_step>(), METH_FASTCALL, nullptr},
                           {"engine_step", fast<engine_step>(), METH_FASTCALL, nullptr},
                           {"signatures", fast<signatures>(), METH_FASTCALL, nullptr},
                           {"build_classes", fast<build_classes>(), METH_FASTCALL, nullptr},
                           {"displacements", fast<displacements>(), METH_FASTCALL, nullptr},
                           {"nfa_signatures", fast<nfa_signatures>(), METH_FASTCALL, nullptr},
                           {"connect", fast<connect>(), METH_FASTCALL, nullptr},
                           {"head_loss", fast<head_loss>(), METH_FASTCALL, nullptr},
                           {"head_loss_grad", fast<head_loss_grad>(), METH_FASTCALL, nullptr},
                           {"mx4_quantize", fast<mx4_quantize>(), METH_FASTCALL, nullptr},
                           {"mx4_values", fast<mx4_values>(), METH_FASTCALL, nullptr},
                           {"mx4_logits", fast<mx4_logits>(), METH_FASTCALL, nullptr},
                           {"connect_head", fast<connect_head>(), METH_FASTCALL, nullptr},
                           {"token_logprobs", fast<token_logprobs>(), METH_FASTCALL, nullptr},
                           {"token_logprobs_grad", fast<token_logprobs_grad>(), METH_FASTCALL, nullptr},
                           {"head_layer", fast<head_layer>(), METH_FASTCALL, nullptr},
                           {"head_layer_grad", fast<head_layer_grad>(), METH_FASTCALL, nullptr},
                           {"connect_layer", fast<connect_layer>(), METH_FASTCALL, nullptr},
                           {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "cfgzip_stepcall", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#define TEXT_OF(x) #x
#define TEXT(x) TEXT_OF(x)
// What this was built for, which the binding compares with what it runs in: torch's C++ layouts are those of one version.
PyMODINIT_FUNC PyInit_cfgzip_stepcall() {
    PyObject *m = PyModule_Create(&g_module);
    if (m && (PyModule_AddStringConstant(m, "python", TEXT(PY_MAJOR_VERSION) "." TEXT(PY_MINOR_VERSION)) < 0 ||
              PyModule_AddStringConstant(m, "torch", BUILT_FOR_TORCH) < 0)) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}
