// The Python binding's short way into the two products (lowra_lora_forward, lowra_lora_backward_input), their batches, and the gradients of the factors:
// tensor checks, the outputs' and the scratch's memory and the call itself without an interpreted line between them; and the tensor checks of the other calls.
// A call for few tokens is one or two launches of 2.5 us each and 5 to 9 us on the GPU; with every check, pointer and argument handled by the interpreter
// its host side took 12 to 14 us.  Host time of the others (256 x 512, 128 tokens, rank 48), us: a batch of three 16.3 -> 5.2, gradients 17.3 -> 8.6, from kept
// projections 13.5 -> 6.4, such a projection's view 5.2 -> 1.6; a training step of three weights 135 -> 66.
//
// forward / backward_input(layout address, its device, packed, absmax, maps, act, A, B, s, out or None, workspace or None) returns the output,
// a status that is not LOWRA_OK, or None for everything that is not the ordinary case - other types, memory of other devices than the
// current one, other layouts in memory, shapes that do not fit, arrays that are too short, subclasses, errors: the caller then takes the
// interpreted way, which says what is wrong.  Likewise
//   forward_epilogue(as forward, then bias or None, the activation's number, multiply, residual and pre or None each)
//   batch(backward, members, s, workspace)                                          the list of outputs
//   gradients(X, dY, A, B, s, dA or None, dB or None, workspace or None)            the pair of gradients
//   gradients_reuse(X, dY, T, U, r, dA or None, dB or None, workspace or None)      likewise
//   projection(workspace, M, r, member)                                             its view of the workspace
//   epilogue_backward(dY, pre, the activation's number, multiply, dZ, dmultiply, dbias, whether dbias is wanted, workspace: dY given, the others may be None)    the three outputs
//   norm_forward(X, weight, bias, eps, the kind's number, residual, sum, Y, mean, rstd: X and weight given, the others may be None)                 Y, rstd, mean, sum
//   norm_backward(dY, X, weight, rstd, mean, dsum, dX, dweight, dbias, whether these are wanted, workspace: the first four given, the others may be None)   dX, dweight, dbias
//   rotary(q, positions, turns, k or None, interleaved, inverse, scale, out or None, k_out or None)                                                out, or the pair
//   cross_entropy(X, W, labels, scale, weights, ignore_index, loss, dX, whether dX is wanted, workspace: tensors but the first three may be None)   loss, dX
//   adamw(members, lr, betas, eps, weight_decay, step, grad_scale or None, dither)                                                                          the members
//   update_factors(members, lr, momentum, nesterov, weight_decay, steps, coefficients, eps, rank or None, workspace or None)                                     the members
#include <torch/extension.h>

#include <algorithm>
#include <initializer_list>
#include <utility>
#include <vector>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include "lowra.h"

namespace {

using Product = lowra_status (*)(const lowra_layout*, const uint8_t*, const float*, const float*, const uint16_t*, int32_t, const uint16_t*,
                                 const uint16_t*, int32_t, float, uint16_t*, void*, size_t, void*);
using ProductEpilogue = lowra_status (*)(const lowra_layout*, const uint8_t*, const float*, const float*, const uint16_t*, int32_t, const uint16_t*, const uint16_t*,
                                         int32_t, float, const lowra_epilogue*, uint16_t*, void*, size_t, void*);
using WorkspaceBytes = size_t (*)(const lowra_layout*, int32_t, int32_t);
using WorkspaceInit = lowra_status (*)(void*, size_t, void*);
using Batch = lowra_status (*)(const lowra_member*, int32_t, int32_t, int32_t, float, void*, size_t, void*);
using Gradients = lowra_status (*)(const uint16_t*, const uint16_t*, int32_t, int32_t, int32_t, const uint16_t*, const uint16_t*, int32_t, float, uint16_t*, uint16_t*,
                                   void*, size_t, void*);
using GradientsReuse = lowra_status (*)(const uint16_t*, const uint16_t*, int32_t, int32_t, int32_t, const uint16_t*, const uint16_t*, int32_t, uint16_t*, uint16_t*, void*,
                                        size_t, void*);
using GradientsBytes = size_t (*)(int32_t, int32_t);
using Projection = const uint16_t* (*)(const void*, int32_t, int32_t, int32_t);
using EpilogueBytes = size_t (*)(int32_t, int32_t);
using EpilogueBackward = lowra_status (*)(const uint16_t*, const uint16_t*, const uint16_t*, int32_t, int32_t, int32_t, uint16_t*, uint16_t*, float*, void*, size_t, void*);
using UpdateBytes = size_t (*)(const lowra_factor*, int32_t, int32_t);
using Update = lowra_status (*)(const lowra_factor*, int32_t, int32_t, const lowra_update_step*, void*, size_t, void*);
using NormBytes = size_t (*)(int32_t, int32_t);
using NormForward = decltype(&lowra_norm_forward);
using NormBackward = decltype(&lowra_norm_backward);
using Rotary = decltype(&lowra_rotary);
using LossBytes = decltype(&lowra_cross_entropy_workspace_bytes);
using Loss = decltype(&lowra_cross_entropy);
using Adamw = decltype(&lowra_adamw);
struct Library {
    Product forward, backward_input;
    WorkspaceBytes workspace_bytes;
    WorkspaceInit workspace_init;
    Batch forward_batch, backward_input_batch;
    Gradients gradients;
    GradientsReuse gradients_reuse;
    GradientsBytes gradients_bytes;
    Projection projection;
    ProductEpilogue forward_epilogue;
    EpilogueBytes epilogue_bytes;
    EpilogueBackward epilogue_backward;
    UpdateBytes update_bytes;
    Update update;
    NormBytes norm_bytes;
    NormForward norm_forward;
    NormBackward norm_backward;
    Rotary rotary;
    LossBytes loss_bytes;
    Loss loss;
    Adamw adamw;
} library;

bool plain(PyObject* o) { return THPVariable_CheckExact(o); }

// memory of device `dev` without gaps
bool on(const at::Tensor& t, int64_t dev) { return t.device() == at::Device(at::kCUDA, (c10::DeviceIndex)dev) && t.is_contiguous(); }
bool matrix(const at::Tensor& t, int64_t rows, int64_t cols, int64_t dev) {
    return on(t, dev) && t.scalar_type() == at::kBFloat16 && t.dim() == 2 && t.size(0) == rows && t.size(1) == cols;
}
bool array(const at::Tensor& t, at::ScalarType type, int64_t least, int64_t dev) { return on(t, dev) && t.scalar_type() == type && t.numel() >= least; }

// Other Python threads run while one of these lives.
struct Released {
    PyThreadState* state = PyEval_SaveThread();
    ~Released() { PyEval_RestoreThread(state); }
};

// A reference of ours.
struct Held {
    PyObject* o = nullptr;
    ~Held() { Py_XDECREF(o); }
};

// epilogue: with the arguments of one behind the others
PyObject* product(PyObject* const* args, Py_ssize_t n, bool backward, bool epilogue = false) {
    if (n != (epilogue ? 16 : 11) || library.forward == nullptr) Py_RETURN_NONE;
    for (int i = 11; i < n; ++i)
        if (i == 12 ? !PyLong_CheckExact(args[i]) : args[i] != Py_None && !plain(args[i])) Py_RETURN_NONE;
    for (int i = 2; i <= 7; ++i)
        if (!plain(args[i])) Py_RETURN_NONE;
    const bool out_given = args[9] != Py_None, workspace_given = args[10] != Py_None;
    if ((out_given && !plain(args[9])) || (workspace_given && !plain(args[10])) || !(PyFloat_CheckExact(args[8]) || PyLong_CheckExact(args[8]))) Py_RETURN_NONE;
    const lowra_layout* layout = static_cast<const lowra_layout*>(PyLong_AsVoidPtr(args[0]));
    const long dev = PyLong_AsLong(args[1]);
    const double s = PyFloat_AsDouble(args[8]);
    if (PyErr_Occurred() != nullptr || layout == nullptr) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
    try {
        const at::Tensor &packed = THPVariable_Unpack(args[2]), &absmax = THPVariable_Unpack(args[3]), &maps = THPVariable_Unpack(args[4]);
        const at::Tensor &act = THPVariable_Unpack(args[5]), &A = THPVariable_Unpack(args[6]), &B = THPVariable_Unpack(args[7]);
        if (act.dim() != 2 || A.dim() != 2 || dev != c10::cuda::current_device()) Py_RETURN_NONE;
        const int64_t M = act.size(0), r = A.size(1), N = layout->N, K = layout->K, cols = backward ? K : N;
        if (!matrix(act, M, backward ? N : K, dev) || !matrix(A, K, r, dev) || !matrix(B, r, N, dev) || M > INT32_MAX || r > INT32_MAX) Py_RETURN_NONE;
        if (!on(packed, dev) || packed.nbytes() < layout->packed_bytes || !array(absmax, at::kFloat, N * (K / 64), dev) || !array(maps, at::kFloat, N * 16, dev)) Py_RETURN_NONE;
        if (out_given && !array(THPVariable_Unpack(args[9]), at::kBFloat16, M * cols, dev)) Py_RETURN_NONE;
        if (workspace_given && !on(THPVariable_Unpack(args[10]), dev)) Py_RETURN_NONE;
        lowra_epilogue behind = {};
        if (epilogue) {
            if (args[11] != Py_None) {
                const at::Tensor& bias = THPVariable_Unpack(args[11]);
                behind.bias_bf16 = bias.scalar_type() == at::kBFloat16;
                if (!array(bias, behind.bias_bf16 ? at::kBFloat16 : at::kFloat, N, dev) || bias.dim() != 1 || bias.size(0) != N) Py_RETURN_NONE;
                behind.bias_dev = bias.data_ptr();
            }
            behind.activation = (int32_t)PyLong_AsLong(args[12]);
            const uint16_t* rows[3] = {};
            for (int i = 0; i < 3; ++i) {
                if (args[13 + i] == Py_None) continue;
                const at::Tensor& t = THPVariable_Unpack(args[13 + i]);
                if (!matrix(t, M, N, dev)) Py_RETURN_NONE;
                rows[i] = static_cast<const uint16_t*>(t.data_ptr());
            }
            behind.multiply_dev = rows[0];
            behind.residual_dev = rows[1];
            behind.pre_dev = const_cast<uint16_t*>(rows[2]);
        }
        const Product call = backward ? library.backward_input : library.forward;
        const auto* packed_p = static_cast<const uint8_t*>(packed.data_ptr());
        const auto *absmax_p = static_cast<const float*>(absmax.data_ptr()), *maps_p = static_cast<const float*>(maps.data_ptr());
        const auto *act_p = static_cast<const uint16_t*>(act.data_ptr()), *A_p = static_cast<const uint16_t*>(A.data_ptr()), *B_p = static_cast<const uint16_t*>(B.data_ptr());
        const at::TensorOptions options = act.options().requires_grad(false);
        at::Tensor out, workspace;
        if (out_given) out = THPVariable_Unpack(args[9]);
        if (workspace_given) workspace = THPVariable_Unpack(args[10]);
        lowra_status st = LOWRA_ERR_WORKSPACE;
        bool called = false;
        {
            Released released;      // (allocations included: one that has to ask the driver for memory takes its time)
            void* stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
            if (!out_given) out = at::empty({M, cols}, options);
            bool ready = true;
            if (!workspace_given) {
                const size_t bytes = library.workspace_bytes(layout, (int32_t)M, (int32_t)r);
                ready = bytes > 0;
                if (ready) workspace = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
                if (ready && layout->deal_dev != nullptr) ready = library.workspace_init(workspace.data_ptr(), bytes, stream) == LOWRA_OK;   // no prologue launch will clear it
            }
            if (ready) {
                auto* out_p = static_cast<uint16_t*>(out.data_ptr());
                st = epilogue ? library.forward_epilogue(layout, packed_p, absmax_p, maps_p, act_p, (int32_t)M, A_p, B_p, (int32_t)r, (float)s, &behind, out_p,
                                                         workspace.data_ptr(), (size_t)workspace.numel(), stream)
                              : call(layout, packed_p, absmax_p, maps_p, act_p, (int32_t)M, A_p, B_p, (int32_t)r, (float)s, out_p, workspace.data_ptr(),
                                     (size_t)workspace.numel(), stream);
                called = true;
            }
        }
        if (!called) Py_RETURN_NONE;
        if (st != LOWRA_OK) return PyLong_FromLong(st);
        if (out_given) {
            Py_INCREF(args[9]);
            return args[9];
        }
        return THPVariable_Wrap(std::move(out));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* forward(PyObject*, PyObject* const* args, Py_ssize_t n) { return product(args, n, false); }
PyObject* backward_input(PyObject*, PyObject* const* args, Py_ssize_t n) { return product(args, n, true); }

PyObject* forward_epilogue(PyObject*, PyObject* const* args, Py_ssize_t n) { return product(args, n, false, true); }

// A number, or not: an exact int within an int32, an exact float or int.
bool number(PyObject* o, int32_t* v) {
    int overflow = 0;
    const long long x = PyLong_CheckExact(o) ? PyLong_AsLongLongAndOverflow(o, &overflow) : -1;
    *v = (int32_t)x;
    return PyLong_CheckExact(o) && overflow == 0 && x >= 0 && x <= INT32_MAX;
}
bool number(PyObject* o, double* v) {
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
    *v = PyFloat_AsDouble(o);
    if (PyErr_Occurred() == nullptr) return true;
    PyErr_Clear();
    return false;
}
uint16_t* bf16(const at::Tensor& t) { return static_cast<uint16_t*>(t.data_ptr()); }

// gradients(X, dY, A, B, s, dA, dB, workspace), and with `reuse` (X, dY, T, U, r, dA, dB, workspace)
PyObject* factor_gradients(PyObject* const* args, Py_ssize_t n, bool reuse) {
    double s = 0.0;
    int32_t rank = 0;
    if (n != 8 || library.forward == nullptr || !(reuse ? number(args[4], &rank) : number(args[4], &s))) Py_RETURN_NONE;
    for (int i = 0; i < 8; ++i)
        if (i != 4 && !(i > 4 && args[i] == Py_None) && !plain(args[i])) Py_RETURN_NONE;
    try {
        const int64_t dev = c10::cuda::current_device();
        const at::Tensor &X = THPVariable_Unpack(args[0]), &dY = THPVariable_Unpack(args[1]), &P = THPVariable_Unpack(args[2]), &Q = THPVariable_Unpack(args[3]);
        if (X.dim() != 2 || dY.dim() != 2 || P.dim() != 2) Py_RETURN_NONE;
        const int64_t M = X.size(0), K = X.size(1), N = dY.size(1), r = reuse ? rank : P.size(1), rp = (r + 63) / 64 * 64;
        if (M > INT32_MAX || K > INT32_MAX || N > INT32_MAX || r > INT32_MAX || !matrix(X, M, K, dev) || !matrix(dY, M, N, dev)) Py_RETURN_NONE;
        if (reuse ? !matrix(P, M, rp, dev) || !matrix(Q, M, rp, dev) : !matrix(P, K, r, dev) || !matrix(Q, r, N, dev)) Py_RETURN_NONE;
        at::Tensor out[2], workspace;
        for (int i = 0; i < 2; ++i) {
            if (args[5 + i] == Py_None) continue;
            out[i] = THPVariable_Unpack(args[5 + i]);
            if (!array(out[i], at::kBFloat16, i == 0 ? K * r : r * N, dev)) Py_RETURN_NONE;
        }
        if (args[7] != Py_None) {
            workspace = THPVariable_Unpack(args[7]);
            if (!on(workspace, dev)) Py_RETURN_NONE;
        }
        const size_t bytes = reuse ? 256 : library.gradients_bytes((int32_t)M, (int32_t)r);
        if (bytes == 0) Py_RETURN_NONE;
        const at::TensorOptions options = X.options().requires_grad(false);
        lowra_status st;
        {
            Released released;
            void* stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
            if (!out[0].defined()) out[0] = at::empty({K, r}, options);
            if (!out[1].defined()) out[1] = at::empty({r, N}, options);
            if (!workspace.defined()) workspace = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
            const size_t size = (size_t)workspace.numel();
            st = reuse ? library.gradients_reuse(bf16(X), bf16(dY), (int32_t)M, (int32_t)K, (int32_t)N, bf16(P), bf16(Q), (int32_t)r, bf16(out[0]), bf16(out[1]),
                                                 workspace.data_ptr(), size, stream)
                       : library.gradients(bf16(X), bf16(dY), (int32_t)M, (int32_t)K, (int32_t)N, bf16(P), bf16(Q), (int32_t)r, (float)s, bf16(out[0]), bf16(out[1]),
                                           workspace.data_ptr(), size, stream);
        }
        if (st != LOWRA_OK) return PyLong_FromLong(st);
        PyObject* both = PyTuple_New(2);
        for (int i = 0; both != nullptr && i < 2; ++i) {
            PyObject* o = args[5 + i];
            if (o != Py_None) Py_INCREF(o);
            else o = THPVariable_Wrap(std::move(out[i]));
            PyTuple_SET_ITEM(both, i, o);
        }
        return both;
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* gradients(PyObject*, PyObject* const* args, Py_ssize_t n) { return factor_gradients(args, n, false); }
PyObject* gradients_reuse(PyObject*, PyObject* const* args, Py_ssize_t n) { return factor_gradients(args, n, true); }

PyObject* projection(PyObject*, PyObject* const* args, Py_ssize_t n) {
    int32_t M = 0, r = 0, member = 0;
    if (n != 4 || library.forward == nullptr || !plain(args[0]) || !number(args[1], &M) || !number(args[2], &r) || !number(args[3], &member)) Py_RETURN_NONE;
    try {
        const at::Tensor& workspace = THPVariable_Unpack(args[0]);
        if (workspace.dim() != 1 || !array(workspace, at::kByte, 0, c10::cuda::current_device())) Py_RETURN_NONE;
        const auto* p = reinterpret_cast<const uint8_t*>(library.projection(workspace.data_ptr(), member, M, r));
        if (p == nullptr) Py_RETURN_NONE;
        const int64_t from = p - static_cast<const uint8_t*>(workspace.data_ptr()), rp = ((int64_t)r + 63) / 64 * 64, bytes = (int64_t)M * rp * 2;
        if (from + bytes > workspace.numel()) Py_RETURN_NONE;
        return THPVariable_Wrap(workspace.slice(0, from, from + bytes).view(at::kBFloat16).view({(int64_t)M, rp}));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// batch(backward, members, s, workspace): a list of dicts with layout, packed, absmax, maps, act, A, B, out
PyObject* batch(PyObject*, PyObject* const* args, Py_ssize_t n) {
    double s = 0.0;
    if (n != 4 || library.forward == nullptr || !PyBool_Check(args[0]) || !PyList_CheckExact(args[1]) || !number(args[2], &s) || !plain(args[3])) Py_RETURN_NONE;
    const bool backward = args[0] == Py_True;
    const Py_ssize_t count = PyList_GET_SIZE(args[1]);
    if (count < 1 || count > LOWRA_MAX_BATCH) Py_RETURN_NONE;
    static PyObject* names[10] = {};      // (interned once)
    if (names[9] == nullptr) {
        constexpr const char* kNames[10] = {"packed", "absmax", "maps", "act", "A", "B", "out", "layout", "address", "device_index"};
        for (int i = 0; i < 10; ++i) names[i] = PyUnicode_InternFromString(kNames[i]);
    }
    // the members' arrays, layouts and outputs: their dicts are the caller's, and other threads run during the call
    at::Tensor arrays[LOWRA_MAX_BATCH][7];
    Held layouts[LOWRA_MAX_BATCH], outs[LOWRA_MAX_BATCH];
    lowra_member members[LOWRA_MAX_BATCH];
    try {
        const int64_t dev = c10::cuda::current_device();
        const at::Tensor& workspace = THPVariable_Unpack(args[3]);
        if (!on(workspace, dev)) Py_RETURN_NONE;
        int64_t M = 0, r = 0;
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject* m = PyList_GET_ITEM(args[1], i);
            if (!PyDict_CheckExact(m)) Py_RETURN_NONE;
            PyObject* o = nullptr;
            for (int j = 0; j < 7; ++j) {
                o = PyDict_GetItemWithError(m, names[j]);
                if (o == nullptr || !plain(o)) {
                    PyErr_Clear();
                    Py_RETURN_NONE;
                }
                arrays[i][j] = THPVariable_Unpack(o);
            }
            outs[i].o = Py_NewRef(o);
            layouts[i].o = Py_XNewRef(PyDict_GetItemWithError(m, names[7]));
            Held address, where;
            if (layouts[i].o != nullptr) address.o = PyObject_GetAttr(layouts[i].o, names[8]);
            if (address.o != nullptr) where.o = PyObject_GetAttr(layouts[i].o, names[9]);
            const bool known = where.o != nullptr && PyLong_CheckExact(address.o) && PyLong_CheckExact(where.o);
            const auto* layout = known ? static_cast<const lowra_layout*>(PyLong_AsVoidPtr(address.o)) : nullptr;
            const bool here = known && PyLong_AsLong(where.o) == dev;
            PyErr_Clear();
            if (layout == nullptr || !here) Py_RETURN_NONE;
            const at::Tensor &packed = arrays[i][0], &absmax = arrays[i][1], &maps = arrays[i][2], &act = arrays[i][3], &A = arrays[i][4], &B = arrays[i][5], &out = arrays[i][6];
            const int64_t N = layout->N, K = layout->K;
            if (i == 0) {
                if (act.dim() != 2 || A.dim() != 2) Py_RETURN_NONE;
                M = act.size(0);
                r = A.size(1);
            }
            if (M > INT32_MAX || r > INT32_MAX || !matrix(act, M, backward ? N : K, dev) || !matrix(out, M, backward ? K : N, dev) || !matrix(A, K, r, dev) ||
                !matrix(B, r, N, dev) || !on(packed, dev) || packed.nbytes() < layout->packed_bytes || !array(absmax, at::kFloat, N * (K / 64), dev) ||
                !array(maps, at::kFloat, N * 16, dev))
                Py_RETURN_NONE;
            members[i] = lowra_member{layout, static_cast<const uint8_t*>(packed.data_ptr()), static_cast<const float*>(absmax.data_ptr()),
                                      static_cast<const float*>(maps.data_ptr()), bf16(act), bf16(A), bf16(B), bf16(out)};
        }
        lowra_status st;
        {
            Released released;
            st = (backward ? library.backward_input_batch : library.forward_batch)(members, (int32_t)count, (int32_t)M, (int32_t)r, (float)s, workspace.data_ptr(),
                                                                                  (size_t)workspace.numel(), c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream());
        }
        if (st != LOWRA_OK) return PyLong_FromLong(st);
        PyObject* list = PyList_New(count);
        for (Py_ssize_t i = 0; list != nullptr && i < count; ++i) PyList_SET_ITEM(list, i, Py_NewRef(outs[i].o));
        return list;
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* epilogue_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    int32_t activation = 0;
    if (n != 9 || library.forward == nullptr || !plain(args[0]) || !number(args[2], &activation) || !PyBool_Check(args[7])) Py_RETURN_NONE;
    for (int i = 1; i < 9; ++i)
        if (i != 2 && i != 7 && args[i] != Py_None && !plain(args[i])) Py_RETURN_NONE;
    try {
        const int64_t dev = c10::cuda::current_device();
        const at::Tensor& dY = THPVariable_Unpack(args[0]);
        if (dY.dim() != 2) Py_RETURN_NONE;
        const int64_t M = dY.size(0), N = dY.size(1);
        if (M > INT32_MAX || N > INT32_MAX || !matrix(dY, M, N, dev)) Py_RETURN_NONE;
        at::Tensor rows[4], dbias, workspace;          // pre, multiply, dZ, dmultiply
        constexpr int kAt[4] = {1, 3, 4, 5};
        for (int i = 0; i < 4; ++i) {
            if (args[kAt[i]] == Py_None) continue;
            rows[i] = THPVariable_Unpack(args[kAt[i]]);
            if (!matrix(rows[i], M, N, dev)) Py_RETURN_NONE;
        }
        if (args[6] != Py_None) {
            dbias = THPVariable_Unpack(args[6]);
            if (!array(dbias, at::kFloat, N, dev) || dbias.dim() != 1 || dbias.size(0) != N) Py_RETURN_NONE;
        }
        if (args[8] != Py_None) {
            workspace = THPVariable_Unpack(args[8]);
            if (!on(workspace, dev)) Py_RETURN_NONE;
        }
        const at::TensorOptions options = dY.options().requires_grad(false);
        const bool with_bias = dbias.defined() || args[7] == Py_True;
        lowra_status st;
        {
            Released released;
            void* stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
            if (!rows[2].defined()) rows[2] = at::empty({M, N}, options);
            if (!rows[3].defined() && rows[1].defined()) rows[3] = at::empty({M, N}, options);
            if (!dbias.defined() && with_bias) dbias = at::empty({N}, options.dtype(at::kFloat));
            if (!workspace.defined() && with_bias) workspace = at::empty({(int64_t)std::max<size_t>(library.epilogue_bytes((int32_t)M, (int32_t)N), 256)}, options.dtype(at::kByte));
            auto at_of = [](const at::Tensor& t) { return t.defined() ? bf16(t) : nullptr; };
            st = library.epilogue_backward(bf16(dY), at_of(rows[0]), at_of(rows[1]), (int32_t)M, (int32_t)N, activation, bf16(rows[2]), at_of(rows[3]),
                                           dbias.defined() ? static_cast<float*>(dbias.data_ptr()) : nullptr, workspace.defined() ? workspace.data_ptr() : nullptr,
                                           workspace.defined() ? (size_t)workspace.nbytes() : 0, stream);
        }
        if (st != LOWRA_OK) return PyLong_FromLong(st);
        PyObject* all = PyTuple_New(3);
        at::Tensor* out[3] = {&rows[2], &rows[3], &dbias};
        for (int i = 0; all != nullptr && i < 3; ++i) {
            PyObject* o = args[4 + i];
            if (o != Py_None) Py_INCREF(o);
            else if (out[i]->defined()) o = THPVariable_Wrap(std::move(*out[i]));
            else Py_INCREF(o);
            PyTuple_SET_ITEM(all, i, o);
        }
        return all;
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* update_factors(PyObject*, PyObject* const* args, Py_ssize_t n) {
    lowra_update_step step = {};
    int32_t rank = 0;
    if (n != 10 || library.forward == nullptr || !PyList_CheckExact(args[0]) || !number(args[1], &step.lr) || !number(args[2], &step.momentum) || !PyBool_Check(args[3]) ||
        !number(args[4], &step.weight_decay) || !number(args[5], &step.steps) || !PyTuple_CheckExact(args[6]) || PyTuple_GET_SIZE(args[6]) != 3 || !number(args[7], &step.eps) ||
        (args[8] != Py_None && !number(args[8], &rank)) || (args[9] != Py_None && !plain(args[9])))
        Py_RETURN_NONE;
    for (int i = 0; i < 3; ++i)
        if (!number(PyTuple_GET_ITEM(args[6], i), &step.coefficients[i])) Py_RETURN_NONE;
    step.nesterov = args[3] == Py_True;
    const Py_ssize_t count = PyList_GET_SIZE(args[0]);
    if (count < 1 || count > LOWRA_MAX_FACTORS) Py_RETURN_NONE;
    enum { kGrad, kMomentum, kMomentumOut, kMaster, kMasterOut, kWeight, kUpdate, kScale, kNames };
    static PyObject* names[kNames] = {};
    if (names[kNames - 1] == nullptr) {
        constexpr const char* kText[kNames] = {"grad", "momentum", "momentum_out", "master", "master_out", "weight", "update", "scale"};
        for (int i = 0; i < kNames; ++i) names[i] = PyUnicode_InternFromString(kText[i]);
    }
    // the members' arrays: their dicts are the caller's, and other threads run during the call
    std::vector<at::Tensor> held;
    held.reserve((size_t)count * kScale + 1);
    lowra_factor factors[LOWRA_MAX_FACTORS];
    int64_t common[2] = {-1, -1};
    try {
        const int64_t dev = c10::cuda::current_device();
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject* m = PyList_GET_ITEM(args[0], i);
            if (!PyDict_CheckExact(m)) Py_RETURN_NONE;
            void* at[kScale] = {};
            int64_t rows = 0, cols = 0;
            lowra_factor& f = factors[i];
            f.grad_fp32 = 0;
            for (int k = 0; k < kScale; ++k) {
                PyObject* o = PyDict_GetItemWithError(m, names[k]);
                if (o == nullptr || o == Py_None) {
                    if (k == kGrad || PyErr_Occurred() != nullptr) {
                        PyErr_Clear();
                        Py_RETURN_NONE;
                    }
                    continue;
                }
                if (!plain(o)) Py_RETURN_NONE;
                held.push_back(THPVariable_Unpack(o));
                const at::Tensor& t = held.back();
                if (t.dim() != 2 || !on(t, dev)) Py_RETURN_NONE;
                if (k == kGrad) {
                    rows = t.size(0);
                    cols = t.size(1);
                    f.grad_fp32 = t.scalar_type() == at::kFloat;
                }
                const at::ScalarType type = k == kWeight || (k == kGrad && !f.grad_fp32) ? at::kBFloat16 : at::kFloat;
                if (t.scalar_type() != type || t.size(0) != rows || t.size(1) != cols || rows > INT32_MAX || cols > INT32_MAX) Py_RETURN_NONE;
                at[k] = t.data_ptr();
            }
            PyObject* scale = PyDict_GetItemWithError(m, names[kScale]);
            f.scale = 1.0;
            if (PyErr_Occurred() != nullptr || (scale != nullptr && !number(scale, &f.scale))) {
                PyErr_Clear();
                Py_RETURN_NONE;
            }
            f.rows = (int32_t)rows;
            f.cols = (int32_t)cols;
            f.grad_dev = at[kGrad];
            f.momentum_dev = static_cast<const float*>(at[kMomentum]);
            f.momentum_out_dev = static_cast<float*>(at[kMomentumOut] != nullptr ? at[kMomentumOut] : at[kMomentum]);
            f.master_dev = static_cast<const float*>(at[kMaster]);
            f.master_out_dev = static_cast<float*>(at[kMasterOut] != nullptr ? at[kMasterOut] : at[kMaster]);
            f.weight_dev = static_cast<uint16_t*>(at[kWeight]);
            f.update_dev = static_cast<float*>(at[kUpdate]);
            // the sides that all have in common
            if (i == 0) {
                common[0] = rows;
                common[1] = cols;
            }
            for (int64_t& c : common)
                if (c != rows && c != cols) c = -1;
        }
        if (args[8] == Py_None) {         // the least of them that can be a rank
            for (const int64_t c : common)
                if (c >= 16 && c <= 128 && c % 16 == 0 && (rank == 0 || c < rank)) rank = (int32_t)c;
            if (rank == 0) Py_RETURN_NONE;
        }
        at::Tensor workspace;
        if (args[9] != Py_None) {
            workspace = THPVariable_Unpack(args[9]);
            if (!on(workspace, dev)) Py_RETURN_NONE;
        }
        lowra_status st;
        {
            Released released;
            void* stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
            if (!workspace.defined()) {
                const size_t bytes = library.update_bytes(factors, (int32_t)count, rank);
                if (bytes > 0) workspace = at::empty({(int64_t)bytes}, held[0].options().requires_grad(false).dtype(at::kByte));
            }
            st = workspace.defined() ? library.update(factors, (int32_t)count, rank, &step, workspace.data_ptr(), (size_t)workspace.nbytes(), stream) : LOWRA_ERR_SHAPE;
        }
        if (st != LOWRA_OK) return PyLong_FromLong(st);
        Py_INCREF(args[0]);
        return args[0];
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// ---- the operators of a training step beside the products
bool each_plain_or_none(PyObject* const* args, std::initializer_list<int> places) {
    for (int i : places)
        if (args[i] != Py_None && !plain(args[i])) return false;
    return true;
}
at::Tensor given(PyObject* o) { return o == Py_None ? at::Tensor() : THPVariable_Unpack(o); }
float* fp32(const at::Tensor& t) { return t.defined() ? static_cast<float*>(t.data_ptr()) : nullptr; }
uint16_t* bf16_or_null(const at::Tensor& t) { return t.defined() ? bf16(t) : nullptr; }
bool vector_of(const at::Tensor& t, int64_t n, int64_t dev) { return !t.defined() || (array(t, at::kFloat, n, dev) && t.dim() == 1 && t.size(0) == n); }
bool rows_of(const at::Tensor& t, int64_t M, int64_t N, int64_t dev) { return !t.defined() || matrix(t, M, N, dev); }
// The results in order: the caller's own objects where they gave some, else the new ones, else None.
PyObject* results(std::initializer_list<std::pair<PyObject*, at::Tensor*>> all) {
    PyObject* tuple = PyTuple_New((Py_ssize_t)all.size());
    Py_ssize_t i = 0;
    for (const auto& [o, t] : all) {
        PyObject* r = o != Py_None || !t->defined() ? Py_NewRef(o) : THPVariable_Wrap(std::move(*t));
        if (tuple != nullptr) PyTuple_SET_ITEM(tuple, i++, r);
        else Py_XDECREF(r);
    }
    return tuple;
}

PyObject* norm_forward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    double eps = 0.0;
    int32_t kind = 0;
    if (n != 10 || library.forward == nullptr || !plain(args[0]) || !plain(args[1]) || !number(args[3], &eps) || !number(args[4], &kind) ||
        !each_plain_or_none(args, {2, 5, 6, 7, 8, 9}))
        Py_RETURN_NONE;
    try {
        const int64_t dev = c10::cuda::current_device();
        const at::Tensor &X = THPVariable_Unpack(args[0]), &weight = THPVariable_Unpack(args[1]);
        if (X.dim() != 2) Py_RETURN_NONE;
        const int64_t M = X.size(0), N = X.size(1);
        const at::ScalarType type = weight.scalar_type();
        if (M > INT32_MAX || N > INT32_MAX || !matrix(X, M, N, dev) || (type != at::kFloat && type != at::kBFloat16)) Py_RETURN_NONE;
        at::Tensor bias = given(args[2]), residual = given(args[5]), sum = given(args[6]), Y = given(args[7]), mean = given(args[8]), rstd = given(args[9]);
        for (const at::Tensor* t : {&weight, static_cast<const at::Tensor*>(&bias)})
            if (t->defined() && (!array(*t, type, N, dev) || t->dim() != 1 || t->size(0) != N)) Py_RETURN_NONE;
        if (!rows_of(residual, M, N, dev) || !rows_of(sum, M, N, dev) || !rows_of(Y, M, N, dev) || !vector_of(mean, M, dev) || !vector_of(rstd, M, dev)) Py_RETURN_NONE;
        const at::TensorOptions options = X.options().requires_grad(false);
        lowra_status st;
        {
            Released released;
            void* stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
            if (!Y.defined()) Y = at::empty({M, N}, options);
            if (!sum.defined() && residual.defined()) sum = at::empty({M, N}, options);
            if (!rstd.defined()) rstd = at::empty({M}, options.dtype(at::kFloat));
            if (!mean.defined() && kind == LOWRA_NORM_LAYER) mean = at::empty({M}, options.dtype(at::kFloat));
            st = library.norm_forward(bf16(X), bf16_or_null(residual), weight.data_ptr(), bias.defined() ? bias.data_ptr() : nullptr, type == at::kFloat, (int32_t)M, (int32_t)N, kind,
                                      (float)eps, bf16_or_null(sum), bf16(Y), fp32(mean), fp32(rstd), stream);
        }
        if (st != LOWRA_OK) return PyLong_FromLong(st);
        return results({{args[7], &Y}, {args[9], &rstd}, {args[8], &mean}, {args[6], &sum}});
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 11 || library.forward == nullptr || !PyBool_Check(args[9]) || !each_plain_or_none(args, {4, 5, 6, 7, 8, 10})) Py_RETURN_NONE;
    for (int i = 0; i < 4; ++i)
        if (!plain(args[i])) Py_RETURN_NONE;
    try {
        const int64_t dev = c10::cuda::current_device();
        const at::Tensor &dY = THPVariable_Unpack(args[0]), &X = THPVariable_Unpack(args[1]), &weight = THPVariable_Unpack(args[2]), &rstd = THPVariable_Unpack(args[3]);
        if (X.dim() != 2) Py_RETURN_NONE;
        const int64_t M = X.size(0), N = X.size(1);
        const at::ScalarType type = weight.scalar_type();
        if (M > INT32_MAX || N > INT32_MAX || !matrix(X, M, N, dev) || !matrix(dY, M, N, dev) || (type != at::kFloat && type != at::kBFloat16) || !array(weight, type, N, dev) ||
            weight.dim() != 1 || weight.size(0) != N || !vector_of(rstd, M, dev))
            Py_RETURN_NONE;
        at::Tensor mean = given(args[4]), dsum = given(args[5]), dX = given(args[6]), dweight = given(args[7]), dbias = given(args[8]), workspace = given(args[10]);
        if (!vector_of(mean, M, dev) || !rows_of(dsum, M, N, dev) || !rows_of(dX, M, N, dev) || !vector_of(dweight, N, dev) || !vector_of(dbias, N, dev) ||
            (workspace.defined() && !on(workspace, dev)))
            Py_RETURN_NONE;
        const at::TensorOptions options = X.options().requires_grad(false);
        const bool want = args[9] == Py_True;
        lowra_status st;
        {
            Released released;
            void* stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
            if (!dX.defined()) dX = at::empty({M, N}, options);
            if (!dweight.defined() && want) dweight = at::empty({N}, options.dtype(at::kFloat));
            if (!dbias.defined() && want && mean.defined()) dbias = at::empty({N}, options.dtype(at::kFloat));
            if (!workspace.defined() && (dweight.defined() || dbias.defined()))
                workspace = at::empty({(int64_t)std::max<size_t>(library.norm_bytes((int32_t)M, (int32_t)N), 256)}, options.dtype(at::kByte));
            st = library.norm_backward(bf16(dY), bf16(X), weight.data_ptr(), type == at::kFloat, fp32(mean), fp32(rstd), bf16_or_null(dsum), (int32_t)M, (int32_t)N, bf16(dX),
                                       fp32(dweight), fp32(dbias), workspace.defined() ? workspace.data_ptr() : nullptr, workspace.defined() ? (size_t)workspace.nbytes() : 0, stream);
        }
        if (st != LOWRA_OK) return PyLong_FromLong(st);
        return results({{args[6], &dX}, {args[7], &dweight}, {args[8], &dbias}});
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* rotary(PyObject*, PyObject* const* args, Py_ssize_t n) {
    double scale = 1.0;
    if (n != 9 || library.forward == nullptr || !plain(args[0]) || !plain(args[1]) || !plain(args[2]) || !PyBool_Check(args[4]) || !PyBool_Check(args[5]) || !number(args[6], &scale) ||
        !each_plain_or_none(args, {3, 7, 8}) || (args[3] == Py_None && args[8] != Py_None))
        Py_RETURN_NONE;
    try {
        const int64_t dev = c10::cuda::current_device();
        const at::Tensor &q = THPVariable_Unpack(args[0]), &positions = THPVariable_Unpack(args[1]), &turns = THPVariable_Unpack(args[2]);
        if (q.dim() != 3 || positions.dim() != 1 || turns.dim() != 1) Py_RETURN_NONE;
        const int64_t M = q.size(0), D = q.size(2), pairs = turns.size(0);
        if (M > INT32_MAX || D > INT32_MAX || pairs > 65536 || !array(positions, at::kInt, M, dev) || positions.size(0) != M || !on(turns, dev) ||
            (turns.scalar_type() != at::kLong && turns.scalar_type() != at::kUInt64))
            Py_RETURN_NONE;
        const int count = args[3] == Py_None ? 1 : 2;
        at::Tensor x[2] = {q, given(args[3])}, out[2] = {given(args[7]), given(args[8])};
        lowra_rotary_part parts[2] = {};
        for (int i = 0; i < count; ++i)
            for (const at::Tensor* t : {&x[i], &out[i]})
                if (t->defined() && (t->device() != at::Device(at::kCUDA, (c10::DeviceIndex)dev) || t->scalar_type() != at::kBFloat16 || t->dim() != 3 || t->size(0) != M ||
                                     t->size(1) != x[i].size(1) || t->size(1) > INT32_MAX || t->size(2) != D || (D > 1 && t->stride(2) != 1)))
                    Py_RETURN_NONE;
        lowra_status st;
        {
            Released released;
            void* stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
            for (int i = 0; i < count; ++i) {
                if (!out[i].defined()) out[i] = at::empty({M, x[i].size(1), D}, q.options().requires_grad(false));
                parts[i] = lowra_rotary_part{bf16(x[i]), bf16(out[i]), x[i].stride(0), x[i].stride(1), out[i].stride(0), out[i].stride(1), (int32_t)x[i].size(1)};
            }
            st = library.rotary(parts, count, (int32_t)M, (int32_t)D, (int32_t)(2 * pairs), static_cast<const int32_t*>(positions.data_ptr()),
                                static_cast<const uint64_t*>(turns.data_ptr()), (float)scale, args[4] == Py_True, args[5] == Py_True, stream);
        }
        if (st != LOWRA_OK) return PyLong_FromLong(st);
        if (count == 2) return results({{args[7], &out[0]}, {args[8], &out[1]}});
        return args[7] != Py_None ? Py_NewRef(args[7]) : THPVariable_Wrap(std::move(out[0]));
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* cross_entropy(PyObject*, PyObject* const* args, Py_ssize_t n) {
    double scale = 1.0;
    int overflow = 0;
    if (n != 10 || library.forward == nullptr || !plain(args[0]) || !plain(args[1]) || !plain(args[2]) || !number(args[3], &scale) || !PyLong_CheckExact(args[5]) ||
        !PyBool_Check(args[8]) || !each_plain_or_none(args, {4, 6, 7, 9}))
        Py_RETURN_NONE;
    const long long ignore = PyLong_AsLongLongAndOverflow(args[5], &overflow);
    if (overflow != 0) Py_RETURN_NONE;
    try {
        const int64_t dev = c10::cuda::current_device();
        const at::Tensor &X = THPVariable_Unpack(args[0]), &W = THPVariable_Unpack(args[1]), &labels = THPVariable_Unpack(args[2]);
        if (X.dim() != 2 || W.dim() != 2 || labels.dim() != 1) Py_RETURN_NONE;
        const int64_t M = X.size(0), K = X.size(1), V = W.size(0);
        at::Tensor weights = given(args[4]), loss = given(args[6]), dX = given(args[7]), workspace = given(args[9]);
        if (M > INT32_MAX || K > INT32_MAX || V > INT32_MAX || !matrix(X, M, K, dev) || !matrix(W, V, K, dev) || !array(labels, at::kLong, M, dev) || labels.size(0) != M ||
            !vector_of(weights, M, dev) || !vector_of(loss, M, dev) || !rows_of(dX, M, K, dev) || (workspace.defined() && !on(workspace, dev)))
            Py_RETURN_NONE;
        const bool grad = dX.defined() || args[8] == Py_True;
        const at::TensorOptions options = X.options().requires_grad(false);
        lowra_status st;
        {
            Released released;
            void* stream = c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
            if (!loss.defined()) loss = at::empty({M}, options.dtype(at::kFloat));
            if (!dX.defined() && grad) dX = at::empty({M, K}, options);
            if (!workspace.defined()) {
                const size_t bytes = library.loss_bytes((int32_t)M, (int32_t)V, (int32_t)K, grad);
                if (bytes > 0) workspace = at::empty({(int64_t)bytes}, options.dtype(at::kByte));
            }
            st = workspace.defined() ? library.loss(bf16(X), bf16(W), static_cast<const int64_t*>(labels.data_ptr()), fp32(weights), (int32_t)M, (int32_t)V, (int32_t)K, ignore,
                                                    (float)scale, fp32(loss), bf16_or_null(dX), workspace.data_ptr(), (size_t)workspace.nbytes(), stream)
                                     : LOWRA_ERR_SHAPE;
        }
        if (st != LOWRA_OK) return PyLong_FromLong(st);
        return results({{args[6], &loss}, {args[7], &dX}});
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

PyObject* adamw(PyObject*, PyObject* const* args, Py_ssize_t n) {
    lowra_adamw_step step = {};
    if (n != 8 || library.forward == nullptr || !PyBool_Check(args[7]) || !PyList_CheckExact(args[0]) || !PyTuple_CheckExact(args[2]) || PyTuple_GET_SIZE(args[2]) != 2 ||
        !number(PyTuple_GET_ITEM(args[2], 0), &step.beta1) || !number(PyTuple_GET_ITEM(args[2], 1), &step.beta2) || !number(args[3], &step.eps) ||
        !number(args[4], &step.weight_decay))
        Py_RETURN_NONE;
    int32_t t = 0;
    const bool lr_here = number(args[1], &step.lr), step_here = number(args[5], &t);
    if ((!lr_here && !plain(args[1])) || (!step_here && !plain(args[5])) || (args[6] != Py_None && !plain(args[6]))) Py_RETURN_NONE;
    step.step = t;
    const Py_ssize_t count = PyList_GET_SIZE(args[0]);
    if (count < 1 || count > LOWRA_MAX_ADAMW) Py_RETURN_NONE;
    // (read in this order; from kMasterOut on each may be missing)
    enum { kGrad, kMaster, kM, kV, kMScale, kVScale, kMasterOut, kMOut, kVOut, kMScaleOut, kVScaleOut, kWeight, kNames };
    static PyObject* names[kNames] = {};
    if (names[kNames - 1] == nullptr) {
        constexpr const char* kText[kNames] = {"grad", "master", "m", "v", "m_scale", "v_scale", "master_out", "m_out", "v_out", "m_scale_out", "v_scale_out", "weight"};
        for (int i = 0; i < kNames; ++i) names[i] = PyUnicode_InternFromString(kText[i]);
    }
    try {
        // (The members' arrays are not held: no other Python thread runs before the call is made.  Its host side takes some 0.4 us a factor.)
        std::vector<lowra_adamw_member> members((size_t)count);
        const int64_t dev = c10::cuda::current_device();
        const at::Device here(at::kCUDA, (c10::DeviceIndex)dev);
        auto scalar = [&](PyObject* o, at::ScalarType type, const void** p) {
            const at::Tensor& t = THPVariable_Unpack(o);
            *p = t.data_ptr();
            return array(t, type, 1, dev) && t.numel() == 1;
        };
        const void *lr = nullptr, *at_step = nullptr, *factor = nullptr;
        if ((!lr_here && !scalar(args[1], at::kFloat, &lr)) || (!step_here && !scalar(args[5], at::kInt, &at_step)) || (args[6] != Py_None && !scalar(args[6], at::kFloat, &factor)))
            Py_RETURN_NONE;
        step.lr_dev = static_cast<const float*>(lr);
        step.step_dev = static_cast<const int32_t*>(at_step);
        step.grad_scale_dev = static_cast<const float*>(factor);
        at::ScalarType grad_type = at::kFloat, state_type = at::kFloat;
        for (Py_ssize_t i = 0; i < count; ++i) {
            PyObject* m = PyList_GET_ITEM(args[0], i);
            if (!PyDict_CheckExact(m)) Py_RETURN_NONE;
            PyObject *of[kNames] = {}, *key = nullptr, *value = nullptr;
            Py_ssize_t place = 0;
            while (PyDict_Next(m, &place, &key, &value)) {      // (one walk; a name is mostly the same object as ours)
                int k = 0;
                while (k < kNames && key != names[k]) ++k;
                for (int j = 0; k == kNames && j < kNames; ++j)
                    if (PyUnicode_CheckExact(key) && PyUnicode_Compare(key, names[j]) == 0) k = j + 2 * kNames;
                if (k == kNames || value == Py_None) continue;
                of[k >= 2 * kNames ? k - 2 * kNames : k] = value;
            }
            if (PyErr_Occurred() != nullptr || of[kGrad] == nullptr || of[kMaster] == nullptr || of[kM] == nullptr || of[kV] == nullptr || !plain(of[kGrad]) || !plain(of[kM])) {
                PyErr_Clear();
                Py_RETURN_NONE;
            }
            const at::Tensor& grad = THPVariable_Unpack(of[kGrad]);
            if (i == 0) {
                grad_type = grad.scalar_type();
                state_type = THPVariable_Unpack(of[kM]).scalar_type();
            }
            const int64_t elements = grad.numel(), blocks = (elements + LOWRA_ADAMW_BLOCK - 1) / LOWRA_ADAMW_BLOCK;
            if (state_type != at::kFloat && (of[kMScale] == nullptr || of[kVScale] == nullptr)) Py_RETURN_NONE;
            void* at[kNames] = {};
            for (int k = 0; k < kNames; ++k) {
                if (of[k] == nullptr) continue;
                if (!plain(of[k])) Py_RETURN_NONE;
                const at::Tensor& a = THPVariable_Unpack(of[k]);
                const bool scales = k == kMScale || k == kVScale || k == kMScaleOut || k == kVScaleOut, states = k == kM || k == kV || k == kMOut || k == kVOut;
                const at::ScalarType type = k == kGrad ? grad_type : k == kWeight ? at::kBFloat16 : states ? state_type : at::kFloat;
                if (a.device() != here || !a.is_contiguous() || a.scalar_type() != type || (scales && state_type == at::kFloat) ||
                    (scales ? a.dim() != 1 || a.size(0) != blocks : !a.sizes().equals(grad.sizes())))
                    Py_RETURN_NONE;
                at[k] = a.data_ptr();
            }
            auto in = [&](int k) { return static_cast<const float*>(at[k]); };
            auto out = [&](int new_place, int old) { return static_cast<float*>(at[new_place] != nullptr ? at[new_place] : at[old]); };
            members[(size_t)i] = lowra_adamw_member{at[kGrad], in(kMaster), out(kMasterOut, kMaster), static_cast<uint16_t*>(at[kWeight]), at[kM], out(kMOut, kM), at[kV], out(kVOut, kV),
                                                    in(kMScale), out(kMScaleOut, kMScale), in(kVScale), out(kVScaleOut, kVScale), elements};
        }
        if ((grad_type != at::kFloat && grad_type != at::kBFloat16) || (state_type != at::kFloat && state_type != at::kFloat8_e4m3fn)) Py_RETURN_NONE;
        step.bits = (state_type == at::kFloat ? 32 : 8) | (args[7] == Py_True ? LOWRA_ADAMW_DITHER : 0);
        step.grad_fp32 = grad_type == at::kFloat;
        const lowra_status st = library.adamw(members.data(), (int32_t)count, &step, c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream());
        if (st != LOWRA_OK) return PyLong_FromLong(st);
        return Py_NewRef(args[0]);
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// fits(device, then for each array: tensor or None, element type, least number of elements) -> whether every one is a plain tensor on that
// device, which is the current one, without gaps, of that type and long enough; None fits.  Types: 'B' bytes of any type, 'u' uint8, 'h' bf16,
// 'f' fp32, 'd' fp64.  The other calls' checks, a tenth of a microsecond an array where the interpreter takes one; what does not fit is looked at
// by the interpreter, which says what is wrong.
PyObject* fits(PyObject*, PyObject* const* args, Py_ssize_t n) {
    const long dev = n % 3 == 1 ? PyLong_AsLong(args[0]) : -1;
    bool good = dev >= 0;
    try {
        good = good && dev == c10::cuda::current_device();
        for (Py_ssize_t i = 1; good && i < n; i += 3) {
            if (args[i] == Py_None) continue;
            const Py_UCS4 type = PyUnicode_Check(args[i + 1]) && PyUnicode_GET_LENGTH(args[i + 1]) == 1 ? PyUnicode_READ_CHAR(args[i + 1], 0) : 0;
            const int64_t least = PyLong_AsLongLong(args[i + 2]);
            if (!plain(args[i])) { good = false; break; }
            const at::Tensor& t = THPVariable_Unpack(args[i]);
            if (type == 'B') good = on(t, dev) && (int64_t)t.nbytes() >= least;
            else good = type != 0 && array(t, type == 'u' ? at::kByte : type == 'h' ? at::kBFloat16 : type == 'f' ? at::kFloat : at::kDouble, least, dev);
        }
    } catch (...) {
        good = false;
    }
    if (PyErr_Occurred() != nullptr) {
        PyErr_Clear();
        good = false;
    }
    return PyBool_FromLong(good);
}

// bind(addresses of lowra_lora_forward, lowra_lora_backward_input, lowra_workspace_bytes, lowra_workspace_init, lowra_lora_forward_batch, lowra_lora_backward_input_batch,
// lowra_lora_backward_adapters, lowra_lora_backward_adapters_reuse, lowra_adapter_workspace_bytes, lowra_workspace_projection, lowra_lora_forward_epilogue,
// lowra_epilogue_workspace_bytes, lowra_epilogue_backward, lowra_update_workspace_bytes, lowra_update_factors, lowra_norm_workspace_bytes, lowra_norm_forward, lowra_norm_backward,
// lowra_rotary, lowra_cross_entropy_workspace_bytes, lowra_cross_entropy, lowra_adamw)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    constexpr int kAddresses = 22;
    void* p[kAddresses] = {};
    for (int i = 0; i < kAddresses; ++i) {
        p[i] = i < n ? PyLong_AsVoidPtr(args[i]) : nullptr;
        if (p[i] == nullptr) {
            if (PyErr_Occurred() == nullptr) PyErr_SetString(PyExc_ValueError, "bind takes twenty-two addresses");
            return nullptr;
        }
    }
    library = Library{reinterpret_cast<Product>(p[0]), reinterpret_cast<Product>(p[1]), reinterpret_cast<WorkspaceBytes>(p[2]), reinterpret_cast<WorkspaceInit>(p[3]),
                      reinterpret_cast<Batch>(p[4]), reinterpret_cast<Batch>(p[5]), reinterpret_cast<Gradients>(p[6]), reinterpret_cast<GradientsReuse>(p[7]),
                      reinterpret_cast<GradientsBytes>(p[8]), reinterpret_cast<Projection>(p[9]), reinterpret_cast<ProductEpilogue>(p[10]), reinterpret_cast<EpilogueBytes>(p[11]), reinterpret_cast<EpilogueBackward>(p[12]),
                      reinterpret_cast<UpdateBytes>(p[13]), reinterpret_cast<Update>(p[14]), reinterpret_cast<NormBytes>(p[15]), reinterpret_cast<NormForward>(p[16]),
                      reinterpret_cast<NormBackward>(p[17]), reinterpret_cast<Rotary>(p[18]), reinterpret_cast<LossBytes>(p[19]), reinterpret_cast<Loss>(p[20]),
                      reinterpret_cast<Adamw>(p[21])};
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"forward", (PyCFunction)(void (*)())forward, METH_FASTCALL, nullptr},
    {"forward_epilogue", (PyCFunction)(void (*)())forward_epilogue, METH_FASTCALL, nullptr},
    {"backward_input", (PyCFunction)(void (*)())backward_input, METH_FASTCALL, nullptr},
    {"batch", (PyCFunction)(void (*)())batch, METH_FASTCALL, nullptr},
    {"gradients", (PyCFunction)(void (*)())gradients, METH_FASTCALL, nullptr},
    {"gradients_reuse", (PyCFunction)(void (*)())gradients_reuse, METH_FASTCALL, nullptr},
    {"projection", (PyCFunction)(void (*)())projection, METH_FASTCALL, nullptr},
    {"epilogue_backward", (PyCFunction)(void (*)())epilogue_backward, METH_FASTCALL, nullptr},
    {"update_factors", (PyCFunction)(void (*)())update_factors, METH_FASTCALL, nullptr},
    {"norm_forward", (PyCFunction)(void (*)())norm_forward, METH_FASTCALL, nullptr},
    {"norm_backward", (PyCFunction)(void (*)())norm_backward, METH_FASTCALL, nullptr},
    {"rotary", (PyCFunction)(void (*)())rotary, METH_FASTCALL, nullptr},
    {"cross_entropy", (PyCFunction)(void (*)())cross_entropy, METH_FASTCALL, nullptr},
    {"adamw", (PyCFunction)(void (*)())adamw, METH_FASTCALL, nullptr},
    {"fits", (PyCFunction)(void (*)())fits, METH_FASTCALL, nullptr},
    {"bind", (PyCFunction)(void (*)())bind, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_py_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__py_calls() { return PyModule_Create(&module); }
