// Host side of the Python binding: the argument checks and descriptor arrays of calls that take
// many tensors.  In Python each tensor costs 1 to 2 us of attribute look-ups, so a decoding
// call on 13 layers spent 35 us on the host for 16 us of GPU work.
//
// recon_args(layers): the kq_recon_layer array (include/kq.h) of a list of dicts as
// kq_reconstruct_stack takes them.  Returns (array as bytes, list of W_hat tensors, device index,
// whether any layer asks for its squared error), or None when a layer is anything but the plain
// case (plain contiguous tensors of the right types and shapes on one GPU, the outputs given): the
// caller then goes through its own checks, which convert, allocate or raise.
//
// The calls of the 4-bit and 8-bit fully-connected layers, of the 8-bit checkpoints and of distillation (group_linear and
// the others below) do the whole call here in the plain case: checks, outputs, scratch and the library call.  A call
// on one token runs a few microseconds on the GPU; in Python its checks and its sixteen arguments took
// 10 us (here 4.3, of which the launch is about 3).  They return the outputs, or None where anything is not plain or the library refuses: the
// caller then goes through its own checks, which convert or raise.  bind(addresses, stream, scratch) gives
// them the library's functions, the current stream's handle by device index, and the scratch buffers.
#define PY_SSIZE_T_CLEAN
#include <ATen/ops/empty.h>
#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/autograd/python_variable.h>

#include <array>
#include <string>
#include <vector>

#include "kq.h"

namespace {

// the item of a dict as a plain GPU tensor: 1 yes, 0 absent or None, -1 anything else
int tensor_item(PyObject* dict, const char* key, c10::ScalarType type, at::Tensor& out) {
    PyObject* const o = PyDict_GetItemString(dict, key);  // borrowed
    if (o == nullptr || o == Py_None) return 0;
    if (!THPVariable_CheckExact(o)) return -1;
    out = THPVariable_Unpack(o);
    return out.is_cuda() && out.scalar_type() == type && out.layout() == c10::kStrided && out.is_contiguous() ? 1 : -1;
}

bool rows9(const at::Tensor& t) { return t.dim() == 2 && t.size(1) == KQ_DIM; }

bool int_item(PyObject* dict, const char* key, bool required, int64_t& v) {
    PyObject* const o = PyDict_GetItemString(dict, key);
    if (o == nullptr) return !required;
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}

// one layer's descriptor and output; false: not the plain case
bool recon_layer(PyObject* d, kq_recon_layer& r, at::Tensor& W, c10::Device& dev, bool first, bool& any_sq) {
    if (!PyDict_CheckExact(d)) return false;
    at::Tensor C, idx, packed, ref, sq;
    int64_t n = 0, bits = 0;
    if (tensor_item(d, "C", at::kFloat, C) != 1 || !rows9(C)) return false;
    if (!int_item(d, "n", true, n) || !int_item(d, "bits", false, bits)) return false;
    if (n < 1 || n > INT32_MAX || bits < 0 || bits > 16 || C.size(0) > INT32_MAX) return false;
    if (first) dev = C.device();
    const int hi = tensor_item(d, "idx", at::kInt, idx);
    if (hi < 0 || (hi == 1 && (idx.dim() != 1 || idx.size(0) != n))) return false;
    if (hi == 0 && tensor_item(d, "packed", at::kByte, packed) != 1) return false;
    if (tensor_item(d, "W_hat", at::kFloat, W) != 1 || !rows9(W) || W.size(0) != n) return false;
    const int hr = tensor_item(d, "W_ref", at::kFloat, ref), hs = tensor_item(d, "sq_error", at::kDouble, sq);
    if (hr < 0 || hs < 0 || (hr == 1 && !rows9(ref))) return false;
    if (C.device() != dev || W.device() != dev) return false;
    r.idx = hi ? (const int32_t*)idx.data_ptr() : nullptr;
    r.packed = hi ? nullptr : (const uint8_t*)packed.data_ptr();
    r.bits = (int32_t)bits;
    r.k = (int32_t)C.size(0);
    r.n = n;
    r.C = (const float*)C.data_ptr();
    r.W_hat = (float*)W.data_ptr();
    r.W_ref = hr ? (const float*)ref.data_ptr() : nullptr;
    r.sq_error = hs ? (double*)sq.data_ptr() : nullptr;
    any_sq |= hs == 1;
    return true;
}

PyObject* recon_args(PyObject*, PyObject* layers) {
    try {
        if (!PyList_CheckExact(layers)) Py_RETURN_NONE;
        const Py_ssize_t m = PyList_GET_SIZE(layers);
        if (m < 1 || m > KQ_MAX_STACK) Py_RETURN_NONE;
        kq_recon_layer arr[KQ_MAX_STACK] = {};
        std::vector<at::Tensor> W((size_t)m);
        c10::Device dev(c10::kCPU);
        bool any_sq = false;
        for (Py_ssize_t q = 0; q < m; ++q)
            if (!recon_layer(PyList_GET_ITEM(layers, q), arr[q], W[(size_t)q], dev, q == 0, any_sq)) Py_RETURN_NONE;
        PyObject* const outs = PyList_New(m);
        if (outs == nullptr) return nullptr;
        for (Py_ssize_t q = 0; q < m; ++q) {
            PyObject* const o = THPVariable_Wrap(W[(size_t)q]);
            if (o == nullptr) {
                Py_DECREF(outs);
                return nullptr;
            }
            PyList_SET_ITEM(outs, q, o);
        }
        return Py_BuildValue("(y#NiO)", (const char*)arr, (Py_ssize_t)(sizeof(kq_recon_layer) * (size_t)m), outs,
                             (int)dev.index(), any_sq ? Py_True : Py_False);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// ---- the 4-bit fully-connected layer and the 8-bit checkpoints ------------------------------------------

struct Library {
    decltype(&kq_quantize_groups) quantize = nullptr;
    decltype(&kq_reconstruct_groups) reconstruct = nullptr;
    decltype(&kq_group_linear_workspace_bytes) linear_ws = nullptr;
    decltype(&kq_group_linear) linear = nullptr;
    decltype(&kq_group_linear_grad_input_workspace_bytes) grad_input_ws = nullptr;
    decltype(&kq_group_linear_grad_input) grad_input = nullptr;
    decltype(&kq_checkpoint_pack) pack = nullptr;
    decltype(&kq_checkpoint_restore) restore = nullptr;
    decltype(&kq_checkpoint_grad_workspace_bytes) grad_ws = nullptr;
    decltype(&kq_checkpoint_grad_scales) grad_scales = nullptr;
    decltype(&kq_checkpoint_grad_weight) grad_weight = nullptr;
    decltype(&kq_quantize_blocks) quantize_blocks = nullptr;
    decltype(&kq_reconstruct_blocks) reconstruct_blocks = nullptr;
    decltype(&kq_block_linear_workspace_bytes) block_linear_ws = nullptr;
    decltype(&kq_block_linear) block_linear = nullptr;
    decltype(&kq_block_linear_grad_input_workspace_bytes) block_grad_input_ws = nullptr;
    decltype(&kq_block_linear_grad_input) block_grad_input = nullptr;
    decltype(&kq_block_linear_grad_weight_workspace_bytes) block_grad_weight_ws = nullptr;
    decltype(&kq_block_linear_grad_weight) block_grad_weight = nullptr;
    decltype(&kq_distill_workspace_bytes) distill_ws = nullptr;
    decltype(&kq_distill) distill = nullptr;
    decltype(&kq_distill_loss) distill_loss = nullptr;
    decltype(&kq_distill_grad) distill_grad = nullptr;
    PyObject* stream = nullptr;   // device index -> stream handle
    PyObject* scratch = nullptr;  // (torch.device, bytes) -> uint8 tensor
} g_lib;

PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t count) {
    constexpr int kFunctions = 23;
    if (count != 3 || !PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != kFunctions) {
        PyErr_SetString(PyExc_TypeError, "bind(23 addresses, stream, scratch)");
        return nullptr;
    }
    void* f[kFunctions];
    for (int i = 0; i < kFunctions; ++i) {
        f[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(a[0], i));
        if (PyErr_Occurred()) return nullptr;
    }
    Library l;
    l.quantize = (decltype(l.quantize))f[0];
    l.reconstruct = (decltype(l.reconstruct))f[1];
    l.linear_ws = (decltype(l.linear_ws))f[2];
    l.linear = (decltype(l.linear))f[3];
    l.grad_input_ws = (decltype(l.grad_input_ws))f[4];
    l.grad_input = (decltype(l.grad_input))f[5];
    l.pack = (decltype(l.pack))f[6];
    l.restore = (decltype(l.restore))f[7];
    l.grad_ws = (decltype(l.grad_ws))f[8];
    l.grad_scales = (decltype(l.grad_scales))f[9];
    l.grad_weight = (decltype(l.grad_weight))f[10];
    l.quantize_blocks = (decltype(l.quantize_blocks))f[11];
    l.reconstruct_blocks = (decltype(l.reconstruct_blocks))f[12];
    l.block_linear_ws = (decltype(l.block_linear_ws))f[13];
    l.block_linear = (decltype(l.block_linear))f[14];
    l.block_grad_input_ws = (decltype(l.block_grad_input_ws))f[15];
    l.block_grad_input = (decltype(l.block_grad_input))f[16];
    l.block_grad_weight_ws = (decltype(l.block_grad_weight_ws))f[17];
    l.block_grad_weight = (decltype(l.block_grad_weight))f[18];
    l.distill_ws = (decltype(l.distill_ws))f[19];
    l.distill = (decltype(l.distill))f[20];
    l.distill_loss = (decltype(l.distill_loss))f[21];
    l.distill_grad = (decltype(l.distill_grad))f[22];
    l.stream = Py_NewRef(a[1]);
    l.scratch = Py_NewRef(a[2]);
    g_lib = l;  // (bound once, when the binding is imported)
    Py_RETURN_NONE;
}

// One call's arguments.  Everything that is not plain sets ok to false.
struct Call {
    bool ok = g_lib.stream != nullptr;
    c10::Device dev{c10::kCPU};

    static int32_t type_of(const at::Tensor& t) {
        return t.scalar_type() == at::kFloat ? KQ_T_F32 : t.scalar_type() == at::kBFloat16 ? KQ_T_BF16
               : t.scalar_type() == at::kHalf ? KQ_T_F16 : -1;
    }
    // a plain tensor on the call's GPU (the first one decides which)
    at::Tensor tensor(PyObject* o) {
        if (!ok || !THPVariable_CheckExact(o)) {
            ok = false;
            return {};
        }
        at::Tensor t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.layout() != c10::kStrided || (dev.is_cuda() && t.device() != dev)) {
            ok = false;
            return {};
        }
        dev = t.device();
        return t;
    }
    at::Tensor dense(PyObject* o, at::ScalarType type, c10::IntArrayRef shape) {
        at::Tensor t = tensor(o);
        if (ok) ok = t.scalar_type() == type && t.is_contiguous() && t.sizes() == shape;
        return t;
    }
    // a matrix of rows with a pitch
    at::Tensor rows(PyObject* o, int64_t& ld) {
        at::Tensor t = tensor(o);
        if (ok) ok = t.dim() == 2 && t.size(1) > 0 && type_of(t) >= 0;
        if (ok) {
            ld = t.size(0) > 1 ? t.stride(0) : t.size(1);
            ok = (t.size(1) == 1 || t.stride(1) == 1) && ld >= t.size(1);
        }
        return t;
    }
    int64_t integer(PyObject* o) {
        int overflow = 0;
        if (!ok || !PyLong_CheckExact(o)) {
            ok = false;
            return 0;
        }
        const int64_t v = PyLong_AsLongLongAndOverflow(o, &overflow);
        ok = overflow == 0 && v >= 1 && v <= INT32_MAX;
        return v;
    }
    int64_t groups(int64_t k, int64_t group) {
        ok = ok && (group == 32 || group == 64 || group == 128);
        return ok ? (k + group - 1) / group : 0;
    }
    static std::array<int64_t, 4> code_shape(int64_t n, int64_t k) { return {(n + 15) / 16, (k + 127) / 128, 16, 64}; }
    const void* levels(PyObject* o) {
        if (o == Py_None) return nullptr;
        const at::Tensor t = dense(o, at::kBFloat16, {16});
        return ok ? t.data_ptr() : nullptr;
    }
    at::Tensor make(c10::IntArrayRef shape, at::ScalarType type) {
        return at::empty(shape, at::TensorOptions().dtype(type).device(dev));
    }
    void* stream() {
        PyObject* const i = PyLong_FromLong(dev.index());
        PyObject* const h = i ? PyObject_CallOneArg(g_lib.stream, i) : nullptr;
        Py_XDECREF(i);
        void* const s = h ? PyLong_AsVoidPtr(h) : nullptr;
        Py_XDECREF(h);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            ok = false;
        }
        return s;
    }
    // the same for a device that is the current one (the general path makes it current)
    void* current_stream() {
        if (ok && c10::impl::VirtualGuardImpl(dev.type()).getDevice() != dev) ok = false;
        return ok ? stream() : nullptr;
    }
    // scratch of the current stream, as the general path takes it
    at::Tensor scratch(size_t bytes) {
        if (!ok || bytes == 0) return {};
        PyObject* const d = THPDevice_New(dev);
        PyObject* const n = PyLong_FromSize_t(bytes);
        PyObject* args[2] = {d, n};
        PyObject* const w = d && n ? PyObject_Vectorcall(g_lib.scratch, args, 2, nullptr) : nullptr;
        Py_XDECREF(d);
        Py_XDECREF(n);
        at::Tensor t;
        if (w && THPVariable_CheckExact(w)) t = THPVariable_Unpack(w);
        else ok = false;
        Py_XDECREF(w);
        if (PyErr_Occurred()) PyErr_Clear();
        return t;
    }
};
void* address(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
size_t bytes_of(const at::Tensor& t) { return t.defined() ? (size_t)t.numel() : 0; }

template <class F>
PyObject* guarded(Py_ssize_t count, Py_ssize_t want, F f) {
    if (count != want) {
        PyErr_SetString(PyExc_TypeError, "wrong number of arguments");
        return nullptr;
    }
    try {
        PyObject* const r = f();
        if (r == nullptr && !PyErr_Occurred()) Py_RETURN_NONE;  // not the plain case
        return r;
    } catch (const std::exception&) {  // (out of memory, say: the general path says so)
        Py_RETURN_NONE;
    }
}
PyObject* pair(const at::Tensor& a, const at::Tensor& b) {
    PyObject* const x = THPVariable_Wrap(a);
    PyObject* const y = b.defined() ? THPVariable_Wrap(b) : Py_NewRef(Py_None);
    PyObject* const t = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return t;
}
constexpr int64_t kCk = KQ_CHECKPOINT_GROUP;

// (W, group, levels)
PyObject* quantize_groups(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 3, [&]() -> PyObject* {
        Call c;
        int64_t ld = 0;
        const at::Tensor W = c.rows(a[0], ld);
        const int64_t group = c.integer(a[1]);
        const void* const levels = c.levels(a[2]);
        if (!c.ok || W.size(0) < 1) return nullptr;
        const int64_t n = W.size(0), k = W.size(1), G = c.groups(k, group);
        void* const s = c.stream();
        if (!c.ok) return nullptr;
        const at::Tensor codes = c.make(Call::code_shape(n, k), at::kByte), scales = c.make({n, G}, at::kBFloat16);
        if (g_lib.quantize(W.data_ptr(), Call::type_of(W), ld, n, k, (int32_t)group, levels, (uint8_t*)codes.data_ptr(),
                           scales.data_ptr(), s) != KQ_OK)
            return nullptr;
        return pair(codes, scales);
    });
}

// codes, scales (or None) and levels of an [n, k] weight
struct Weights {
    const uint8_t* codes = nullptr;
    const void* scales = nullptr;
    const void* levels = nullptr;
    Weights(Call& c, PyObject* codes_o, PyObject* scales_o, PyObject* levels_o, int64_t n, int64_t k, int64_t group) {
        const int64_t G = c.groups(k, group);
        if (!c.ok) return;
        const at::Tensor t = c.dense(codes_o, at::kByte, Call::code_shape(n, k));
        if (scales_o) {
            const at::Tensor u = c.dense(scales_o, at::kBFloat16, {n, G});
            if (c.ok) scales = u.data_ptr();
        }
        levels = c.levels(levels_o);
        if (c.ok) codes = (const uint8_t*)t.data_ptr();
    }
};
int64_t rows_of(PyObject* o) {  // size(0) of a matrix, 0 for anything else
    if (!THPVariable_CheckExact(o)) return 0;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.dim() == 2 ? t.size(0) : 0;
}

// (codes, scales, k, group, levels, dtype's type number)
PyObject* reconstruct_groups(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 6, [&]() -> PyObject* {
        Call c;
        const int64_t k = c.integer(a[2]), group = c.integer(a[3]), n = rows_of(a[1]);
        if (!c.ok || n < 1) return nullptr;
        const Weights w(c, a[0], a[1], a[4], n, k, group);
        if (!c.ok || !PyLong_CheckExact(a[5])) return nullptr;
        const long type = PyLong_AsLong(a[5]);
        void* const s = c.stream();
        if (!c.ok || type < 0 || type > 2) return nullptr;
        const at::Tensor W = c.make({n, k}, type == KQ_T_F32 ? at::kFloat : type == KQ_T_BF16 ? at::kBFloat16 : at::kHalf);
        if (g_lib.reconstruct(w.codes, w.scales, w.levels, n, k, (int32_t)group, (int32_t)type, W.data_ptr(), k, s) != KQ_OK)
            return nullptr;
        return THPVariable_Wrap(W);
    });
}

// (X, codes, scales, group, levels, bias, Y)
PyObject* group_linear(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 7, [&]() -> PyObject* {
        Call c;
        int64_t ldx = 0, ldy = 0;
        const at::Tensor X = c.rows(a[0], ldx);
        const int64_t group = c.integer(a[3]), n = rows_of(a[2]);
        if (!c.ok || n < 1 || X.scalar_type() == at::kFloat) return nullptr;
        const int64_t m = X.size(0), k = X.size(1);
        const Weights w(c, a[1], a[2], a[4], n, k, group);
        const float* bias = nullptr;
        if (a[5] != Py_None) {
            const at::Tensor b = c.dense(a[5], at::kFloat, {n});
            if (c.ok) bias = (const float*)b.data_ptr();
        }
        at::Tensor Y;
        if (a[6] != Py_None) {
            Y = c.rows(a[6], ldy);
            if (!c.ok || Y.scalar_type() != X.scalar_type() || Y.size(0) != m || Y.size(1) != n) return nullptr;
        }
        void* const s = c.stream();
        if (!c.ok) return nullptr;
        const at::Tensor ws = c.scratch(g_lib.linear_ws(X.data_ptr(), ldx, m, n, k));
        if (!Y.defined()) {
            Y = c.make({m, n}, X.scalar_type());
            ldy = n;
        }
        if (!c.ok || g_lib.linear(X.data_ptr(), Call::type_of(X), ldx, m, n, k, w.codes, w.scales, w.levels, (int32_t)group, bias,
                                  Y.data_ptr(), ldy, address(ws), bytes_of(ws), s) != KQ_OK)
            return nullptr;
        return a[6] != Py_None ? Py_NewRef(a[6]) : THPVariable_Wrap(Y);
    });
}

// (dY, codes, scales, k, group, levels, dX)
PyObject* grad_input(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 7, [&]() -> PyObject* {
        Call c;
        int64_t ldy = 0, ldx = 0;
        const at::Tensor dY = c.rows(a[0], ldy);
        const int64_t k = c.integer(a[3]), group = c.integer(a[4]);
        if (!c.ok || dY.scalar_type() == at::kFloat) return nullptr;
        const int64_t m = dY.size(0), n = dY.size(1);
        const Weights w(c, a[1], a[2], a[5], n, k, group);
        at::Tensor dX;
        if (a[6] != Py_None) {
            dX = c.rows(a[6], ldx);
            if (!c.ok || dX.scalar_type() != dY.scalar_type() || dX.size(0) != m || dX.size(1) != k) return nullptr;
        }
        void* const s = c.stream();
        if (!c.ok) return nullptr;
        const at::Tensor ws = c.scratch(g_lib.grad_input_ws(dY.data_ptr(), ldy, m, n, k));
        if (!dX.defined()) {
            dX = c.make({m, k}, dY.scalar_type());
            ldx = k;
        }
        if (!c.ok || g_lib.grad_input(dY.data_ptr(), Call::type_of(dY), ldy, m, n, k, w.codes, w.scales, w.levels, (int32_t)group,
                                      dX.data_ptr(), ldx, address(ws), bytes_of(ws), s) != KQ_OK)
            return nullptr;
        return a[6] != Py_None ? Py_NewRef(a[6]) : THPVariable_Wrap(dX);
    });
}

// (X)
PyObject* checkpoint_pack(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 1, [&]() -> PyObject* {
        Call c;
        int64_t ld = 0;
        const at::Tensor X = c.rows(a[0], ld);
        if (!c.ok) return nullptr;
        void* const s = c.stream();
        if (!c.ok) return nullptr;
        const int64_t m = X.size(0), k = X.size(1), g = (k + kCk - 1) / kCk;
        const at::Tensor q = c.make({m, g * kCk}, at::kChar), e = c.make({m, g}, at::kByte);
        if (g_lib.pack(X.data_ptr(), Call::type_of(X), ld, m, k, (int8_t*)q.data_ptr(), (uint8_t*)e.data_ptr(), s) != KQ_OK)
            return nullptr;
        return pair(q, e);
    });
}

// q and exps of a checkpoint of k columns
struct Checkpoint {
    int64_t m = 0;
    const int8_t* q = nullptr;
    const uint8_t* exps = nullptr;
    Checkpoint(Call& c, PyObject* q_o, PyObject* exps_o, int64_t k) {
        m = rows_of(q_o);
        const int64_t g = (k + kCk - 1) / kCk;
        if (!c.ok) return;
        const at::Tensor t = c.dense(q_o, at::kChar, {m, g * kCk}), e = c.dense(exps_o, at::kByte, {m, g});
        if (!c.ok) return;
        q = (const int8_t*)t.data_ptr();
        exps = (const uint8_t*)e.data_ptr();
    }
};

// (q, exps, k, dtype's type number)
PyObject* checkpoint_restore(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 4, [&]() -> PyObject* {
        Call c;
        const int64_t k = c.integer(a[2]);
        const Checkpoint ck(c, a[0], a[1], k);
        if (!c.ok || !PyLong_CheckExact(a[3])) return nullptr;
        const long type = PyLong_AsLong(a[3]);
        void* const s = c.stream();
        if (!c.ok || type < 0 || type > 2) return nullptr;
        const at::Tensor X = c.make({ck.m, k}, type == KQ_T_F32 ? at::kFloat : type == KQ_T_BF16 ? at::kBFloat16 : at::kHalf);
        if (g_lib.restore(ck.q, ck.exps, ck.m, k, (int32_t)type, X.data_ptr(), k, s) != KQ_OK) return nullptr;
        return THPVariable_Wrap(X);
    });
}

// (dY, q, exps, codes, k, group, levels, bias)
PyObject* grad_scales(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 8, [&]() -> PyObject* {
        Call c;
        int64_t ldy = 0;
        const at::Tensor dY = c.rows(a[0], ldy);
        const int64_t k = c.integer(a[4]), group = c.integer(a[5]);
        if (!c.ok || dY.scalar_type() == at::kFloat || (a[7] != Py_True && a[7] != Py_False)) return nullptr;
        const int64_t m = dY.size(0), n = dY.size(1), G = c.groups(k, group);
        const Checkpoint ck(c, a[1], a[2], k);
        const Weights w(c, a[3], nullptr, a[6], n, k, group);
        if (!c.ok || ck.m != m) return nullptr;
        void* const s = c.stream();
        const at::Tensor ws = c.scratch(g_lib.grad_ws(m, n, k, (int32_t)group));
        if (!c.ok) return nullptr;
        const at::Tensor ds = c.make({n, G}, at::kFloat);
        at::Tensor db;
        if (a[7] == Py_True) db = c.make({n}, at::kFloat);
        if (g_lib.grad_scales(dY.data_ptr(), Call::type_of(dY), ldy, m, n, k, ck.q, ck.exps, w.codes, w.levels, (int32_t)group,
                              (float*)ds.data_ptr(), (float*)address(db), address(ws), bytes_of(ws), s) != KQ_OK)
            return nullptr;
        return pair(ds, db);
    });
}

// (dY, q, exps, k, bias)
PyObject* grad_weight(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 5, [&]() -> PyObject* {
        Call c;
        int64_t ldy = 0;
        const at::Tensor dY = c.rows(a[0], ldy);
        const int64_t k = c.integer(a[3]);
        if (!c.ok || dY.scalar_type() == at::kFloat || (a[4] != Py_True && a[4] != Py_False)) return nullptr;
        const int64_t m = dY.size(0), n = dY.size(1);
        const Checkpoint ck(c, a[1], a[2], k);
        if (!c.ok || ck.m != m) return nullptr;
        void* const s = c.stream();
        const at::Tensor ws = c.scratch(g_lib.grad_ws(m, n, k, 0));
        if (!c.ok) return nullptr;
        const at::Tensor dW = c.make({n, k}, at::kFloat);
        at::Tensor db;
        if (a[4] == Py_True) db = c.make({n}, at::kFloat);
        if (g_lib.grad_weight(dY.data_ptr(), Call::type_of(dY), ldy, m, n, k, ck.q, ck.exps, (float*)dW.data_ptr(), k,
                              (float*)address(db), address(ws), bytes_of(ws), s) != KQ_OK)
            return nullptr;
        return pair(dW, db);
    });
}

// ---- the 8-bit fully-connected layer --------------------------------------------------------------------

constexpr int64_t kBlock = KQ_BLOCK;
at::ScalarType scalar_of(int64_t type) { return type == KQ_T_F32 ? at::kFloat : type == KQ_T_BF16 ? at::kBFloat16 : at::kHalf; }

// dtype's type number, -1 for None; anything else is not plain
int64_t type_number(Call& c, PyObject* o) {
    if (!PyLong_CheckExact(o)) {
        c.ok = false;
        return -1;
    }
    const long v = PyLong_AsLong(o);
    c.ok = c.ok && v >= -1 && v <= 2;
    return v;
}

// values and exponents of an 8-bit matrix of k columns (0: as many as there are)
struct Blocks {
    int64_t m = 0, k = 0;
    const uint8_t* values = nullptr;
    const uint8_t* exps = nullptr;
    Blocks(Call& c, PyObject* values_o, PyObject* exps_o, int64_t k_, int64_t rows) {
        at::Tensor t = c.tensor(values_o);
        c.ok = c.ok && t.dim() == 2 && t.scalar_type() == at::kFloat8_e4m3fn && t.is_contiguous();
        if (!c.ok) return;
        m = t.size(0);
        k = k_ > 0 ? k_ : t.size(1);
        const int64_t kb = (k + kBlock - 1) / kBlock;
        const at::Tensor e = c.dense(exps_o, at::kByte, {(m + rows - 1) / rows, kb});
        c.ok = c.ok && m > 0 && kb > 0 && t.size(1) == kb * kBlock;
        if (!c.ok) return;
        values = (const uint8_t*)t.data_ptr();
        exps = (const uint8_t*)e.data_ptr();
    }
};

// (X, rows)
PyObject* quantize_blocks(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 2, [&]() -> PyObject* {
        Call c;
        int64_t ld = 0;
        const at::Tensor X = c.rows(a[0], ld);
        const int64_t rows = c.integer(a[1]);
        if (!c.ok || (rows != 1 && rows != kBlock)) return nullptr;
        void* const s = c.current_stream();
        if (!c.ok) return nullptr;
        const int64_t m = X.size(0), k = X.size(1), kb = (k + kBlock - 1) / kBlock;
        const at::Tensor v = c.make({m, kb * kBlock}, at::kFloat8_e4m3fn), e = c.make({(m + rows - 1) / rows, kb}, at::kByte);
        if (g_lib.quantize_blocks(X.data_ptr(), Call::type_of(X), ld, m, k, (int32_t)rows, (uint8_t*)v.data_ptr(), (uint8_t*)e.data_ptr(), s) != KQ_OK)
            return nullptr;
        return pair(v, e);
    });
}

// (values, exps, k, rows, dtype's type number)
PyObject* reconstruct_blocks(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 5, [&]() -> PyObject* {
        Call c;
        const int64_t k = c.integer(a[2]), rows = c.integer(a[3]), type = type_number(c, a[4]);
        if (!c.ok || (rows != 1 && rows != kBlock) || type < 0) return nullptr;
        const Blocks w(c, a[0], a[1], k, rows);
        if (!c.ok) return nullptr;
        void* const s = c.current_stream();
        if (!c.ok) return nullptr;
        const at::Tensor X = c.make({w.m, k}, scalar_of(type));
        if (g_lib.reconstruct_blocks(w.values, w.exps, w.m, k, (int32_t)rows, (int32_t)type, X.data_ptr(), k, s) != KQ_OK) return nullptr;
        return THPVariable_Wrap(X);
    });
}

// (X, values, exps, bias, x_exps, dtype's type number or -1, Y)
PyObject* block_linear(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 7, [&]() -> PyObject* {
        Call c;
        int64_t m, k, ldx = 0, type = type_number(c, a[5]);
        int32_t xt;
        const void* x;
        const uint8_t* xe = nullptr;
        if (a[4] == Py_None) {
            const at::Tensor X = c.rows(a[0], ldx);
            if (!c.ok) return nullptr;
            m = X.size(0), k = X.size(1), xt = Call::type_of(X), x = X.data_ptr();
        } else {
            const Blocks q(c, a[0], a[4], 0, 1);
            if (!c.ok) return nullptr;
            m = q.m, k = ldx = q.k, xt = KQ_T_E4M3, x = q.values, xe = q.exps;
        }
        const Blocks w(c, a[1], a[2], k, kBlock);
        const float* bias = nullptr;
        if (a[3] != Py_None) {
            const at::Tensor b = c.dense(a[3], at::kFloat, {w.m});
            if (c.ok) bias = (const float*)b.data_ptr();
        }
        at::Tensor Y;
        int64_t ldy = w.m;
        if (a[6] != Py_None) {
            Y = c.rows(a[6], ldy);
            if (!c.ok || Y.size(0) != m || Y.size(1) != w.m || (type >= 0 && Call::type_of(Y) != type)) return nullptr;
            type = Call::type_of(Y);
        }
        if (type < 0) type = xt == KQ_T_E4M3 ? KQ_T_BF16 : xt;
        if (!c.ok) return nullptr;
        void* const s = c.current_stream();
        const at::Tensor ws = c.scratch(g_lib.block_linear_ws(xt, (int32_t)type, m, w.m, k));
        if (!c.ok) return nullptr;
        if (!Y.defined()) Y = c.make({m, w.m}, scalar_of(type));
        if (g_lib.block_linear(x, xt, ldx, xe, m, w.m, k, w.values, w.exps, bias, Y.data_ptr(), (int32_t)type, ldy, address(ws), bytes_of(ws), s) != KQ_OK)
            return nullptr;
        return a[6] != Py_None ? Py_NewRef(a[6]) : THPVariable_Wrap(Y);
    });
}

// (dY, values, exps, k, dX)
PyObject* block_grad_input(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 5, [&]() -> PyObject* {
        Call c;
        int64_t ldy = 0, ldx = 0;
        const at::Tensor dY = c.rows(a[0], ldy);
        const int64_t k = c.integer(a[3]);
        if (!c.ok) return nullptr;
        const Blocks w(c, a[1], a[2], k, kBlock);
        const int64_t m = dY.size(0), n = dY.size(1);
        const int32_t type = Call::type_of(dY);
        if (!c.ok || w.m != n) return nullptr;
        at::Tensor dX;
        if (a[4] != Py_None) {
            dX = c.rows(a[4], ldx);
            if (!c.ok || dX.scalar_type() != dY.scalar_type() || dX.size(0) != m || dX.size(1) != k) return nullptr;
        }
        void* const s = c.current_stream();
        const at::Tensor ws = c.scratch(g_lib.block_grad_input_ws(type, m, n, k));
        if (!c.ok) return nullptr;
        if (!dX.defined()) {
            dX = c.make({m, k}, dY.scalar_type());
            ldx = k;
        }
        if (g_lib.block_grad_input(dY.data_ptr(), type, ldy, m, n, k, w.values, w.exps, dX.data_ptr(), ldx, address(ws), bytes_of(ws), s) != KQ_OK)
            return nullptr;
        return a[4] != Py_None ? Py_NewRef(a[4]) : THPVariable_Wrap(dX);
    });
}

// (dY, x_values, x_exps, k, bias, dtype's type number)
PyObject* block_grad_weight(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 6, [&]() -> PyObject* {
        Call c;
        int64_t ldy = 0;
        const at::Tensor dY = c.rows(a[0], ldy);
        const int64_t k = c.integer(a[3]), type = type_number(c, a[5]);
        if (!c.ok || type < 0 || (a[4] != Py_True && a[4] != Py_False)) return nullptr;
        const Blocks x(c, a[1], a[2], k, 1);
        const int64_t m = dY.size(0), n = dY.size(1);
        if (!c.ok || x.m != m) return nullptr;
        void* const s = c.current_stream();
        const at::Tensor ws = c.scratch(g_lib.block_grad_weight_ws((int32_t)type, m, n, k));
        if (!c.ok) return nullptr;
        const at::Tensor dW = c.make({n, k}, scalar_of(type));
        at::Tensor db;
        if (a[4] == Py_True) db = c.make({n}, at::kFloat);
        if (g_lib.block_grad_weight(dY.data_ptr(), Call::type_of(dY), ldy, m, n, k, x.values, x.exps, dW.data_ptr(), (int32_t)type, k,
                                    (float*)address(db), address(ws), bytes_of(ws), s) != KQ_OK)
            return nullptr;
        return pair(dW, db);
    });
}

// ---- distillation -----------------------------------------------------------------------------------------

float number(Call& c, PyObject* o) {
    if (!PyFloat_CheckExact(o)) {
        c.ok = false;
        return 0.0f;
    }
    return (float)PyFloat_AS_DOUBLE(o);
}
int32_t index_bytes(Call& c, const at::Tensor& t) {
    const int32_t b = t.scalar_type() == at::kLong ? 8 : t.scalar_type() == at::kInt ? 4 : 0;
    c.ok = c.ok && b != 0;
    return b;
}

// (Z, top_values, top_idx, temperature, labels, alpha): the first six arguments of each call
struct Distill {
    kq_distill_args args = {};
    at::Tensor Z;
    Distill(Call& c, PyObject* const* a) {
        Z = c.rows(a[0], args.ldz);
        const at::Tensor tv = c.tensor(a[1]), ti = c.tensor(a[2]);
        args.temperature = number(c, a[3]);
        args.alpha = number(c, a[5]);
        if (!c.ok || Z.size(0) < 1 || tv.dim() != 2 || !tv.is_contiguous() || !ti.is_contiguous() || ti.sizes() != tv.sizes() || tv.size(0) != Z.size(0) ||
            Call::type_of(tv) < 0) {
            c.ok = false;
            return;
        }
        args.Z = Z.data_ptr();
        args.type = Call::type_of(Z);
        args.m = Z.size(0);
        args.v = Z.size(1);
        args.top_values = tv.data_ptr();
        args.top_type = Call::type_of(tv);
        args.top_idx = ti.data_ptr();
        args.idx_bytes = index_bytes(c, ti);
        c.ok = c.ok && tv.size(1) >= 1 && tv.size(1) <= KQ_DISTILL_MAX_TOP;
        args.top = (int32_t)tv.size(1);
        if (a[4] != Py_None) {
            const at::Tensor y = c.tensor(a[4]);
            if (!c.ok || y.dim() != 1 || y.size(0) != args.m || !y.is_contiguous()) {
                c.ok = false;
                return;
            }
            args.labels = y.data_ptr();
            args.label_bytes = index_bytes(c, y);
        }
    }
};
const float* row_floats(Call& c, PyObject* o, int64_t m) {
    if (o == Py_None) return nullptr;
    const at::Tensor t = c.dense(o, at::kFloat, {m});
    return c.ok ? (const float*)t.data_ptr() : nullptr;
}
// dZ, given or made like Z
at::Tensor gradient(Call& c, PyObject* o, const at::Tensor& Z, int64_t& ld) {
    if (o == Py_None) {
        if (!c.ok) return {};
        ld = Z.size(1);
        return c.make(Z.sizes(), Z.scalar_type());
    }
    at::Tensor t = c.rows(o, ld);
    c.ok = c.ok && t.scalar_type() == Z.scalar_type() && t.sizes() == Z.sizes();
    return t;
}

// (.., scale, dloss, dZ)
PyObject* distill(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 9, [&]() -> PyObject* {
        Call c;
        const Distill d(c, a);
        const float scale = number(c, a[6]);
        if (!c.ok) return nullptr;
        const float* const dloss = row_floats(c, a[7], d.args.m);
        int64_t ld = 0;
        void* const s = c.current_stream();
        const at::Tensor ws = c.scratch(g_lib.distill_ws(d.args.type, d.args.m, d.args.v, d.args.top));
        const at::Tensor dZ = gradient(c, a[8], d.Z, ld);
        if (!c.ok) return nullptr;
        const at::Tensor loss = c.make({d.args.m}, at::kFloat);
        if (g_lib.distill(&d.args, dloss, scale, (float*)loss.data_ptr(), dZ.data_ptr(), ld, address(ws), bytes_of(ws), s) != KQ_OK) return nullptr;
        PyObject* const r = pair(loss, dZ);
        if (r && a[8] != Py_None && PyTuple_SetItem(r, 1, Py_NewRef(a[8])) != 0) {
            Py_DECREF(r);
            return nullptr;
        }
        return r;
    });
}

PyObject* distill_loss(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 6, [&]() -> PyObject* {
        Call c;
        const Distill d(c, a);
        if (!c.ok) return nullptr;
        void* const s = c.current_stream();
        const at::Tensor ws = c.scratch(g_lib.distill_ws(d.args.type, d.args.m, d.args.v, d.args.top));
        if (!c.ok) return nullptr;
        const at::Tensor loss = c.make({d.args.m}, at::kFloat), stats = c.make({d.args.m, 3}, at::kFloat);
        if (g_lib.distill_loss(&d.args, (float*)loss.data_ptr(), (float*)stats.data_ptr(), address(ws), bytes_of(ws), s) != KQ_OK) return nullptr;
        return pair(loss, stats);
    });
}

// (.., scale, stats, dloss, dZ)
PyObject* distill_grad(PyObject*, PyObject* const* a, Py_ssize_t count) {
    return guarded(count, 10, [&]() -> PyObject* {
        Call c;
        const Distill d(c, a);
        const float scale = number(c, a[6]);
        if (!c.ok) return nullptr;
        const at::Tensor stats = c.dense(a[7], at::kFloat, {d.args.m, 3});
        const float* const dloss = row_floats(c, a[8], d.args.m);
        int64_t ld = 0;
        void* const s = c.current_stream();
        const at::Tensor dZ = gradient(c, a[9], d.Z, ld);
        if (!c.ok) return nullptr;
        if (g_lib.distill_grad(&d.args, (const float*)stats.data_ptr(), dloss, scale, dZ.data_ptr(), ld, s) != KQ_OK) return nullptr;
        return a[9] != Py_None ? Py_NewRef(a[9]) : THPVariable_Wrap(dZ);
    });
}

#define KQ_FAST(NAME) {#NAME, (PyCFunction)(void (*)(void))NAME, METH_FASTCALL, "the plain case of a call, or None"}
PyMethodDef methods[] = {{"recon_args", recon_args, METH_O, "descriptor array of kq_reconstruct_stack, or None"},
                         {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, "the library's functions, stream, scratch"},
                         KQ_FAST(quantize_groups),
                         KQ_FAST(reconstruct_groups),
                         KQ_FAST(group_linear),
                         KQ_FAST(grad_input),
                         KQ_FAST(checkpoint_pack),
                         KQ_FAST(checkpoint_restore),
                         KQ_FAST(grad_scales),
                         KQ_FAST(grad_weight),
                         KQ_FAST(quantize_blocks),
                         KQ_FAST(reconstruct_blocks),
                         KQ_FAST(block_linear),
                         KQ_FAST(block_grad_input),
                         KQ_FAST(block_grad_weight),
                         KQ_FAST(distill),
                         KQ_FAST(distill_loss),
                         KQ_FAST(distill_grad),
                         {nullptr, nullptr, 0, nullptr}};
#undef KQ_FAST
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kqhost", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kqhost(void) { return PyModule_Create(&module); }
