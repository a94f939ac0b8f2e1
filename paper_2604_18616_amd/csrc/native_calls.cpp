// The plain calls of the Python binding (attn_fwd, gemm_bf16, those of the quantised cache and rope_bf16 on torch's current
// stream, results allocated here) without Python's share of the work: checking the tensors, allocating the results and
// marshalling two dozen arguments takes longer there than a small kernel runs.  Host time per call on the machine measured,
// Python against this: attn_fwd with its keys cut 14.0 against 8.1 us, uncut 8.5 / 4.4, gemm_bf16 7.2 / 3.9; calls of a decoding
// step, host and GPU: attn_kv_fp8 21.4 / 9.9, kv_fp8_write 13.5 / 6.6, kv_fp8_read 15.8 / 7.2, rope_bf16 13.7 / 5.8.
//
// Each function returns None for everything that is not such a call, however slightly (another type, a subclass, a tensor of
// a transform, a wrong shape), and the Python code then does what it always did, errors included; it returns an int for
// an error code of the library.  The library's entry points arrive as addresses from the binding, which has it loaded.
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "../../include/attn_workspace.h"
#include "../../include/gemm_workspace.h"
#include "../../include/kv_cache.h"
#include "../../include/rope.h"

namespace {

using At = at::Tensor;
// The library's entry points, with the headers' own types.
struct Entries {
    decltype(&::attn_fwd) attn_fwd;
    decltype(&::attn_fwd_strided) attn_fwd_strided;
    decltype(&::attn_fwd_workspace_bytes) attn_fwd_workspace_bytes;
    decltype(&::attn_fwd_workspace) attn_fwd_workspace;
    decltype(&::gemm_bf16_workspace_bytes) gemm_bf16_workspace_bytes;
    decltype(&::gemm_bf16_tile) gemm_bf16_tile;
    decltype(&::gemm_bf16_workspace) gemm_bf16_workspace;
    decltype(&::kv_fp8_write) kv_fp8_write;
    decltype(&::kv_fp8_read) kv_fp8_read;
    decltype(&::attn_kv_fp8_workspace_bytes) attn_kv_fp8_workspace_bytes;
    decltype(&::attn_kv_fp8) attn_kv_fp8;
    decltype(&::rope_bf16) rope_bf16;
} entry = {};

// A torch.Tensor or Parameter proper whose memory is its values: on a GPU, no subclass, no tensor of a transform.
bool plain(PyObject* obj, int64_t dim, c10::ScalarType type = at::kBFloat16) {
    if (!THPVariable_CheckExact(obj)) return false;
    const At& t = THPVariable_Unpack(obj);
    constexpr c10::DispatchKeySet kStrange({c10::DispatchKey::Python, c10::DispatchKey::PythonTLSSnapshot, c10::DispatchKey::FuncTorchBatched,
                                            c10::DispatchKey::FuncTorchGradWrapper, c10::DispatchKey::Functionalize, c10::DispatchKey::BatchedNestedTensor,
                                            c10::DispatchKey::NestedTensor, c10::DispatchKey::ZeroTensor, c10::DispatchKey::Negative, c10::DispatchKey::Conjugate});
    return t.defined() && t.is_cuda() && t.layout() == c10::kStrided && t.scalar_type() == type && t.dim() == dim &&
           !t.key_set().has_any(kStrange) && (t.stride(dim - 1) == 1 || (t.size(dim - 1) == 1 && type != at::kBFloat16));
}
bool fits(int64_t v) { return v >= 0 && v < (int64_t(1) << 31); }

// Memory for a call's parts; undefined where there is none left: such a call runs uncut, as it would without it.
At scratch(size_t need, const At& like) {
    try {
        return at::empty({(int64_t)need}, like.options().dtype(at::kByte));
    } catch (const c10::OutOfMemoryError&) {
        return At();
    }
}
void* stream_of(const At& t) { return (void*)c10::hip::getCurrentHIPStream(t.get_device()).stream(); }

PyObject* attn(PyObject*, PyObject* const* args, Py_ssize_t n) {      // q, k, v, causal, scale
    HANDLE_TH_ERRORS
    if (!entry.attn_fwd || n != 5 || !plain(args[0], 4) || !plain(args[1], 4) || !plain(args[2], 4) || !PyBool_Check(args[3]) || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    const At &q = THPVariable_Unpack(args[0]), &k = THPVariable_Unpack(args[1]), &v = THPVariable_Unpack(args[2]);
    const int64_t B = q.size(0), Hq = q.size(1), Sq = q.size(2), D = q.size(3), Hkv = k.size(1), Sk = k.size(2);
    if (k.sizes() != v.sizes() || k.size(0) != B || k.size(3) != D || D == 0 || k.device() != q.device() || v.device() != q.device()) Py_RETURN_NONE;
    if (!fits(B) || !fits(Hq) || !fits(Sq) || !fits(D) || !fits(Hkv) || !fits(Sk)) Py_RETURN_NONE;
    double scale;
    if (args[4] == Py_None) scale = std::pow((double)D, -0.5);
    else if (PyFloat_CheckExact(args[4])) scale = PyFloat_AS_DOUBLE(args[4]);
    else Py_RETURN_NONE;
    const int causal = args[3] == Py_True;
    At o, lse;
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        o = at::empty_like(q);                       // keeps q's layout for dense views
        if (o.stride(3) != 1) rc = INT_MIN;
        else {
            lse = at::empty({B, Hq, Sq}, q.options().dtype(at::kFloat));
            void* const stream = stream_of(q);
            // few query rows or few heads: the keys are cut over workgroups too (the same conditions as in the Python code)
            const size_t need = Sq <= 64 || B * Hq * Sq <= 160 * 128 ? entry.attn_fwd_workspace_bytes(B, Hq, Hkv, Sq, Sk, D) : 0;
            At ws;
            if (need && (Sk + 64) * std::max(k.stride(2), v.stride(2)) < (int64_t(1) << 31)) ws = scratch(need, q);
            const long long qs[3] = {q.stride(0), q.stride(1), q.stride(2)}, ks[3] = {k.stride(0), k.stride(1), k.stride(2)},
                            vs[3] = {v.stride(0), v.stride(1), v.stride(2)}, os[3] = {o.stride(0), o.stride(1), o.stride(2)};
            if (ws.defined())
                rc = entry.attn_fwd_workspace(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), (float*)lse.data_ptr(), B, Hq, Hkv, Sq, Sk, D, qs, ks, vs, os,
                                              causal, (float)scale, ws.data_ptr(), need, (int)(need / (4 * (size_t)B * Hq * Sq * (D + 2))), stream);
            else if (q.is_contiguous() && k.is_contiguous() && v.is_contiguous() && o.is_contiguous())
                rc = entry.attn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), (float*)lse.data_ptr(), B, Hq, Hkv, Sq, Sk, D, causal, (float)scale, stream);
            else
                rc = entry.attn_fwd_strided(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), (float*)lse.data_ptr(), B, Hq, Hkv, Sq, Sk, D, qs, ks, vs, os,
                                            causal, (float)scale, stream);
        }
    }
    if (rc == INT_MIN) Py_RETURN_NONE;
    if (rc != 0) return PyLong_FromLong(rc);
    PyObject* const out[2] = {THPVariable_Wrap(std::move(o)), THPVariable_Wrap(std::move(lse))};
    PyObject* const both = PyTuple_Pack(2, out[0], out[1]);
    Py_XDECREF(out[0]);
    Py_XDECREF(out[1]);
    return both;
    END_HANDLE_TH_ERRORS
}

PyObject* gemm(PyObject*, PyObject* const* args, Py_ssize_t n) {      // a, b, b_is_nk
    HANDLE_TH_ERRORS
    if (!entry.attn_fwd || n != 3 || !plain(args[0], 2) || !plain(args[1], 2) || !PyBool_Check(args[2]) || at::impl::torch_function_mode_enabled()) Py_RETURN_NONE;
    const At &a = THPVariable_Unpack(args[0]), &b = THPVariable_Unpack(args[1]);
    const int nk = args[2] == Py_True;
    const int64_t M = a.size(0), K = a.size(1), N = b.size(nk ? 0 : 1);
    if (b.size(nk ? 1 : 0) != K || b.device() != a.device() || !fits(M) || !fits(N) || !fits(K)) Py_RETURN_NONE;
    At c;
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        c = at::empty({M, N}, a.options());
        void* const stream = stream_of(a);
        // results of few tiles: k is cut over workgroups too, for operands whose rows start at multiples of 16 bytes
        const size_t need = entry.gemm_bf16_workspace_bytes(M, N, K);
        At ws;
        if (need && !((((uintptr_t)a.data_ptr() | (uintptr_t)b.data_ptr() | (uintptr_t)c.data_ptr()) & 15) || ((a.stride(0) | b.stride(0) | c.stride(0)) & 7)))
            ws = scratch(need, a);
        if (ws.defined())
            rc = entry.gemm_bf16_workspace(a.data_ptr(), b.data_ptr(), c.data_ptr(), M, N, K, a.stride(0), b.stride(0), c.stride(0), nk, 0, 0, ws.data_ptr(), need, stream);
        else
            rc = entry.gemm_bf16_tile(a.data_ptr(), b.data_ptr(), c.data_ptr(), M, N, K, a.stride(0), b.stride(0), c.stride(0), nk, 0, stream);
    }
    if (rc != 0) return PyLong_FromLong(rc);
    return THPVariable_Wrap(std::move(c));
    END_HANDLE_TH_ERRORS
}

// The structure of a cache (a tuple of four tensors) and its page table; false where they are not plain.
struct Cache {
    KvFp8Cache c;
    int64_t B, W, pitch;
    const int* table;
    c10::Device device = c10::Device(c10::kCPU);
};
bool cache_of(PyObject* cache, PyObject* table, Cache& out) {
    if (!PyTuple_Check(cache) || PyTuple_GET_SIZE(cache) != 4 || !plain(table, 2, at::kInt)) return false;
    for (int i = 0; i < 4; ++i)
        if (!plain(PyTuple_GET_ITEM(cache, i), i < 2 ? 4 : 2, at::kByte) || !THPVariable_Unpack(PyTuple_GET_ITEM(cache, i)).is_contiguous()) return false;
    const At &k = THPVariable_Unpack(PyTuple_GET_ITEM(cache, 0)), &v = THPVariable_Unpack(PyTuple_GET_ITEM(cache, 1)),
             &ke = THPVariable_Unpack(PyTuple_GET_ITEM(cache, 2)), &ve = THPVariable_Unpack(PyTuple_GET_ITEM(cache, 3)), &t = THPVariable_Unpack(table);
    const int64_t P = k.size(0), H = k.size(1), page = k.size(2), D = k.size(3);
    if (v.size(0) != P || v.size(1) != H || v.size(2) != D || v.size(3) != page || ke.size(0) != P || ke.size(1) != H || ve.sizes() != ke.sizes()) return false;
    out.device = k.device();
    if (v.device() != out.device || ke.device() != out.device || ve.device() != out.device || t.device() != out.device) return false;
    if (c10::hip::current_device() != out.device.index()) return false;
    if (!fits(P) || !fits(H) || !fits(page) || !fits(D) || !fits(t.size(0)) || !fits(t.size(1))) return false;
    out.c = KvFp8Cache{k.data_ptr(), v.data_ptr(), (unsigned char*)ke.data_ptr(), (unsigned char*)ve.data_ptr(), (int)P, (int)H, (int)page, (int)D};
    out.B = t.size(0), out.W = t.size(1), out.pitch = t.stride(0), out.table = (const int*)t.data_ptr();
    return true;
}
// An int32 vector with an entry per sequence; None, where that is allowed, is a null pointer.
bool per_sequence(PyObject* obj, const Cache& c, bool optional, const int*& out) {
    out = nullptr;
    if (obj == Py_None) return optional;
    if (!plain(obj, 1, at::kInt)) return false;
    const At& t = THPVariable_Unpack(obj);
    if (t.size(0) != c.B || t.device() != c.device) return false;
    out = (const int*)t.data_ptr();
    return true;
}
bool whole_number(PyObject* obj, int& out) {
    if (!PyLong_CheckExact(obj)) return false;
    int over = 0;
    const long long v = PyLong_AsLongLongAndOverflow(obj, &over);
    if (over || v < INT_MIN || v > INT_MAX) return false;
    out = (int)v;
    return true;
}
struct Strides { long long s[3]; };
Strides strides(const At& t) { return {{t.stride(0), t.stride(1), t.stride(2)}}; }

PyObject* pair_of(At&& a, At&& b) {
    PyObject* const out[2] = {THPVariable_Wrap(std::move(a)), THPVariable_Wrap(std::move(b))};
    PyObject* const both = PyTuple_Pack(2, out[0], out[1]);
    Py_XDECREF(out[0]);
    Py_XDECREF(out[1]);
    return both;
}

PyObject* attn_kv(PyObject*, PyObject* const* args, Py_ssize_t n) {   // q, cache, table, lens, q_lens, causal, window, sinks, scale, max_len
    HANDLE_TH_ERRORS
    Cache c;
    const int *lens, *q_lens;
    int window, sinks, max_len;
    if (!entry.attn_fwd || n != 10 || at::impl::torch_function_mode_enabled() || !plain(args[0], 4) || !cache_of(args[1], args[2], c) ||
        !per_sequence(args[3], c, false, lens) || !per_sequence(args[4], c, true, q_lens) || !PyBool_Check(args[5]) ||
        !whole_number(args[6], window) || !whole_number(args[7], sinks) || !whole_number(args[9], max_len)) Py_RETURN_NONE;
    const At& q = THPVariable_Unpack(args[0]);
    const int64_t B = q.size(0), Hq = q.size(1), Sq = q.size(2), D = q.size(3);
    if (B != c.B || D != c.c.D || c.c.Hkv == 0 || Hq % c.c.Hkv || q.device() != c.device || !fits(Hq) || !fits(Sq)) Py_RETURN_NONE;
    double scale;
    if (args[8] == Py_None) scale = std::pow((double)D, -0.5);
    else if (PyFloat_CheckExact(args[8])) scale = PyFloat_AS_DOUBLE(args[8]);
    else Py_RETURN_NONE;
    const int causal = args[5] == Py_True;
    At o, lse;
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        o = at::empty_like(q);
        if (o.stride(3) != 1) rc = INT_MIN;
        else {
            lse = at::empty({B, Hq, Sq}, q.options().dtype(at::kFloat));
            const int64_t most = c.W * c.c.page, longest = max_len > 0 && max_len < most ? max_len : most;
            const size_t need = fits(longest) ? entry.attn_kv_fp8_workspace_bytes((int)B, (int)Hq, c.c.Hkv, (int)Sq, (int)longest, (int)D, window, sinks) : 0;
            At ws;
            if (need) ws = scratch(need, q);
            rc = entry.attn_kv_fp8(q.data_ptr(), &c.c, c.table, c.pitch, (int)c.W, lens, q_lens, o.data_ptr(), (float*)lse.data_ptr(), (int)B, (int)Hq, (int)Sq,
                                   strides(q).s, strides(o).s, causal, window, sinks, (float)scale, max_len, ws.defined() ? ws.data_ptr() : nullptr,
                                   ws.defined() ? need : 0, ws.defined() ? (int)(need / (4 * (size_t)B * Hq * Sq * (D + 2))) : 1, 0, stream_of(q));
        }
    }
    if (rc == INT_MIN) Py_RETURN_NONE;
    if (rc != 0) return PyLong_FromLong(rc);
    return pair_of(std::move(o), std::move(lse));
    END_HANDLE_TH_ERRORS
}

PyObject* kv_write(PyObject*, PyObject* const* args, Py_ssize_t n) {  // cache, k, v, table, start, count
    HANDLE_TH_ERRORS
    Cache c;
    const int *start, *count;
    if (!entry.attn_fwd || n != 6 || at::impl::torch_function_mode_enabled() || !plain(args[1], 4) || !plain(args[2], 4) || !cache_of(args[0], args[3], c) ||
        !per_sequence(args[4], c, false, start) || !per_sequence(args[5], c, true, count)) Py_RETURN_NONE;
    const At &k = THPVariable_Unpack(args[1]), &v = THPVariable_Unpack(args[2]);
    if (k.sizes() != v.sizes() || k.size(0) != c.B || k.size(1) != c.c.Hkv || k.size(3) != c.c.D || !fits(k.size(2)) || k.device() != c.device || v.device() != c.device) Py_RETURN_NONE;
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        rc = entry.kv_fp8_write(&c.c, k.data_ptr(), v.data_ptr(), strides(k).s, strides(v).s, c.table, c.pitch, (int)c.W, start, count, (int)c.B, (int)k.size(2), stream_of(k));
    }
    if (rc != 0) return PyLong_FromLong(rc);
    Py_INCREF(args[0]);
    return args[0];
    END_HANDLE_TH_ERRORS
}

PyObject* kv_read(PyObject*, PyObject* const* args, Py_ssize_t n) {   // cache, table, lens, S, first
    HANDLE_TH_ERRORS
    Cache c;
    const int* lens;
    int S, first;
    if (!entry.attn_fwd || n != 5 || at::impl::torch_function_mode_enabled() || !cache_of(args[0], args[1], c) || !per_sequence(args[2], c, false, lens) ||
        !whole_number(args[3], S) || !whole_number(args[4], first) || S <= 0) Py_RETURN_NONE;
    At k, v;
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        const At& codes = THPVariable_Unpack(PyTuple_GET_ITEM(args[0], 0));
        k = at::empty({c.B, c.c.Hkv, S, c.c.D}, codes.options().dtype(at::kBFloat16));
        v = at::empty_like(k);
        rc = entry.kv_fp8_read(&c.c, c.table, c.pitch, (int)c.W, lens, k.data_ptr(), v.data_ptr(), strides(k).s, strides(v).s, (int)c.B, S, first, stream_of(k));
    }
    if (rc != 0) return PyLong_FromLong(rc);
    return pair_of(std::move(k), std::move(v));
    END_HANDLE_TH_ERRORS
}

PyObject* rope(PyObject*, PyObject* const* args, Py_ssize_t n) {      // q, positions, inv_freq, k, interleaved, inverse, scale
    HANDLE_TH_ERRORS
    if (!entry.attn_fwd || n != 7 || at::impl::torch_function_mode_enabled() || !plain(args[0], 4) || !plain(args[2], 1, at::kDouble) ||
        !PyBool_Check(args[4]) || !PyBool_Check(args[5]) || !PyFloat_CheckExact(args[6])) Py_RETURN_NONE;
    const bool shared = plain(args[1], 1, at::kInt);
    if (!shared && !plain(args[1], 2, at::kInt)) Py_RETURN_NONE;
    const bool has_k = args[3] != Py_None;
    if (has_k && !plain(args[3], 4)) Py_RETURN_NONE;
    const At &q = THPVariable_Unpack(args[0]), &pos = THPVariable_Unpack(args[1]), &inv = THPVariable_Unpack(args[2]);
    const At k = has_k ? THPVariable_Unpack(args[3]) : At();
    const int64_t B = q.size(0), Hq = q.size(1), S = q.size(2), D = q.size(3), Hk = has_k ? k.size(1) : 0;
    if (pos.size(shared ? 0 : 1) != S || (!shared && pos.size(0) != B) || pos.device() != q.device() || inv.device() != q.device() || inv.size(0) > (1 << 20)) Py_RETURN_NONE;
    if (has_k && (k.size(0) != B || Hk == 0 || k.size(2) != S || k.size(3) != D || k.device() != q.device())) Py_RETURN_NONE;
    if (c10::hip::current_device() != q.get_device() || !fits(B) || !fits(Hq) || !fits(Hk) || !fits(S) || !fits(D)) Py_RETURN_NONE;
    At qo, ko;
    int rc;
    {
        pybind11::gil_scoped_release no_gil;
        qo = at::empty_like(q);
        if (has_k) ko = at::empty_like(k);
        if (qo.stride(3) != 1 || (has_k && ko.stride(3) != 1)) rc = INT_MIN;
        else
            rc = entry.rope_bf16(q.data_ptr(), qo.data_ptr(), has_k ? k.data_ptr() : nullptr, has_k ? ko.data_ptr() : nullptr, (int)B, (int)Hq, (int)Hk, (int)S, (int)D,
                                 (int)(2 * inv.size(0)), strides(q).s, strides(qo).s, has_k ? strides(k).s : nullptr, has_k ? strides(ko).s : nullptr, (const int*)pos.data_ptr(),
                                 shared ? 0 : pos.stride(0), (const double*)inv.data_ptr(), args[4] == Py_True, args[5] == Py_True, (float)PyFloat_AS_DOUBLE(args[6]), stream_of(q));
    }
    if (rc == INT_MIN) Py_RETURN_NONE;
    if (rc != 0) return PyLong_FromLong(rc);
    if (!has_k) return THPVariable_Wrap(std::move(qo));
    return pair_of(std::move(qo), std::move(ko));
    END_HANDLE_TH_ERRORS
}

// The entry points' addresses, in the order of Entries.
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    constexpr int kEntries = sizeof(Entries) / sizeof(void*);
    void* p[kEntries];
    if (n != kEntries) { PyErr_SetString(PyExc_TypeError, "an address for every entry point"); return nullptr; }
    for (int i = 0; i < kEntries; ++i) {
        p[i] = PyLong_AsVoidPtr(args[i]);
        if (!p[i]) { if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address is null"); return nullptr; }
    }
    int at = 0;
    auto next = [&](auto& f) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(p[at++]); };
    next(entry.attn_fwd), next(entry.attn_fwd_strided), next(entry.attn_fwd_workspace_bytes), next(entry.attn_fwd_workspace);
    next(entry.gemm_bf16_workspace_bytes), next(entry.gemm_bf16_tile), next(entry.gemm_bf16_workspace);
    next(entry.kv_fp8_write), next(entry.kv_fp8_read), next(entry.attn_kv_fp8_workspace_bytes), next(entry.attn_kv_fp8), next(entry.rope_bf16);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void*)bind, METH_FASTCALL, nullptr},
    {"attn", (PyCFunction)(void*)attn, METH_FASTCALL, nullptr},
    {"gemm", (PyCFunction)(void*)gemm, METH_FASTCALL, nullptr},
    {"attn_kv", (PyCFunction)(void*)attn_kv, METH_FASTCALL, nullptr},
    {"kv_write", (PyCFunction)(void*)kv_write, METH_FASTCALL, nullptr},
    {"kv_read", (PyCFunction)(void*)kv_read, METH_FASTCALL, nullptr},
    {"rope", (PyCFunction)(void*)rope, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
    PyObject* const m = PyModule_Create(&module);
    // the torch it was compiled for, which the binding compares with the one in use
    if (m && PyModule_AddStringConstant(m, "torch_version", NATIVE_TORCH) != 0) { Py_DECREF(m); return nullptr; }
    return m;
}
