// The calls that a serving loop makes once or more per layer, without Python between the argument checks, the output
// tensor and the launch: one token through one projection (quantise, multiply) took 30 us of which the GPU works for 6.
//
// Every function answers with its result, with the library's error code (an int), or with None: anything but the plain
// case -- other objects than torch.Tensor itself, wrong types, shapes or strides, numbers that do not fit, a workspace
// that has to be made first -- goes back to the caller, whose general path runs it or raises what it always raised.
// The library is reached through the addresses that bind() is handed, so that it is the one that api.py has loaded.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/GradMode.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <climits>
#include <cmath>
#include <vector>

#include "liquidgemm.h"

namespace {

struct Library {
    decltype(&w4a8_gemm) gemm;
    decltype(&w4a8_gemm_workspace_size) workspace_size;
    decltype(&w4a8_quantize_activations) quantize;
    decltype(&w4a8_grouped_gemm) grouped;
    decltype(&liquidquant_packed_size) packed_size;
} lib{};
struct Attention {
    decltype(&attn_qk_norm_rope) rope;
    decltype(&kv4_write) write;
    decltype(&kv4_append) append;
    decltype(&kv4_read) read;
    decltype(&kv4_attention_workspace_size) workspace_size;
    decltype(&kv4_attention) decode;
    decltype(&attn_prompt_workspace_size) prompt_workspace_size;
    decltype(&attn_prompt) prompt;
} attn{};

struct Layer {
    decltype(&kv4_attention_chunks_workspace_size) chunks_workspace_size;
    decltype(&kv4_attention_chunks) chunks;
    decltype(&w4a8_norm_quantize) norm;
    decltype(&w4a8_swiglu_quantize) swiglu;
    decltype(&moe_dispatch) dispatch;
    decltype(&moe_combine) combine;
    decltype(&moe_combine_backward) combine_backward;
} layer{};

// The GIL is given up for the allocation and the launch (both may wait), also where they throw.
struct WithoutGil {
    PyThreadState *const state = PyEval_SaveThread();
    ~WithoutGil() { PyEval_RestoreThread(state); }
};

// What the general path's checks accept: a tensor on the GPU of that type and shape, contiguous
bool plain(PyObject *o, at::ScalarType type, std::initializer_list<int64_t> shape)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.is_cuda() && t.scalar_type() == type && t.layout() == at::kStrided && t.sizes().equals(shape) && t.is_contiguous();
}
const at::Tensor &tensor(PyObject *o) { return THPVariable_Unpack(o); }

bool small_int(PyObject *o, int &v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long long x = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow || x < INT_MIN || x > INT_MAX) return false;
    v = (int)x;
    return true;
}

// stream: None (torch's current one) or its number
bool stream_of(PyObject *o, void *&stream)
{
    if (o == Py_None) {
        stream = c10::hip::getCurrentHIPStream().stream();
        return true;
    }
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long long x = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow || x < 0) return false;
    stream = reinterpret_cast<void *>((uintptr_t)x);
    return true;
}

// rows of a matrix of `type` on the GPU, or -1
int64_t rows_of(PyObject *o, at::ScalarType type)
{
    if (!THPVariable_CheckExact(o)) return -1;
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.layout() != at::kStrided || t.dim() != 2 || t.size(0) > INT_MAX || t.size(1) > INT_MAX)
        return -1;
    return t.size(0);
}

// A call's workspace: the given one, or the buffer of this device and stream in `workspaces` if there is one that is large enough
// (nothing where need is 0).  False, without a Python error, where there is none; with one where the lookup failed.
bool workspace_of(PyObject *given, PyObject *workspaces, const at::Tensor &x, void *stream, size_t need, at::Tensor &workspace)
{
    if (given != Py_None) {
        if (!THPVariable_CheckExact(given)) return false;
        workspace = tensor(given);
        return workspace.is_cuda() && workspace.scalar_type() == at::kByte && workspace.layout() == at::kStrided && workspace.is_contiguous();
    }
    if (need == 0) return true;
    PyObject *const key = Py_BuildValue("(iK)", (int)x.device().index(), (unsigned long long)(uintptr_t)stream);
    if (!key) return false;
    PyObject *const found = PyDict_GetItemWithError(workspaces, key);
    Py_DECREF(key);
    if (!found || !THPVariable_CheckExact(found) || (size_t)tensor(found).numel() < need) return false;
    workspace = tensor(found);
    return true;
}

// quantize(X_f16, smooth, out_q, out_scales, stream) -> (X_i8, act_scales)
PyObject *quantize(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    const int64_t M = n == 5 ? rows_of(a[0], at::kHalf) : -1;
    if (M < 0) Py_RETURN_NONE;
    const at::Tensor &x = tensor(a[0]);
    const int64_t K = x.size(1);
    if (!x.is_contiguous() || (a[1] != Py_None && !plain(a[1], at::kFloat, {K})) || (a[2] != Py_None && !plain(a[2], at::kChar, {M, K})) ||
        (a[3] != Py_None && !plain(a[3], at::kFloat, {M})) || !stream_of(a[4], stream))
        Py_RETURN_NONE;
    at::Tensor q = a[2] != Py_None ? tensor(a[2]) : at::Tensor(), s = a[3] != Py_None ? tensor(a[3]) : at::Tensor();
    const float *smooth = a[1] != Py_None ? static_cast<const float *>(tensor(a[1]).data_ptr()) : nullptr;
    int rc;
    {
        const WithoutGil released;
        if (!q.defined()) q = at::empty({M, K}, x.options().dtype(at::kChar));
        if (!s.defined()) s = at::empty({M}, x.options().dtype(at::kFloat));
        rc = lib.quantize((int)M, (int)K, static_cast<const uint16_t *>(x.data_ptr()), smooth, static_cast<int8_t *>(q.data_ptr()),
                          static_cast<float *>(s.data_ptr()), stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    PyObject *const pq = a[2] != Py_None ? (Py_INCREF(a[2]), a[2]) : THPVariable_Wrap(std::move(q));
    PyObject *const ps = a[3] != Py_None ? (Py_INCREF(a[3]), a[3]) : THPVariable_Wrap(std::move(s));
    PyObject *const both = pq && ps ? PyTuple_Pack(2, pq, ps) : nullptr;
    Py_XDECREF(pq);
    Py_XDECREF(ps);
    return both;
    END_HANDLE_TH_ERRORS
}

// gemm(X, act_scales, W_packed, gparams, w_scales, N, K, group, out, workspace, stream, workspaces) -> out
PyObject *gemm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    int N, K, group;
    size_t codes = 0, gparams = 0;
    const int64_t M = n == 12 ? rows_of(a[0], at::kChar) : -1;
    if (M < 1 || !small_int(a[5], N) || !small_int(a[6], K) || !small_int(a[7], group) ||
        lib.packed_size(N, K, group, &codes, &gparams) != LQ_OK || !plain(a[0], at::kChar, {M, K}) || !plain(a[1], at::kFloat, {M}) ||
        !plain(a[2], at::kByte, {(int64_t)codes}) || !plain(a[3], at::kByte, {(int64_t)gparams}) || !plain(a[4], at::kFloat, {N}) ||
        (a[8] != Py_None && !plain(a[8], at::kHalf, {M, N})) || !stream_of(a[10], stream))
        Py_RETURN_NONE;
    const at::Tensor &x = tensor(a[0]);
    at::Tensor workspace;
    if (!workspace_of(a[9], a[11], x, stream, a[9] != Py_None ? 0 : lib.workspace_size((int)M, N, K, group), workspace)) {
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
    at::Tensor out = a[8] != Py_None ? tensor(a[8]) : at::Tensor();
    int rc;
    {
        const WithoutGil released;
        if (!out.defined()) out = at::empty({M, N}, x.options().dtype(at::kHalf));
        rc = lib.gemm((int)M, N, K, group, static_cast<const int8_t *>(x.data_ptr()), static_cast<const float *>(tensor(a[1]).data_ptr()),
                      tensor(a[2]).data_ptr(), static_cast<const uint8_t *>(tensor(a[3]).data_ptr()),
                      static_cast<const float *>(tensor(a[4]).data_ptr()), static_cast<uint16_t *>(out.data_ptr()),
                      workspace.defined() ? workspace.data_ptr() : nullptr, workspace.defined() ? (size_t)workspace.numel() : 0, stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return a[8] != Py_None ? (Py_INCREF(a[8]), a[8]) : THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// grouped(row_offsets (a list), X, act_scales, W_packed, gparams, w_scales, N, K, group, out_y, stream) -> out_y
PyObject *grouped(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    int N, K, group;
    size_t codes = 0, gparams = 0;
    if (n != 11 || !PyList_CheckExact(a[0]) || PyList_GET_SIZE(a[0]) < 2 || PyList_GET_SIZE(a[0]) > 65) Py_RETURN_NONE;
    const int E = (int)PyList_GET_SIZE(a[0]) - 1;
    int offsets[65];
    for (int i = 0; i <= E; ++i)
        if (!small_int(PyList_GET_ITEM(a[0], i), offsets[i])) Py_RETURN_NONE;
    const int64_t M = offsets[E];
    if (M < 1 || !small_int(a[6], N) || !small_int(a[7], K) || !small_int(a[8], group) ||
        lib.packed_size(N, K, group, &codes, &gparams) != LQ_OK || !plain(a[1], at::kChar, {M, K}) || !plain(a[2], at::kFloat, {M}) ||
        !plain(a[3], at::kByte, {(int64_t)codes * E}) || !plain(a[4], at::kByte, {(int64_t)gparams * E}) ||
        !plain(a[5], at::kFloat, {E, N}) || (a[9] != Py_None && !plain(a[9], at::kHalf, {M, N})) || !stream_of(a[10], stream))
        Py_RETURN_NONE;
    const at::Tensor &x = tensor(a[1]);
    at::Tensor out = a[9] != Py_None ? tensor(a[9]) : at::Tensor();
    int rc;
    {
        const WithoutGil released;
        if (!out.defined()) out = at::empty({M, N}, x.options().dtype(at::kHalf));
        rc = lib.grouped(E, offsets, N, K, group, static_cast<const int8_t *>(x.data_ptr()), static_cast<const float *>(tensor(a[2]).data_ptr()),
                         tensor(a[3]).data_ptr(), static_cast<const uint8_t *>(tensor(a[4]).data_ptr()),
                         static_cast<const float *>(tensor(a[5]).data_ptr()), static_cast<uint16_t *>(out.data_ptr()), nullptr, stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return a[9] != Py_None ? (Py_INCREF(a[9]), a[9]) : THPVariable_Wrap(std::move(out));
    END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------------------------- attention
// A gradient is asked for: the general path says that there is none
bool wants_gradient(PyObject *o) { return o != Py_None && c10::GradMode::is_enabled() && tensor(o).requires_grad(); }
// [.., heads, head_dim] with strides of its own, FP16 or BF16 (`like`: as that one)
bool heads(PyObject *o, int64_t dims, const at::Tensor *like = nullptr)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda() || t.layout() != at::kStrided || t.dim() != dims || (like ? t.scalar_type() != like->scalar_type() : t.scalar_type() != at::kHalf && t.scalar_type() != at::kBFloat16))
        return false;
    for (const int64_t n : t.sizes())
        if (n > INT_MAX) return false;
    return t.stride(dims - 1) == 1 && t.size(dims - 1) > 1 && !wants_gradient(o);
}
bool heads_of(PyObject *o, const at::Tensor &like, std::initializer_list<int64_t> shape)
{
    return heads(o, (int64_t)shape.size(), &like) && tensor(o).sizes().equals(shape);
}
int dtype_of(const at::Tensor &t) { return t.scalar_type() == at::kHalf ? LQ_F16 : LQ_BF16; }
const float *floats(PyObject *o) { return o == Py_None ? nullptr : static_cast<const float *>(tensor(o).data_ptr()); }
const int *ints(PyObject *o) { return static_cast<const int *>(tensor(o).data_ptr()); }

// on the current device, whose stream the call goes to (the general path says so where it is another)
bool here(const at::Tensor &t) { return t.device().index() == c10::hip::getCurrentHIPStream().device_index(); }
bool all_here(PyObject *const *a, int n)
{
    for (int i = 0; i < n; ++i)
        if (a[i] != Py_None && !here(tensor(a[i]))) return false;
    return true;
}

// a contiguous tensor of `dims` dimensions
bool plain_dims(PyObject *o, at::ScalarType type, int64_t dims)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = tensor(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.layout() != at::kStrided || t.dim() != dims || !t.is_contiguous()) return false;
    for (const int64_t n : t.sizes())
        if (n > INT_MAX) return false;
    return true;
}

struct Cache {
    void *p;
    int pages, heads, page, dim;
};
bool cache_of(PyObject *o, Cache &c)
{
    if (!plain_dims(o, at::kByte, 3)) return false;
    const at::Tensor &t = tensor(o);
    c = Cache{t.data_ptr(), (int)t.size(0), (int)t.size(1), 0, 0};
    for (const int dim : {64, 128}) {
        const int64_t page = t.size(2) / (dim + 8);
        if (page * (dim + 8) == t.size(2) && page >= 16 && page <= 256 && !(page & (page - 1))) c.page = (int)page, c.dim = dim;
    }
    return c.dim != 0;
}

// what rope and append share: a[0..1] = q, k; positions, table, interleaved, q_norm, k_norm, eps
struct Rotation {
    int interleaved;
    double eps;
};
bool rotation(PyObject *positions, PyObject *table, PyObject *interleaved, PyObject *q_norm, PyObject *k_norm, PyObject *eps, int64_t T, int64_t D, Rotation &r)
{
    if (!plain(positions, at::kInt, {T}) || !plain_dims(table, at::kFloat, 2) || !PyBool_Check(interleaved) || !PyFloat_CheckExact(eps) ||
        (q_norm != Py_None && !plain(q_norm, at::kFloat, {D})) || (k_norm != Py_None && !plain(k_norm, at::kFloat, {D})) ||
        wants_gradient(table) || wants_gradient(q_norm) || wants_gradient(k_norm))
        return false;
    r = Rotation{interleaved == Py_True, PyFloat_AS_DOUBLE(eps)};
    return true;
}

PyObject *wrapped(PyObject *given, at::Tensor &&t) { return given != Py_None ? (Py_INCREF(given), given) : THPVariable_Wrap(std::move(t)); }
PyObject *pair(PyObject *a, PyObject *b)
{
    PyObject *const both = a && b ? PyTuple_Pack(2, a, b) : nullptr;
    Py_XDECREF(a);
    Py_XDECREF(b);
    return both;
}

// rope(q, k, positions, table, interleaved, q_norm, k_norm, eps, out_q, out_k, stream) -> (out_q, out_k)
PyObject *rope(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    Rotation r;
    if (n != 11 || !heads(a[0], 3)) Py_RETURN_NONE;
    const at::Tensor &q = tensor(a[0]);
    const int64_t T = q.size(0), Hq = q.size(1), D = q.size(2);
    if (!heads(a[1], 3, &q)) Py_RETURN_NONE;
    const at::Tensor &k = tensor(a[1]);
    const int64_t Hkv = k.size(1);
    if (k.size(0) != T || k.size(2) != D || !rotation(a[2], a[3], a[4], a[5], a[6], a[7], T, D, r) ||
        (a[8] != Py_None && !heads_of(a[8], q, {T, Hq, D})) || (a[9] != Py_None && !heads_of(a[9], q, {T, Hkv, D})) || !stream_of(a[10], stream))
        Py_RETURN_NONE;
    const at::Tensor &table = tensor(a[3]);
    at::Tensor oq = a[8] != Py_None ? tensor(a[8]) : at::Tensor(), ok = a[9] != Py_None ? tensor(a[9]) : at::Tensor();
    int rc;
    {
        const WithoutGil released;
        if (!oq.defined()) oq = at::empty({T, Hq, D}, q.options());
        if (!ok.defined()) ok = at::empty({T, Hkv, D}, q.options());
        rc = attn.rope(dtype_of(q), (int)T, (int)Hq, (int)Hkv, (int)D, q.data_ptr(), q.stride(0), q.stride(1), k.data_ptr(), k.stride(0), k.stride(1),
                       ints(a[2]), floats(a[3]), (int)table.size(0), (int)table.size(1), r.interleaved, floats(a[5]), floats(a[6]), (float)r.eps,
                       oq.data_ptr(), oq.stride(0), oq.stride(1), ok.data_ptr(), ok.stride(0), ok.stride(1), stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return pair(wrapped(a[8], std::move(oq)), wrapped(a[9], std::move(ok)));
    END_HANDLE_TH_ERRORS
}

// write(k, v, slots, cache, stream) -> cache
PyObject *write(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    Cache c;
    if (n != 5 || !heads(a[0], 3)) Py_RETURN_NONE;
    const at::Tensor &k = tensor(a[0]);
    const int64_t T = k.size(0), Hkv = k.size(1), D = k.size(2);
    if (!heads_of(a[1], k, {T, Hkv, D}) || !plain(a[2], at::kInt, {T}) || !cache_of(a[3], c) || c.heads != Hkv || c.dim != D || !stream_of(a[4], stream))
        Py_RETURN_NONE;
    const at::Tensor &v = tensor(a[1]);
    int rc;
    {
        const WithoutGil released;
        rc = attn.write(dtype_of(k), (int)T, (int)Hkv, (int)D, k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1),
                        ints(a[2]), c.p, c.pages, c.page, stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    Py_INCREF(a[3]);
    return a[3];
    END_HANDLE_TH_ERRORS
}

// append(q, k, v, positions, table, slots, cache, interleaved, q_norm, k_norm, eps, out_q, stream) -> out_q
PyObject *append(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    Rotation r;
    Cache c;
    if (n != 13 || !heads(a[0], 3)) Py_RETURN_NONE;
    const at::Tensor &q = tensor(a[0]);
    const int64_t T = q.size(0), Hq = q.size(1), D = q.size(2);
    if (!heads(a[1], 3, &q)) Py_RETURN_NONE;
    const at::Tensor &k = tensor(a[1]);
    const int64_t Hkv = k.size(1);
    if (k.size(0) != T || k.size(2) != D || !heads_of(a[2], q, {T, Hkv, D}) || !rotation(a[3], a[4], a[7], a[8], a[9], a[10], T, D, r) ||
        !plain(a[5], at::kInt, {T}) || !cache_of(a[6], c) || c.heads != Hkv || c.dim != D ||
        (a[11] != Py_None && !heads_of(a[11], q, {T, Hq, D})) || !stream_of(a[12], stream))
        Py_RETURN_NONE;
    const at::Tensor &v = tensor(a[2]), &table = tensor(a[4]);
    at::Tensor oq = a[11] != Py_None ? tensor(a[11]) : at::Tensor();
    int rc;
    {
        const WithoutGil released;
        if (!oq.defined()) oq = at::empty({T, Hq, D}, q.options());
        rc = attn.append(dtype_of(q), (int)T, (int)Hq, (int)Hkv, (int)D, q.data_ptr(), q.stride(0), q.stride(1), k.data_ptr(), k.stride(0), k.stride(1),
                         v.data_ptr(), v.stride(0), v.stride(1), ints(a[3]), floats(a[4]), (int)table.size(0), (int)table.size(1), r.interleaved,
                         floats(a[8]), floats(a[9]), (float)r.eps, oq.data_ptr(), oq.stride(0), oq.stride(1), ints(a[5]), c.p, c.pages, c.page, stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return wrapped(a[11], std::move(oq));
    END_HANDLE_TH_ERRORS
}

// read(cache, slots, bf16 (a bool), stream) -> (k, v)
PyObject *read(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    Cache c;
    if (n != 4 || !cache_of(a[0], c) || !plain_dims(a[1], at::kInt, 1) || !PyBool_Check(a[2]) || !stream_of(a[3], stream)) Py_RETURN_NONE;
    const int64_t T = tensor(a[1]).size(0);
    at::Tensor k, v;
    int rc;
    {
        const WithoutGil released;
        const auto options = tensor(a[0]).options().dtype(a[2] == Py_True ? at::kBFloat16 : at::kHalf);
        k = at::empty({T, c.heads, c.dim}, options);
        v = at::empty({T, c.heads, c.dim}, options);
        rc = attn.read(dtype_of(k), (int)T, c.heads, c.dim, c.p, c.pages, c.page, ints(a[1]), k.data_ptr(), v.data_ptr(), stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return pair(THPVariable_Wrap(std::move(k)), THPVariable_Wrap(std::move(v)));
    END_HANDLE_TH_ERRORS
}

// scale: None (1 / sqrt(head_dim)) or a float
bool scale_of(PyObject *o, int64_t D, double &scale)
{
    if (o != Py_None && !PyFloat_CheckExact(o)) return false;
    scale = o == Py_None ? 1.0 / std::sqrt((double)D) : PyFloat_AS_DOUBLE(o);
    return true;
}

// decode(q, cache, block_table, context, scale, out, workspace, stream, workspaces) -> out
PyObject *decode(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    Cache c;
    double scale;
    if (n != 9 || !THPVariable_CheckExact(a[0])) Py_RETURN_NONE;
    const at::Tensor &q = tensor(a[0]);
    const int64_t dims = q.dim();
    if ((dims != 3 && dims != 4) || !heads(a[0], dims) || !cache_of(a[1], c) || q.size(dims - 1) != c.dim) Py_RETURN_NONE;
    const int64_t B = q.size(0), fresh = dims == 4 ? q.size(1) : 1, Hq = q.size(dims - 2);
    if (!plain_dims(a[2], at::kInt, 2) || tensor(a[2]).size(0) != B || !plain(a[3], at::kInt, {B}) || !scale_of(a[4], c.dim, scale) ||
        (a[5] != Py_None && !(heads(a[5], dims, &q) && tensor(a[5]).sizes().equals(q.sizes()) && tensor(a[5]).is_contiguous())) || !stream_of(a[7], stream))
        Py_RETURN_NONE;
    at::Tensor workspace;
    const size_t need = attn.workspace_size((int)B, (int)fresh, (int)Hq, c.heads, c.dim);
    if (!workspace_of(a[6], a[8], q, stream, need, workspace)) {
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
    at::Tensor out = a[5] != Py_None ? tensor(a[5]) : at::Tensor();
    int rc;
    {
        const WithoutGil released;
        if (!out.defined()) out = at::empty(q.sizes(), q.options());
        rc = attn.decode(dtype_of(q), (int)B, (int)fresh, (int)Hq, c.heads, c.dim, q.data_ptr(), q.stride(0), dims == 4 ? q.stride(1) : 0, q.stride(dims - 2),
                         c.p, c.pages, c.page, ints(a[2]), (int)tensor(a[2]).size(1), ints(a[3]), (float)scale, out.data_ptr(),
                         workspace.defined() ? workspace.data_ptr() : nullptr, workspace.defined() ? (size_t)workspace.numel() : 0, stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return wrapped(a[5], std::move(out));
    END_HANDLE_TH_ERRORS
}

// prompt(q, k, v, starts_q, starts_k, scale, causal, out, workspace, stream, workspaces) -> out
PyObject *prompt(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    double scale;
    if (n != 11 || !heads(a[0], 3)) Py_RETURN_NONE;
    const at::Tensor &q = tensor(a[0]);
    if (!heads(a[1], 3, &q)) Py_RETURN_NONE;
    const at::Tensor &k = tensor(a[1]);
    const int64_t T = q.size(0), Hq = q.size(1), D = q.size(2), Tk = k.size(0), Hkv = k.size(1);
    if (k.size(2) != D || !heads_of(a[2], q, {Tk, Hkv, D}) || !plain_dims(a[3], at::kInt, 1) || tensor(a[3]).size(0) < 1 ||
        !plain(a[4], at::kInt, {tensor(a[3]).size(0)}) || !scale_of(a[5], D, scale) || !PyBool_Check(a[6]) ||
        (a[7] != Py_None && !plain(a[7], q.scalar_type(), {T, Hq, D})) || wants_gradient(a[7]) || !stream_of(a[9], stream))
        Py_RETURN_NONE;
    const int S = (int)tensor(a[3]).size(0) - 1;
    at::Tensor workspace;
    if (!workspace_of(a[8], a[10], q, stream, attn.prompt_workspace_size(S, (int)T, (int)Tk, (int)Hq, (int)Hkv, (int)D), workspace)) {
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
    const at::Tensor &v = tensor(a[2]);
    at::Tensor out = a[7] != Py_None ? tensor(a[7]) : at::Tensor();
    int rc;
    {
        const WithoutGil released;
        if (!out.defined()) out = at::empty({T, Hq, D}, q.options());
        rc = attn.prompt(dtype_of(q), S, (int)T, (int)Tk, (int)Hq, (int)Hkv, (int)D, q.data_ptr(), q.stride(0), q.stride(1),
                         k.data_ptr(), k.stride(0), k.stride(1), v.data_ptr(), v.stride(0), v.stride(1), ints(a[3]), ints(a[4]), (float)scale,
                         a[6] == Py_True, out.data_ptr(), workspace.defined() ? workspace.data_ptr() : nullptr,
                         workspace.defined() ? (size_t)workspace.numel() : 0, stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return wrapped(a[7], std::move(out));
    END_HANDLE_TH_ERRORS
}

// chunks(q, cache, block_table, context, starts_q, scale, out, workspace, stream, workspaces) -> out
PyObject *chunks(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    Cache c;
    double scale;
    if (n != 10 || !heads(a[0], 3) || !cache_of(a[1], c)) Py_RETURN_NONE;
    const at::Tensor &q = tensor(a[0]);
    const int64_t T = q.size(0), Hq = q.size(1);
    if (q.size(2) != c.dim || !plain_dims(a[4], at::kInt, 1) || tensor(a[4]).size(0) < 1) Py_RETURN_NONE;
    const int64_t S = tensor(a[4]).size(0) - 1;
    if (!plain_dims(a[2], at::kInt, 2) || tensor(a[2]).size(0) != S || !plain(a[3], at::kInt, {S}) || !scale_of(a[5], c.dim, scale) ||
        (a[6] != Py_None && !plain(a[6], q.scalar_type(), {T, Hq, c.dim})) || wants_gradient(a[6]) || !here(q) || !all_here(a + 1, 4) || !all_here(a + 6, 1) ||
        !stream_of(a[8], stream))
        Py_RETURN_NONE;
    const int width = (int)tensor(a[2]).size(1);
    at::Tensor workspace;
    if (!workspace_of(a[7], a[9], q, stream, layer.chunks_workspace_size((int)S, (int)T, (int)Hq, c.heads, c.dim, c.page, width), workspace)) {
        if (PyErr_Occurred()) return nullptr;
        Py_RETURN_NONE;
    }
    if (workspace.defined() && !here(workspace)) Py_RETURN_NONE;
    at::Tensor out = a[6] != Py_None ? tensor(a[6]) : at::Tensor();
    int rc;
    {
        const WithoutGil released;
        if (!out.defined()) out = at::empty({T, Hq, c.dim}, q.options());
        rc = layer.chunks(dtype_of(q), (int)S, (int)T, (int)Hq, c.heads, c.dim, q.data_ptr(), q.stride(0), q.stride(1), ints(a[4]), c.p, c.pages, c.page,
                          ints(a[2]), width, ints(a[3]), (float)scale, out.data_ptr(), workspace.defined() ? workspace.data_ptr() : nullptr,
                          workspace.defined() ? (size_t)workspace.numel() : 0, stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return wrapped(a[6], std::move(out));
    END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------- norm and gated activation, tokens sorted by expert and back
// a matrix whose rows may have a stride of their own
bool matrix(PyObject *o, at::ScalarType type)
{
    if (rows_of(o, type) < 0) return false;
    const at::Tensor &t = tensor(o);
    return t.size(1) > 1 && t.stride(1) == 1 && !wants_gradient(o) && here(t);
}
bool matrix_of(PyObject *o, const at::Tensor &like) { return matrix(o, like.scalar_type()) && tensor(o).sizes().equals(like.sizes()); }
bool float16(PyObject *o) { return matrix(o, at::kHalf) || matrix(o, at::kBFloat16); }
// None, or a contiguous tensor
bool given(PyObject *o, at::ScalarType type, std::initializer_list<int64_t> shape) { return o == Py_None || (plain(o, type, shape) && !wants_gradient(o) && here(tensor(o))); }
template <class T = void>
T *pointer(PyObject *o) { return o == Py_None ? nullptr : static_cast<T *>(tensor(o).data_ptr()); }
at::Tensor given_or_none(PyObject *o) { return o == Py_None ? at::Tensor() : tensor(o); }
PyObject *tuple_of(std::initializer_list<PyObject *> items)  // (takes the references)
{
    bool whole = true;
    for (PyObject *const o : items) whole = whole && o;
    PyObject *const t = whole ? PyTuple_New((Py_ssize_t)items.size()) : nullptr;
    Py_ssize_t i = 0;
    for (PyObject *const o : items) {
        if (t)
            PyTuple_SET_ITEM(t, i++, o);
        else
            Py_XDECREF(o);
    }
    return t;
}
PyObject *none() { Py_RETURN_NONE; }

// norm(x, weight, residual, eps, want_y, out_q, out_scales, out_h, out_y, stream) -> (X_i8, act_scales, h or None, y or None)
PyObject *norm(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    if (n != 10 || !float16(a[0]) || !PyFloat_CheckExact(a[3]) || !PyBool_Check(a[4])) Py_RETURN_NONE;
    const at::Tensor &x = tensor(a[0]);
    const int64_t M = x.size(0), K = x.size(1);
    const bool residual = a[2] != Py_None, want_y = a[4] == Py_True;
    if (!given(a[1], at::kFloat, {K}) || (residual && !matrix_of(a[2], x)) || (!residual && a[7] != Py_None) || !given(a[5], at::kChar, {M, K}) ||
        !given(a[6], at::kFloat, {M}) || !given(a[7], x.scalar_type(), {M, K}) || !given(a[8], x.scalar_type(), {M, K}) || !stream_of(a[9], stream))
        Py_RETURN_NONE;
    at::Tensor q = given_or_none(a[5]), s = given_or_none(a[6]), h = given_or_none(a[7]), y = given_or_none(a[8]);
    int rc;
    {
        const WithoutGil released;
        if (!q.defined()) q = at::empty({M, K}, x.options().dtype(at::kChar));
        if (!s.defined()) s = at::empty({M}, x.options().dtype(at::kFloat));
        if (residual && !h.defined()) h = at::empty({M, K}, x.options());
        if (want_y && !y.defined()) y = at::empty({M, K}, x.options());
        rc = layer.norm(dtype_of(x), (int)M, (int)K, x.data_ptr(), x.stride(0), pointer(a[2]), residual ? tensor(a[2]).stride(0) : 0, floats(a[1]),
                        (float)PyFloat_AS_DOUBLE(a[3]), residual ? h.data_ptr() : nullptr, want_y ? y.data_ptr() : nullptr,
                        static_cast<int8_t *>(q.data_ptr()), static_cast<float *>(s.data_ptr()), stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return tuple_of({wrapped(a[5], std::move(q)), wrapped(a[6], std::move(s)), residual ? wrapped(a[7], std::move(h)) : none(),
                     want_y ? wrapped(a[8], std::move(y)) : none()});
    END_HANDLE_TH_ERRORS
}

// swiglu(x, out_q, out_scales, stream) -> (X_i8, act_scales)
PyObject *swiglu(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    if (n != 4 || !float16(a[0]) || tensor(a[0]).size(1) % 2) Py_RETURN_NONE;
    const at::Tensor &x = tensor(a[0]);
    const int64_t M = x.size(0), K = x.size(1) / 2;
    if (!given(a[1], at::kChar, {M, K}) || !given(a[2], at::kFloat, {M}) || !stream_of(a[3], stream)) Py_RETURN_NONE;
    at::Tensor q = given_or_none(a[1]), s = given_or_none(a[2]);
    int rc;
    {
        const WithoutGil released;
        if (!q.defined()) q = at::empty({M, K}, x.options().dtype(at::kChar));
        if (!s.defined()) s = at::empty({M}, x.options().dtype(at::kFloat));
        rc = layer.swiglu(dtype_of(x), (int)M, (int)K, x.data_ptr(), x.stride(0), static_cast<int8_t *>(q.data_ptr()), static_cast<float *>(s.data_ptr()), stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return pair(wrapped(a[1], std::move(q)), wrapped(a[2], std::move(s)));
    END_HANDLE_TH_ERRORS
}

// dispatch(X, experts, n_experts, act_scales, out, out_scales, stream) -> (rows, row_scales or None, row_offsets, places)
PyObject *dispatch(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    int n_experts;
    if (n != 7 || !(matrix(a[0], at::kChar) || float16(a[0])) || !plain_dims(a[1], at::kInt, 2) || !here(tensor(a[1])) || !small_int(a[2], n_experts) ||
        n_experts < 1 || n_experts > 256)
        Py_RETURN_NONE;
    const at::Tensor &x = tensor(a[0]);
    const int64_t T = x.size(0), K = x.size(1), each = tensor(a[1]).size(1);
    const bool scales = a[3] != Py_None;
    if (tensor(a[1]).size(0) != T || each < 1 || T * each > INT_MAX || !given(a[3], at::kFloat, {T}) || !given(a[4], x.scalar_type(), {T * each, K}) ||
        (!scales && a[5] != Py_None) || !given(a[5], at::kFloat, {T * each}) || !stream_of(a[6], stream))
        Py_RETURN_NONE;
    at::Tensor rows = given_or_none(a[4]), row_scales = given_or_none(a[5]), offsets, places;
    int rc;
    {
        const WithoutGil released;
        if (!rows.defined()) rows = at::empty({T * each, K}, x.options());
        if (scales && !row_scales.defined()) row_scales = at::empty({T * each}, x.options().dtype(at::kFloat));
        offsets = at::empty({n_experts + 1}, x.options().dtype(at::kInt));
        places = at::empty({T, each}, x.options().dtype(at::kInt));
        rc = layer.dispatch(x.scalar_type() == at::kChar ? LQ_I8 : dtype_of(x), (int)T, (int)each, n_experts, (int)K, x.data_ptr(), x.stride(0), floats(a[3]),
                            ints(a[1]), rows.data_ptr(), scales ? static_cast<float *>(row_scales.data_ptr()) : nullptr,
                            static_cast<int *>(offsets.data_ptr()), static_cast<int *>(places.data_ptr()), stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return tuple_of({wrapped(a[4], std::move(rows)), scales ? wrapped(a[5], std::move(row_scales)) : none(), THPVariable_Wrap(std::move(offsets)),
                     THPVariable_Wrap(std::move(places))});
    END_HANDLE_TH_ERRORS
}

// combine(Y, places, weights, out, stream) -> out
PyObject *combine(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    if (n != 5 || !float16(a[0]) || !plain_dims(a[1], at::kInt, 2) || !here(tensor(a[1]))) Py_RETURN_NONE;
    const at::Tensor &y = tensor(a[0]);
    const int64_t T = tensor(a[1]).size(0), each = tensor(a[1]).size(1), R = y.size(0), N = y.size(1);
    if (!given(a[2], at::kFloat, {T, each}) || !given(a[3], y.scalar_type(), {T, N}) || !stream_of(a[4], stream)) Py_RETURN_NONE;
    at::Tensor out = given_or_none(a[3]);
    int rc;
    {
        const WithoutGil released;
        if (!out.defined()) out = at::empty({T, N}, y.options());
        rc = layer.combine(dtype_of(y), (int)T, (int)each, (int)R, (int)N, y.data_ptr(), y.stride(0), ints(a[1]), floats(a[2]), out.data_ptr(), stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return wrapped(a[3], std::move(out));
    END_HANDLE_TH_ERRORS
}

// combine_backward(grad, Y, places, weights, row_offsets, out_Y, out_weights, stream) -> (grad_Y, grad_weights)
PyObject *combine_backward(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    HANDLE_TH_ERRORS
    void *stream;
    if (n != 8 || !float16(a[1]) || !matrix(a[0], tensor(a[1]).scalar_type()) || !plain_dims(a[2], at::kInt, 2) || !here(tensor(a[2]))) Py_RETURN_NONE;
    const at::Tensor &grad = tensor(a[0]), &y = tensor(a[1]);
    const int64_t T = tensor(a[2]).size(0), each = tensor(a[2]).size(1), R = y.size(0), N = y.size(1);
    const bool used = a[4] != Py_None;
    if (grad.size(0) != T || grad.size(1) != N || a[3] == Py_None || !given(a[3], at::kFloat, {T, each}) ||
        (used && (!plain_dims(a[4], at::kInt, 1) || tensor(a[4]).size(0) < 1 || !here(tensor(a[4])))) || !given(a[5], y.scalar_type(), {R, N}) ||
        !given(a[6], at::kFloat, {T, each}) || !stream_of(a[7], stream))
        Py_RETURN_NONE;
    at::Tensor out = given_or_none(a[5]), weights = given_or_none(a[6]);
    if (!out.defined() && !used) Py_RETURN_NONE;  // (cleared on the current stream: the general path does it)
    int rc;
    {
        const WithoutGil released;
        if (!out.defined()) out = at::empty({R, N}, y.options());
        if (!weights.defined()) weights = at::empty({T, each}, y.options().dtype(at::kFloat));
        rc = layer.combine_backward(dtype_of(y), (int)T, (int)each, (int)R, (int)N, grad.data_ptr(), grad.stride(0), y.data_ptr(), y.stride(0), ints(a[2]),
                                    floats(a[3]), used ? ints(a[4]) + tensor(a[4]).size(0) - 1 : nullptr, out.data_ptr(),
                                    static_cast<float *>(weights.data_ptr()), stream);
    }
    if (rc != LQ_OK) return PyLong_FromLong(rc);
    return pair(wrapped(a[5], std::move(out)), wrapped(a[6], std::move(weights)));
    END_HANDLE_TH_ERRORS
}

// bind_layer(kv4_attention_chunks_workspace_size, kv4_attention_chunks, w4a8_norm_quantize, w4a8_swiglu_quantize, moe_dispatch, moe_combine,
// moe_combine_backward): their addresses
PyObject *bind_layer(PyObject *, PyObject *args)
{
    unsigned long long z, c, n, s, d, m, b;
    if (!PyArg_ParseTuple(args, "KKKKKKK", &z, &c, &n, &s, &d, &m, &b)) return nullptr;
    layer = Layer{reinterpret_cast<decltype(layer.chunks_workspace_size)>(z), reinterpret_cast<decltype(layer.chunks)>(c),
                  reinterpret_cast<decltype(layer.norm)>(n), reinterpret_cast<decltype(layer.swiglu)>(s), reinterpret_cast<decltype(layer.dispatch)>(d),
                  reinterpret_cast<decltype(layer.combine)>(m), reinterpret_cast<decltype(layer.combine_backward)>(b)};
    Py_RETURN_NONE;
}

// bind_attention(attn_qk_norm_rope, kv4_write, kv4_append, kv4_read, kv4_attention_workspace_size, kv4_attention,
// attn_prompt_workspace_size, attn_prompt): their addresses
PyObject *bind_attention(PyObject *, PyObject *args)
{
    unsigned long long r, w, a, d, s, t, z, p;
    if (!PyArg_ParseTuple(args, "KKKKKKKK", &r, &w, &a, &d, &s, &t, &z, &p)) return nullptr;
    attn = Attention{reinterpret_cast<decltype(attn.rope)>(r), reinterpret_cast<decltype(attn.write)>(w), reinterpret_cast<decltype(attn.append)>(a),
                     reinterpret_cast<decltype(attn.read)>(d), reinterpret_cast<decltype(attn.workspace_size)>(s),
                     reinterpret_cast<decltype(attn.decode)>(t),
                     reinterpret_cast<decltype(attn.prompt_workspace_size)>(z), reinterpret_cast<decltype(attn.prompt)>(p)};
    Py_RETURN_NONE;
}

// bind(w4a8_gemm, w4a8_gemm_workspace_size, w4a8_quantize_activations, w4a8_grouped_gemm, liquidquant_packed_size): their addresses
PyObject *bind(PyObject *, PyObject *args)
{
    unsigned long long g, w, q, m, p;
    if (!PyArg_ParseTuple(args, "KKKKK", &g, &w, &q, &m, &p)) return nullptr;
    lib = Library{reinterpret_cast<decltype(lib.gemm)>(g), reinterpret_cast<decltype(lib.workspace_size)>(w),
                  reinterpret_cast<decltype(lib.quantize)>(q), reinterpret_cast<decltype(lib.grouped)>(m),
                  reinterpret_cast<decltype(lib.packed_size)>(p)};
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(quantize)), METH_FASTCALL, nullptr},
    {"gemm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(gemm)), METH_FASTCALL, nullptr},
    {"grouped", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(grouped)), METH_FASTCALL, nullptr},
    {"rope", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(rope)), METH_FASTCALL, nullptr},
    {"write", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(write)), METH_FASTCALL, nullptr},
    {"append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(append)), METH_FASTCALL, nullptr},
    {"read", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(read)), METH_FASTCALL, nullptr},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(decode)), METH_FASTCALL, nullptr},
    {"prompt", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(prompt)), METH_FASTCALL, nullptr},
    {"chunks", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(chunks)), METH_FASTCALL, nullptr},
    {"norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(norm)), METH_FASTCALL, nullptr},
    {"swiglu", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(swiglu)), METH_FASTCALL, nullptr},
    {"dispatch", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(dispatch)), METH_FASTCALL, nullptr},
    {"combine", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(combine)), METH_FASTCALL, nullptr},
    {"combine_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(combine_backward)), METH_FASTCALL, nullptr},
    {"bind", bind, METH_VARARGS, nullptr},
    {"bind_layer", bind_layer, METH_VARARGS, nullptr},
    {"bind_attention", bind_attention, METH_VARARGS, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module{PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__binding()
{
    PyObject *const m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", BUILT_FOR) == 0) return m;  // (api.py looks at it before the first call)
    Py_XDECREF(m);
    return nullptr;
}
