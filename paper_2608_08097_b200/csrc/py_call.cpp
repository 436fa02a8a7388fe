// Python calls of the draft-tree operators, of the packed cache and of the rotary positions: checks the tensors and makes the call
// of the C ABI.
//
// The smallest of these calls take the GPU 3 to 9 us, and checking ten tensors from Python and converting twenty arguments
// for a foreign function takes 5 to 7 us beside the launch's 3: a decode loop that is not captured in a graph would wait for
// its host.  Here a tensor's type, shape, device and layout are read in nanoseconds.  What is refused, and with which
// exception, is what the other calls of the binding refuse.
#include <Python.h>

#include <climits>
#include <initializer_list>
#include <string>
#include <vector>

#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/oasis.h"

namespace {

// The entry points of the library that the binding has loaded (`bind`).
decltype(&oasis_tree_attn) g_tree_attn = nullptr;
decltype(&oasis_verify_tree) g_verify_tree = nullptr;
decltype(&oasis_commit_kv_layers_after_select) g_commit_kv_layers = nullptr;
decltype(&oasis_pack_blocks) g_pack_blocks = nullptr;
decltype(&oasis_unpack_blocks) g_unpack_blocks = nullptr;
decltype(&oasis_packed_attn) g_packed_attn = nullptr;
decltype(&oasis_rotate_qkv) g_rotate_qkv = nullptr;

struct Refused {
    PyObject *type;
    std::string text;
};
struct Raised {};                                          // a Python exception is set

[[noreturn]] void refuse(PyObject *type, const std::string &text) { throw Refused{type, text}; }

template <typename F>
PyObject *guarded(F &&body)
{
    try {
        return body();
    } catch (const Refused &r) {
        PyErr_SetString(r.type, r.text.c_str());
    } catch (const Raised &) {
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "unknown C++ exception");
    }
    return nullptr;
}

std::string text_of(at::IntArrayRef shape)
{
    std::string s = "(";
    for (size_t i = 0; i < shape.size(); ++i) s += (i ? ", " : "") + std::to_string(shape[i]);
    return s + ")";
}

const at::Tensor &tensor(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) refuse(PyExc_TypeError, std::string(name) + ": expected a tensor");
    return THPVariable_Unpack(o);
}

void on_device(const at::Tensor &t, const char *name, int device, const char *or_else = "")
{
    if (!t.is_cuda() || t.get_device() != device)
        refuse(PyExc_ValueError, std::string(name) + " must be on the current CUDA device" + or_else);
}

void of_type(const at::Tensor &t, at::ScalarType type, const char *name)
{
    if (t.scalar_type() != type)
        refuse(PyExc_TypeError, std::string(name) + ": expected " + c10::toString(type) + ", got " + c10::toString(t.scalar_type()));
}

// Address of a dense tensor of this type and shape on `device`.
void *dense(PyObject *o, at::ScalarType type, at::IntArrayRef want, const char *name, int device)
{
    const at::Tensor &t = tensor(o, name);
    of_type(t, type, name);
    if (t.sizes() != want) refuse(PyExc_ValueError, std::string(name) + ": expected shape " + text_of(want) + ", got " + text_of(t.sizes()));
    on_device(t, name, device);
    if (!t.is_contiguous()) refuse(PyExc_ValueError, std::string(name) + " must be contiguous");
    return t.data_ptr();
}
void *dense(PyObject *o, at::ScalarType type, std::initializer_list<int64_t> shape, const char *name, int device)
{
    return dense(o, type, at::IntArrayRef(shape.begin(), shape.size()), name, device);
}
void *dense_or_null(PyObject *o, at::ScalarType type, std::initializer_list<int64_t> shape, const char *name, int device)
{
    return o == Py_None ? nullptr : dense(o, type, shape, name, device);
}

// Address of a pool of entries [..][2][16][128] in device memory (or, `host_ok`, in pinned host memory).
void *pool(PyObject *o, const char *name, int device, bool host_ok = false)
{
    const at::Tensor &t = tensor(o, name);
    of_type(t, at::kBFloat16, name);
    const int64_t n = t.dim();
    if (n < 3 || t.size(n - 3) != 2 || t.size(n - 2) != 16 || t.size(n - 1) != 128 || !t.is_contiguous())
        refuse(PyExc_ValueError, std::string(name) + " must be a contiguous pool of [2][16][128] entries");
    if (!(host_ok && t.is_cpu() && t.is_pinned())) on_device(t, name, device, host_ok ? " or in pinned host memory" : "");
    return t.data_ptr();
}

// Address of packed entries [..][2304] in device memory (or, `host_ok`, in pinned host memory).
void *packed_entries(PyObject *o, const char *name, int device, bool host_ok = false)
{
    const at::Tensor &t = tensor(o, name);
    of_type(t, at::kByte, name);
    if (t.dim() < 1 || t.size(t.dim() - 1) != OASIS_PACKED_BYTES || !t.is_contiguous())
        refuse(PyExc_ValueError, std::string(name) + " must be contiguous packed entries of " + std::to_string(OASIS_PACKED_BYTES) + " bytes");
    if (!(host_ok && t.is_cpu() && t.is_pinned())) on_device(t, name, device, host_ok ? " or in pinned host memory" : "");
    return t.data_ptr();
}

struct Rows {
    void *data;
    int64_t batch_stride, row_stride;
};
// A [B][T][V] tensor whose rows are dense.
Rows rows(const at::Tensor &t, const char *name, int64_t B, int64_t T, int64_t V, int device)
{
    const int64_t want[3] = {B, T, V};
    if (t.sizes() != at::IntArrayRef(want, 3))
        refuse(PyExc_ValueError, std::string(name) + ": expected shape " + text_of(at::IntArrayRef(want, 3)) + ", got " + text_of(t.sizes()));
    on_device(t, name, device);
    int64_t sb = t.stride(0), sr = t.stride(1);
    if (t.stride(2) != 1 && V > 1) refuse(PyExc_ValueError, std::string(name) + ": the rows must be dense");
    if (T == 1 && sr < V) sr = V;                          // (the stride of a single row means nothing)
    if (sr < V || (sb < 0 && B > 1)) refuse(PyExc_ValueError, std::string(name) + ": rows must not overlap");
    return {t.data_ptr(), sb < 0 ? 0 : sb, sr};
}

int32_t narrow(int64_t v, const char *name)
{
    if (v > INT_MAX || v < INT_MIN) refuse(PyExc_ValueError, std::string(name) + " is too large");
    return (int32_t)v;
}

int64_t integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}
template <typename T>
T address(PyObject *o)
{
    void *p = PyLong_AsVoidPtr(o);
    if (!p && PyErr_Occurred()) throw Raised{};
    return reinterpret_cast<T>(p);
}

void *stream_of(PyObject *o, int device)                   // a raw handle, or None: the current stream
{
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    return address<void *>(o);
}

void takes(Py_ssize_t n, Py_ssize_t want)
{
    if (n != want) refuse(PyExc_TypeError, "expected " + std::to_string(want) + " arguments");
}

template <typename F>
PyObject *status(F &&call)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = call();
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(rc);
}

PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        takes(n, 7);
        g_tree_attn = address<decltype(g_tree_attn)>(a[0]);
        g_verify_tree = address<decltype(g_verify_tree)>(a[1]);
        g_commit_kv_layers = address<decltype(g_commit_kv_layers)>(a[2]);
        g_pack_blocks = address<decltype(g_pack_blocks)>(a[3]);
        g_unpack_blocks = address<decltype(g_unpack_blocks)>(a[4]);
        g_packed_attn = address<decltype(g_packed_attn)>(a[5]);
        g_rotate_qkv = address<decltype(g_rotate_qkv)>(a[6]);
        Py_RETURN_NONE;
    });
}

// addresses(tensors, kind, shape, name): the addresses of a list of tensors, one pointer after the other.  Kind 0: dense bf16 of
// this shape, 1: dense int32 of this shape, 2: pools of entries in device memory, 3: the same or in pinned host memory, or None,
// 4: packed entries in device memory or in pinned host memory, 5: dense int64 of this shape, 6: dense bf16 of this shape, or None.
PyObject *addresses(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        takes(n, 4);
        if (!PyList_Check(a[0]) || !PyTuple_Check(a[2])) refuse(PyExc_TypeError, "addresses: expected a list and a tuple");
        const int64_t kind = integer(a[1]);
        std::vector<int64_t> shape;
        for (Py_ssize_t i = 0; i < PyTuple_GET_SIZE(a[2]); ++i) shape.push_back(integer(PyTuple_GET_ITEM(a[2], i)));
        const char *name = PyUnicode_AsUTF8(a[3]);
        if (!name) throw Raised{};
        const int device = c10::cuda::current_device();
        std::vector<const void *> got;
        for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[0]); ++i) {
            PyObject *t = PyList_GET_ITEM(a[0], i);
            if ((kind == 3 || kind == 6) && t == Py_None) got.push_back(nullptr);
            else if (kind == 4) got.push_back(packed_entries(t, name, device, true));
            else if (kind == 2 || kind == 3) got.push_back(pool(t, name, device, kind == 3));
            else got.push_back(dense(t, kind == 1 ? at::kInt : kind == 5 ? at::kLong : at::kBFloat16, at::IntArrayRef(shape), name, device));
        }
        return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(got.data()), (Py_ssize_t)(got.size() * sizeof(void *)));
    });
}

// tree_attn(dims, q, tree_kv, parent, n_nodes, hbm_pool, slot_tbl, blk_tbl, seq_len, scale, out, lse, workspace, stream)
PyObject *tree_attn(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        takes(n, 14);
        const auto *dims = address<const oasis_dims_t *>(a[0]);
        const int device = c10::cuda::current_device();
        const int64_t B = dims->batch, Hq = dims->n_q_heads, Hkv = dims->n_kv_heads;
        const at::Tensor &q = tensor(a[1], "q"), &table = tensor(a[7], "blk_tbl");
        if (q.dim() != 4) refuse(PyExc_ValueError, "q: expected shape [B][T][Hq][128], got " + text_of(q.sizes()));
        if (table.dim() != 3) refuse(PyExc_ValueError, "blk_tbl: expected shape [B][Hkv][columns], got " + text_of(table.sizes()));
        const int64_t T = q.size(1), cols = table.size(2);
        void *ws = nullptr;
        size_t ws_bytes = 0;
        if (a[12] != Py_None) {
            const at::Tensor &w = tensor(a[12], "workspace");
            if (!w.is_cuda() || w.get_device() != device || !w.is_contiguous())
                refuse(PyExc_ValueError, "workspace must be contiguous and on the current CUDA device");
            ws = w.data_ptr();
            ws_bytes = w.nbytes();
        }
        const double scale = PyFloat_AsDouble(a[9]);
        if (scale == -1.0 && PyErr_Occurred()) throw Raised{};
        const void *pq = dense(a[1], at::kBFloat16, {B, T, Hq, 128}, "q", device);
        const void *kv = dense(a[2], at::kBFloat16, {B, T, Hkv, 2, 128}, "tree_kv", device);
        const auto *parent = (const int32_t *)dense(a[3], at::kInt, {B, T}, "parent", device);
        const auto *nodes = (const int32_t *)dense(a[4], at::kInt, {B}, "n_nodes", device);
        const void *entries = pool(a[5], "hbm_pool", device);
        const auto *slot = (const int32_t *)dense(a[6], at::kInt, {B, Hkv, cols}, "slot_tbl", device);
        const auto *blk = (const int32_t *)dense(a[7], at::kInt, {B, Hkv, cols}, "blk_tbl", device);
        const auto *len = (const int32_t *)dense(a[8], at::kInt, {B}, "seq_len", device);
        void *out = dense(a[10], at::kBFloat16, {B, T, Hq, 128}, "out", device);
        auto *lse = (float *)dense_or_null(a[11], at::kFloat, {B, T, Hq}, "lse", device);
        const int32_t t = narrow(T, "n_tree"), c = narrow(cols, "n_cols");
        void *stream = stream_of(a[13], device);
        return status([&] {
            return g_tree_attn(dims, pq, t, kv, parent, nodes, entries, slot, blk, c, len, (float)scale, out, lse, ws, ws_bytes, stream);
        });
    });
}

// verify_tree(logits, tokens, parent, n_nodes, uniforms, temperature, path, n_commit, next_token, draft_probs, stream)
PyObject *verify_tree(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        takes(n, 11);
        const at::Tensor &logits = tensor(a[0], "logits");
        int type;
        switch (logits.scalar_type()) {
        case at::kFloat: type = OASIS_F32; break;
        case at::kBFloat16: type = OASIS_BF16; break;
        case at::kHalf: type = OASIS_F16; break;
        default: refuse(PyExc_TypeError, std::string("logits: expected Float, BFloat16 or Half, got ") + c10::toString(logits.scalar_type()));
        }
        if (logits.dim() != 3) refuse(PyExc_ValueError, "logits must be [B][T][V]");
        const int device = c10::cuda::current_device();
        const int64_t B = logits.size(0), T = logits.size(1), V = logits.size(2);
        const Rows l = rows(logits, "logits", B, T, V, device);
        Rows d = {nullptr, 0, 0};
        if (a[9] != Py_None) {
            const at::Tensor &draft = tensor(a[9], "draft_probs");
            of_type(draft, at::kFloat, "draft_probs");
            d = rows(draft, "draft_probs", B, T, V, device);
        }
        const at::Tensor &kept = tensor(a[6], "path");
        if (kept.dim() != 2) refuse(PyExc_ValueError, "path: expected shape [B][max_path], got " + text_of(kept.sizes()));
        const int64_t M = kept.size(1);
        const auto *tokens = (const int32_t *)dense(a[1], at::kInt, {B, T}, "tokens", device);
        const auto *parent = (const int32_t *)dense(a[2], at::kInt, {B, T}, "parent", device);
        const auto *nodes = (const int32_t *)dense(a[3], at::kInt, {B}, "n_nodes", device);
        const auto *uniforms = (const float *)dense(a[4], at::kFloat, {B, T}, "uniforms", device);
        const auto *temperature = (const float *)dense(a[5], at::kFloat, {B}, "temperature", device);
        auto *path = (int32_t *)dense(a[6], at::kInt, {B, M}, "path", device);
        auto *n_commit = (int32_t *)dense(a[7], at::kInt, {B}, "n_commit", device);
        auto *next = (int32_t *)dense(a[8], at::kInt, {B}, "next_token", device);
        const int32_t b = narrow(B, "batch"), t = narrow(T, "n_tree"), v = narrow(V, "vocab"), m = narrow(M, "max_path");
        void *stream = stream_of(a[10], device);
        return status([&] {
            return g_verify_tree(b, t, v, l.data, type, l.batch_stride, l.row_stride, tokens, parent, nodes, uniforms, temperature,
                                 (const float *)d.data, d.batch_stride, d.row_stride, path, m, n_commit, next, stream);
        });
    });
}

// commit_kv_layers(plan, path, n_commit, seq_len, next_len, stream, n_candidates), plan = (device, dims, n_layers, tree_kvs, T, block_tables,
// slot_tbls, blk_tbls, n_cols, local_col, pools, host_kvs): numbers and the addresses of arrays that the caller holds
PyObject *commit_kv_layers(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        takes(n, 7);
        if (!PyTuple_Check(a[0]) || PyTuple_GET_SIZE(a[0]) != 12) refuse(PyExc_TypeError, "plan: expected a CommitPlan's tuple");
        const auto item = [&](int i) { return PyTuple_GET_ITEM(a[0], i); };
        const int device = c10::cuda::current_device();
        if (integer(item(0)) != device) refuse(PyExc_ValueError, "the plan's buffers are on another device");
        const auto *dims = address<const oasis_dims_t *>(item(1));
        const int64_t B = dims->batch;
        const at::Tensor &kept = tensor(a[1], "path");
        if (kept.dim() != 2) refuse(PyExc_ValueError, "path: expected shape [B][max_path], got " + text_of(kept.sizes()));
        const int64_t M = kept.size(1);
        const auto *path = (const int32_t *)dense(a[1], at::kInt, {B, M}, "path", device);
        const auto *n_commit = (const int32_t *)dense(a[2], at::kInt, {B}, "n_commit", device);
        const auto *len = (const int32_t *)dense(a[3], at::kInt, {B}, "seq_len", device);
        auto *next = (int32_t *)dense_or_null(a[4], at::kInt, {B}, "next_len", device);
        const auto *candidates = (const int32_t *)dense_or_null(a[6], at::kInt, {B}, "n_candidates", device);
        const int32_t layers = narrow(integer(item(2)), "n_layers"), T = narrow(integer(item(4)), "n_tree"), m = narrow(M, "max_path");
        const int32_t cols = narrow(integer(item(8)), "n_cols"), local = narrow(integer(item(9)), "local_col");
        const auto *kv = address<const void *const *>(item(3));
        const auto *tables = address<const int32_t *const *>(item(5)), *slots = address<const int32_t *const *>(item(6));
        const auto *blks = address<int32_t *const *>(item(7));
        const auto *pools = address<void *const *>(item(10)), *hosts = address<void *const *>(item(11));
        void *stream = stream_of(a[5], device);
        return status([&] {
            return g_commit_kv_layers(dims, layers, kv, T, path, m, n_commit, len, tables, slots, blks, cols, local, pools, hosts, candidates, next, stream);
        });
    });
}

// pack_blocks(dims, kv_pool, src_table, first_block, n_blocks, max_new_blocks, packed, block_table, summaries, stream)
PyObject *pack_blocks(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        takes(n, 10);
        const auto *dims = address<const oasis_dims_t *>(a[0]);
        const int device = c10::cuda::current_device();
        const int64_t B = dims->batch, Hkv = dims->n_kv_heads, mb = dims->max_blocks;
        const void *kv = pool(a[1], "kv_pool", device, true);
        const auto *src = (const int32_t *)dense(a[2], at::kInt, {B, mb}, "src_table", device);
        const auto *first = (const int32_t *)dense(a[3], at::kInt, {B}, "first_block", device);
        const auto *count = (const int32_t *)dense(a[4], at::kInt, {B}, "n_blocks", device);
        const int32_t most = narrow(integer(a[5]), "max_new_blocks");
        void *packed = packed_entries(a[6], "packed", device, true);
        const auto *table = (const int32_t *)dense(a[7], at::kInt, {B, mb}, "block_table", device);
        void *summaries = dense_or_null(a[8], at::kBFloat16, {B, Hkv, mb, 2, 128}, "summaries", device);
        void *stream = stream_of(a[9], device);
        return status([&] { return g_pack_blocks(dims, kv, src, first, count, most, packed, table, summaries, stream); });
    });
}

// unpack_blocks(packed, idx, out, stream)
PyObject *unpack_blocks(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        takes(n, 4);
        const int device = c10::cuda::current_device();
        const void *packed = packed_entries(a[0], "packed", device, true);
        const int64_t items = tensor(a[1], "idx").numel();
        const auto *idx = (const int64_t *)dense(a[1], at::kLong, {items}, "idx", device);
        void *out = dense(a[2], at::kBFloat16, {items, 2, 16, 128}, "out", device);
        const int32_t count = narrow(items, "idx");
        void *stream = stream_of(a[3], device);
        return status([&] { return g_unpack_blocks(packed, idx, count, out, stream); });
    });
}

// packed_attn(dims, q, packed_pool, hbm_pool, slot_tbl, blk_tbl, local_col, seq_len, scale, out, lse, workspace, stream)
PyObject *packed_attn(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        takes(n, 13);
        const auto *dims = address<const oasis_dims_t *>(a[0]);
        const int device = c10::cuda::current_device();
        const int64_t B = dims->batch, Hq = dims->n_q_heads, Hkv = dims->n_kv_heads;
        const at::Tensor &q = tensor(a[1], "q"), &table = tensor(a[5], "blk_tbl");
        if (q.dim() != 4) refuse(PyExc_ValueError, "q: expected shape [B][T][Hq][128], got " + text_of(q.sizes()));
        if (table.dim() != 3) refuse(PyExc_ValueError, "blk_tbl: expected shape [B][Hkv][columns], got " + text_of(table.sizes()));
        const int64_t T = q.size(1), cols = table.size(2);
        void *ws = nullptr;
        size_t ws_bytes = 0;
        if (a[11] != Py_None) {
            const at::Tensor &w = tensor(a[11], "workspace");
            if (!w.is_cuda() || w.get_device() != device || !w.is_contiguous())
                refuse(PyExc_ValueError, "workspace must be contiguous and on the current CUDA device");
            ws = w.data_ptr();
            ws_bytes = w.nbytes();
        }
        const double scale = PyFloat_AsDouble(a[8]);
        if (scale == -1.0 && PyErr_Occurred()) throw Raised{};
        const void *pq = dense(a[1], at::kBFloat16, {B, T, Hq, 128}, "q", device);
        const void *packed = a[2] == Py_None ? nullptr : packed_entries(a[2], "packed_pool", device);
        const void *entries = a[3] == Py_None ? nullptr : pool(a[3], "hbm_pool", device);
        const auto *slot = (const int32_t *)dense(a[4], at::kInt, {B, Hkv, cols}, "slot_tbl", device);
        const auto *blk = (const int32_t *)dense(a[5], at::kInt, {B, Hkv, cols}, "blk_tbl", device);
        const int32_t local = narrow(integer(a[6]), "local_col");
        const auto *len = (const int32_t *)dense(a[7], at::kInt, {B}, "seq_len", device);
        void *out = dense(a[9], at::kBFloat16, {B, T, Hq, 128}, "out", device);
        auto *lse = (float *)dense_or_null(a[10], at::kFloat, {B, T, Hq}, "lse", device);
        const int32_t t = narrow(T, "n_q_tokens"), c = narrow(cols, "n_cols");
        void *stream = stream_of(a[12], device);
        return status([&] {
            return g_packed_attn(dims, pq, t, packed, entries, slot, blk, c, local, len, (float)scale, out, lse, ws, ws_bytes, stream);
        });
    });
}

// rotate_qkv(dims, qkv, freqs, rot_dim, interleaved, factor, q, kv, positions, seq_len, parent, n_nodes, stream)
PyObject *rotate_qkv(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    return guarded([&]() -> PyObject * {
        takes(n, 13);
        const auto *dims = address<const oasis_dims_t *>(a[0]);
        const int device = c10::cuda::current_device();
        const int64_t B = dims->batch, Hq = dims->n_q_heads, Hkv = dims->n_kv_heads, width = (Hq + 2 * Hkv) * 128;
        const at::Tensor &qkv = tensor(a[1], "qkv");
        int type;
        switch (qkv.scalar_type()) {
        case at::kFloat: type = OASIS_F32; break;
        case at::kBFloat16: type = OASIS_BF16; break;
        case at::kHalf: type = OASIS_F16; break;
        default: refuse(PyExc_TypeError, std::string("qkv: expected Float, BFloat16 or Half, got ") + c10::toString(qkv.scalar_type()));
        }
        if (qkv.dim() != 3 || qkv.size(0) != B || qkv.size(2) != width)
            refuse(PyExc_ValueError, "qkv: expected shape [" + std::to_string(B) + "][T][" + std::to_string(width) + "], got " + text_of(qkv.sizes()));
        if (qkv.stride(2) != 1) refuse(PyExc_ValueError, "qkv: the rows must be dense");
        on_device(qkv, "qkv", device);
        const int64_t T = qkv.size(1), rot = integer(a[3]);
        const auto *freqs = (const double *)dense(a[2], at::kDouble, {rot / 2}, "freqs", device);
        const int64_t pairs = integer(a[4]);
        const double factor = PyFloat_AsDouble(a[5]);
        if (factor == -1.0 && PyErr_Occurred()) throw Raised{};
        void *q = dense(a[6], at::kBFloat16, {B, T, Hq, 128}, "q", device);
        void *kv = dense(a[7], at::kBFloat16, {B, T, Hkv, 2, 128}, "kv", device);
        const auto *positions = (const int32_t *)dense_or_null(a[8], at::kInt, {B, T}, "positions", device);
        const auto *len = (const int32_t *)dense_or_null(a[9], at::kInt, {B}, "seq_len", device);
        const auto *parent = (const int32_t *)dense_or_null(a[10], at::kInt, {B, T}, "parent", device);
        const auto *nodes = (const int32_t *)dense_or_null(a[11], at::kInt, {B}, "n_nodes", device);
        const int32_t t = narrow(T, "n_tokens"), r = narrow(rot, "rot_dim");
        const void *from = qkv.data_ptr();
        const int64_t sb = qkv.stride(0), st = qkv.stride(1);
        void *stream = stream_of(a[12], device);
        return status([&] {
            return g_rotate_qkv(dims, from, type, sb, st, t, positions, len, parent, nodes, freqs, r, pairs != 0, (float)factor, q, kv, stream);
        });
    });
}

PyMethodDef methods[] = {
    {"bind", (PyCFunction)(void (*)(void))bind, METH_FASTCALL, nullptr},
    {"addresses", (PyCFunction)(void (*)(void))addresses, METH_FASTCALL, nullptr},
    {"tree_attn", (PyCFunction)(void (*)(void))tree_attn, METH_FASTCALL, nullptr},
    {"verify_tree", (PyCFunction)(void (*)(void))verify_tree, METH_FASTCALL, nullptr},
    {"commit_kv_layers", (PyCFunction)(void (*)(void))commit_kv_layers, METH_FASTCALL, nullptr},
    {"pack_blocks", (PyCFunction)(void (*)(void))pack_blocks, METH_FASTCALL, nullptr},
    {"unpack_blocks", (PyCFunction)(void (*)(void))unpack_blocks, METH_FASTCALL, nullptr},
    {"packed_attn", (PyCFunction)(void (*)(void))packed_attn, METH_FASTCALL, nullptr},
    {"rotate_qkv", (PyCFunction)(void (*)(void))rotate_qkv, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call(void) { return PyModule_Create(&module); }
