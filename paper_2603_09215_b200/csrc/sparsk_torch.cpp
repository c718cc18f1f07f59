// The paged calls' arguments, from torch tensors to the C ABI's blocks (include/sparsk.h).
//
// Marshalling only, as in binding.py, which wraps these functions: a call of a serving step has five to fourteen tensors, each
// of which is checked for type, device and layout, and in Python that takes longer (6 to 8 us a call) than the kernels
// of a small batch.  The entry points are called through addresses that binding.py hands in, so that this file
// links against torch alone.
#include <Python.h>

#include <cstdint>
#include <exception>
#include <string>

#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/sparsk.h"

namespace {

PyObject *error_class = nullptr;  // binding.SparskError(code, text)
int (*page_map_fn)(const sparsk_page_map_args *, void *) = nullptr;
int (*append_fn)(const sparsk_paged_append_args *, void *) = nullptr;
size_t (*scratch_fn)(const sparsk_paged_attn_args *) = nullptr;
int (*attention_fn)(const sparsk_paged_attn_args *, void *, size_t, void *) = nullptr;
int (*sample_fn)(const sparsk_sample_args *, void *) = nullptr;

struct Refused {
    int code;
    std::string text;
};
[[noreturn]] void refuse(const std::string &text) { throw Refused{SPARSK_EINVAL, text}; }

const at::Tensor &tensor(PyObject *o, const char *what)
{
    if (!THPVariable_Check(o)) refuse(std::string(what) + ": a tensor is wanted");
    return THPVariable_Unpack(o);
}
// The device that a call's tensors are on.
int device_of(const at::Tensor &t, const char *what)
{
    if (!t.is_cuda()) refuse(std::string(what) + ": a tensor on a CUDA device is wanted");
    return t.get_device();
}
void same_device(const at::Tensor &t, int dev, const char *what)
{
    if (!t.is_cuda() || t.get_device() != dev) refuse(std::string(what) + ": a tensor on cuda:" + std::to_string(dev) + " is wanted");
}
// Address of a contiguous array of at least n numbers; None (where that is allowed): NULL.
template <class T>
T *array(PyObject *o, at::ScalarType type, int64_t n, int dev, const char *what, bool may_be_none = false)
{
    if (may_be_none && o == Py_None) return nullptr;
    const at::Tensor &t = tensor(o, what);
    if (t.scalar_type() != type || !t.is_cuda() || t.get_device() != dev || t.numel() < n || !t.is_contiguous())
        refuse(std::string(what) + ": a contiguous array of at least " + std::to_string(n) + " " + c10::toString(type) + " numbers on cuda:" +
               std::to_string(dev) + " is wanted");
    return static_cast<T *>(t.data_ptr());
}
int32_t number(PyObject *o, const char *what)
{
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        refuse(std::string(what) + ": a whole number is wanted");
    }
    if (x < INT32_MIN || x > INT32_MAX) refuse(std::string(what) + ": out of range");
    return (int32_t)x;
}
int32_t size(int64_t x, const char *what)
{
    if (x > INT32_MAX) refuse(std::string(what) + ": too large");
    return (int32_t)x;
}
int type_of(const at::Tensor &t)
{
    switch (t.scalar_type()) {
    case at::kFloat: return SPARSK_FP32;
    case at::kBFloat16: return SPARSK_BF16;
    case at::kHalf: return SPARSK_FP16;
    case at::kFloat8_e4m3fn: return SPARSK_E4M3;
    default: return -1;
    }
}
// Pools as [n_pages, n_kv_heads, page_size, head_dim]; pools whose positions lie before their heads come transposed.
int pool_of(PyObject *ko, PyObject *vo, PyObject *k_scale, PyObject *v_scale, sparsk_page_pool &p)
{
    const at::Tensor &k = tensor(ko, "k_cache"), &v = tensor(vo, "v_cache");
    const int dev = device_of(k, "k_cache");
    if (k.dim() != 4 || k.stride(3) != 1 || v.sizes() != k.sizes() || v.strides() != k.strides() || v.scalar_type() != k.scalar_type() ||
        !v.is_cuda() || v.get_device() != dev)
        refuse("pools: two of one shape, layout and type on one CUDA device, a head's numbers contiguous");
    p.k = k.data_ptr();
    p.v = v.data_ptr();
    p.k_scale = array<float>(k_scale, at::kFloat, k.size(1), dev, "k_scale", true);
    p.v_scale = array<float>(v_scale, at::kFloat, k.size(1), dev, "v_scale", true);
    p.page_stride = k.stride(0); p.head_stride = k.stride(1); p.pos_stride = k.stride(2);
    p.type = type_of(k);
    p.n_pages = size(k.size(0), "pages"); p.n_kv_heads = size(k.size(1), "kv heads");
    p.page_size = size(k.size(2), "page size"); p.head_dim = size(k.size(3), "head_dim");
    return dev;
}
// Address and strides of [n, heads, head_dim].
void *rows(const at::Tensor &t, int64_t n, int64_t heads, int64_t head_dim, int dev, const char *what, int64_t &row_stride, int64_t &head_stride)
{
    same_device(t, dev, what);
    if (t.dim() != 3 || t.size(0) != n || t.size(1) != heads || t.size(2) != head_dim || (head_dim > 1 && t.stride(2) != 1))
        refuse(std::string(what) + ": [" + std::to_string(n) + ", " + std::to_string(heads) + ", " + std::to_string(head_dim) +
               "] is wanted, the last dimension contiguous");
    row_stride = t.stride(0);
    head_stride = t.stride(1);
    return t.data_ptr();
}
int32_t *table(PyObject *o, int64_t n, int dev, int64_t &stride, int32_t &blocks)
{
    const at::Tensor &t = tensor(o, "block_table");
    same_device(t, dev, "block_table");
    if (t.scalar_type() != at::kInt || t.dim() != 2 || t.size(0) < n || (t.size(1) > 1 && t.stride(1) != 1))
        refuse("block_table: int32 [sequences, blocks], a row's entries contiguous");
    // (where one row is read its stride says nothing; rows that share memory, as expanded ones do, have no place of their own
    // for the pages that a step enters, and no distance that the ABI takes)
    if (n > 1 && t.stride(0) < t.size(1)) refuse("block_table: rows that do not overlap are wanted");
    stride = n > 1 ? t.stride(0) : t.size(1);
    blocks = size(t.size(1), "blocks");
    return static_cast<int32_t *>(t.data_ptr());
}
// Python's lock is let go while CUDA is called: a launch waits when the stream's queue is full, and what it waits for may need Python.
struct Unlocked {
    PyThreadState *state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};
// One entry point, on the current stream of device `dev` whichever device is current.
template <class F>
void launch(int dev, const char *what, F f)
{
    int rc;
    Unlocked unlocked;
    if (c10::cuda::current_device() == dev) rc = f(c10::cuda::getCurrentCUDAStream(dev).stream());
    else {
        c10::cuda::CUDAGuard guard((c10::DeviceIndex)dev);
        rc = f(c10::cuda::getCurrentCUDAStream(dev).stream());
    }
    if (rc != SPARSK_OK) throw Refused{rc, what};
}
// What a function does, with every C++ exception turned into a Python one.
template <class F>
PyObject *guarded(Py_ssize_t have, Py_ssize_t want, F f)
{
    if (have != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments are wanted, not %zd", want, have);
        return nullptr;
    }
    try {
        f();
    } catch (const Refused &r) {
        PyObject *e = PyObject_CallFunction(error_class, "is", r.code, r.text.c_str());
        if (e) {
            PyErr_SetObject(error_class, e);
            Py_DECREF(e);
        }
        return nullptr;
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    } catch (...) {
        PyErr_SetString(PyExc_RuntimeError, "an unknown exception");
        return nullptr;
    }
    Py_RETURN_NONE;
}

// (lens, rows, block_table, ring, old_queue, page_size, seq_len, queue, row_start, row_seq, row_pos, slot_map, status)
PyObject *page_map(PyObject *, PyObject *const *x, Py_ssize_t n_args)
{
    return guarded(n_args, 13, [&] {
        const at::Tensor &lens = tensor(x[0], "lens"), &row_seq = tensor(x[9], "row_seq"), &ring = tensor(x[3], "ring");
        const int dev = device_of(lens, "lens");
        const int64_t n = lens.numel(), m = row_seq.numel();
        sparsk_page_map_args a{};
        a.seq_len = array<int32_t>(x[0], at::kInt, n, dev, "lens");
        a.seq_rows = array<int32_t>(x[1], at::kInt, n, dev, "rows");
        a.block_table = table(x[2], n, dev, a.table_stride, a.max_blocks);
        a.ring = array<int32_t>(x[3], at::kInt, 1, dev, "ring");
        a.queue = array<int32_t>(x[4], at::kInt, 2, dev, "old_queue");
        a.seq_len_out = array<int32_t>(x[6], at::kInt, n, dev, "seq_len");
        a.queue_out = array<int32_t>(x[7], at::kInt, 2, dev, "queue");
        a.row_start = array<int32_t>(x[8], at::kInt, n + 1, dev, "row_start");
        a.row_seq = array<int32_t>(x[9], at::kInt, m, dev, "row_seq");
        a.row_pos = array<int32_t>(x[10], at::kInt, m, dev, "row_pos");
        a.slot_map = array<int64_t>(x[11], at::kLong, m, dev, "slot_map");
        a.status = array<int32_t>(x[12], at::kInt, 1, dev, "status");
        a.n_seqs = size(n, "sequences");
        a.page_size = number(x[5], "page_size");
        a.ring_size = size(ring.numel(), "ring");
        a.max_rows = size(m, "rows");
        launch(dev, "sparsk_page_map", [&](void *st) { return page_map_fn(&a, st); });
    });
}

// (k, v, k_cache, v_cache, slot_map, q, q_out, row_pos, rope, k_scale, v_scale)
PyObject *paged_append(PyObject *, PyObject *const *x, Py_ssize_t n_args)
{
    return guarded(n_args, 11, [&] {
        sparsk_paged_append_args a{};
        const int dev = pool_of(x[2], x[3], x[9], x[10], a.pool);
        const at::Tensor &k = tensor(x[0], "k"), &v = tensor(x[1], "v");
        const int64_t n = k.dim() ? k.size(0) : 0, hd = a.pool.head_dim;
        a.k = rows(k, n, a.pool.n_kv_heads, hd, dev, "k", a.k_row_stride, a.k_head_stride);
        a.v = rows(v, n, a.pool.n_kv_heads, hd, dev, "v", a.v_row_stride, a.v_head_stride);
        if (v.scalar_type() != k.scalar_type()) refuse("k and v: of one type");
        a.x_type = type_of(k);
        a.q_out_type = SPARSK_BF16;
        a.slot_map = array<int64_t>(x[4], at::kLong, n, dev, "slot_map");
        if (x[5] != Py_None) {
            const at::Tensor &q = tensor(x[5], "q"), &q_out = tensor(x[6], "q_out");
            const int64_t hq = q.dim() == 3 ? q.size(1) : 0;
            a.q = rows(q, n, hq, hd, dev, "q", a.q_row_stride, a.q_head_stride);
            a.q_out = rows(q_out, n, hq, hd, dev, "q_out", a.q_out_row_stride, a.q_out_head_stride);
            if (q.scalar_type() != k.scalar_type()) refuse("q and k: of one type");
            a.q_out_type = type_of(q_out);
            a.n_q_heads = size(hq, "query heads");
        }
        if (x[8] != Py_None) {
            const at::Tensor &rope = tensor(x[8], "rope");
            if (rope.dim() != 3 || rope.size(1) != hd / 2 || rope.size(2) != 2 || x[7] == Py_None)
                refuse("rope: [positions, head_dim / 2, 2], and row_pos with it");
            a.rope = array<float>(x[8], at::kFloat, 1, dev, "rope");
            a.rope_len = size(rope.size(0), "positions");
            a.row_pos = array<int32_t>(x[7], at::kInt, n, dev, "row_pos");
        }
        a.n_rows = size(n, "rows");
        if (n) launch(dev, "sparsk_paged_append", [&](void *st) { return append_fn(&a, st); });
    });
}

// (q, k_cache, v_cache, block_table, seq_len, row_start, max_rows, max_len, scale, k_scale, v_scale, out, lse, scratch, status)
PyObject *paged_attention(PyObject *, PyObject *const *x, Py_ssize_t n_args)
{
    return guarded(n_args, 15, [&] {
        sparsk_paged_attn_args a{};
        const int dev = pool_of(x[1], x[2], x[9], x[10], a.pool);
        const at::Tensor &q = tensor(x[0], "q"), &out = tensor(x[11], "out"), &lens = tensor(x[4], "seq_len");
        if (q.dim() != 3) refuse("q: [rows, query heads, head_dim] is wanted");
        const int64_t n = q.size(0), hq = q.size(1), n_seqs = lens.numel();
        a.q = rows(q, n, hq, a.pool.head_dim, dev, "q", a.q_row_stride, a.q_head_stride);
        a.out = rows(out, n, hq, a.pool.head_dim, dev, "out", a.out_row_stride, a.out_head_stride);
        if (out.scalar_type() != q.scalar_type()) refuse("q and out: of one type");
        a.q_type = type_of(q);
        a.lse = array<float>(x[12], at::kFloat, n * hq, dev, "lse", true);
        a.block_table = table(x[3], n_seqs, dev, a.table_stride, a.max_blocks);
        a.seq_len = array<int32_t>(x[4], at::kInt, n_seqs, dev, "seq_len");
        a.row_start = array<int32_t>(x[5], at::kInt, n_seqs + 1, dev, "row_start", true);
        a.n_rows = size(n, "rows"); a.n_seqs = size(n_seqs, "sequences"); a.n_q_heads = size(hq, "query heads");
        a.max_rows = number(x[6], "max_rows"); a.max_len = number(x[7], "max_len");
        const double scale = PyFloat_AsDouble(x[8]);
        if (scale == -1.0 && PyErr_Occurred()) {
            PyErr_Clear();
            refuse("scale: a number is wanted");
        }
        a.scale = (float)scale;
        if (scale != 0 && a.scale == 0.f) refuse("scale: too small for fp32, where 0 stands for 1 / sqrt(head_dim)");
        a.status = array<int32_t>(x[14], at::kInt, 1, dev, "status", true);
        if (n == 0) return;
        at::Tensor own;  // (held until the launch; then the stream's order keeps it)
        void *scratch;
        size_t bytes;
        if (x[13] == Py_None) {
            bytes = scratch_fn(&a);
            if (!bytes) refuse("sparsk_paged_attention: a size, type, stride or address that it does not take");
            Unlocked unlocked;
            own = at::empty({(int64_t)bytes}, q.options().dtype(at::kByte));
            scratch = own.data_ptr();
        } else {
            scratch = array<void>(x[13], at::kByte, 1, dev, "scratch");
            bytes = (size_t)tensor(x[13], "scratch").numel();
        }
        launch(dev, "sparsk_paged_attention", [&](void *st) { return attention_fn(&a, scratch, bytes, st); });
    });
}

// (logits, uniforms, temperature, top_k, top_p, min_p, id_lo, id_hi, token, logprob)
PyObject *sample(PyObject *, PyObject *const *x, Py_ssize_t n_args)
{
    return guarded(n_args, 10, [&] {
        const at::Tensor &z = tensor(x[0], "logits");
        const int dev = device_of(z, "logits");
        if (z.dim() != 2 || (z.size(1) > 1 && z.stride(1) != 1)) refuse("logits: [rows, ids], a row's numbers contiguous");
        const int64_t n = z.size(0);
        sparsk_sample_args a{};
        a.logits = z.data_ptr();
        a.uniforms = array<float>(x[1], at::kFloat, n, dev, "uniforms");
        a.temperature = array<float>(x[2], at::kFloat, n, dev, "temperature", true);
        a.top_k = array<int32_t>(x[3], at::kInt, n, dev, "top_k", true);
        a.top_p = array<float>(x[4], at::kFloat, n, dev, "top_p", true);
        a.min_p = array<float>(x[5], at::kFloat, n, dev, "min_p", true);
        a.id_lo = array<int32_t>(x[6], at::kInt, n, dev, "id_lo", true);
        a.id_hi = array<int32_t>(x[7], at::kInt, n, dev, "id_hi", true);
        a.token = array<int32_t>(x[8], at::kInt, n, dev, "token");
        a.logprob = array<float>(x[9], at::kFloat, n, dev, "logprob", true);
        a.row_stride = z.stride(0);
        a.type = type_of(z);
        a.n_rows = size(n, "rows"); a.n_ids = size(z.size(1), "ids");
        if (n) launch(dev, "sparsk_sample", [&](void *st) { return sample_fn(&a, st); });
    });
}

// (SparskError, addresses of the five entry points)
PyObject *bind(PyObject *, PyObject *args)
{
    PyObject *e;
    unsigned long long f[5];
    if (!PyArg_ParseTuple(args, "OKKKKK", &e, &f[0], &f[1], &f[2], &f[3], &f[4])) return nullptr;
    Py_INCREF(e);
    Py_XSETREF(error_class, e);
    page_map_fn = reinterpret_cast<decltype(page_map_fn)>(f[0]);
    append_fn = reinterpret_cast<decltype(append_fn)>(f[1]);
    scratch_fn = reinterpret_cast<decltype(scratch_fn)>(f[2]);
    attention_fn = reinterpret_cast<decltype(attention_fn)>(f[3]);
    sample_fn = reinterpret_cast<decltype(sample_fn)>(f[4]);
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, nullptr},
                         {"page_map", (PyCFunction)(void *)page_map, METH_FASTCALL, nullptr},
                         {"paged_append", (PyCFunction)(void *)paged_append, METH_FASTCALL, nullptr},
                         {"paged_attention", (PyCFunction)(void *)paged_attention, METH_FASTCALL, nullptr},
                         {"sample", (PyCFunction)(void *)sample, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_paged", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__paged() { return PyModule_Create(&module); }
