// Marshalling of torch tensors into the C ABI's arguments for the calls that take a few microseconds on the device (the paged
// cache and the reading of logits): shapes, types, strides and devices are checked here, outputs that the caller does not
// bring are allocated, and the library image of the tensors' 16-bit type is called on the current stream of their device.
// Done in Python the same checks cost 9 to 18 us a call.  The functions of the images are handed over by address once an
// image is loaded (bind), so this module links to neither.
#include <Python.h>

#include <string>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/zeros.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/kraken.h"

namespace {

using at::Tensor;

constexpr int NOT_BOUND = 1;   // (statuses of the ABI are 0 or negative)

struct Image {
    decltype(&kraken_op_paged_append) append;
    decltype(&kraken_op_paged_attention) attention;
    decltype(&kraken_paged_attention_workspace) workspace;
    decltype(&kraken_op_token_logprobs) logprobs;
};
Image images[2];   // bfloat16, half

struct Refused {   // carries the text of a ValueError
    std::string what;
};

void need(bool ok, const char *what) {
    if (!ok) throw Refused{what};
}

const Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) throw Refused{std::string(name) + " must be a tensor"};
    return THPVariable_Unpack(o);
}

bool is_16bit(const Tensor &t) { return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kHalf; }

int to_int32(int64_t v, const char *name) {
    if (v < INT32_MIN || v > INT32_MAX) throw Refused{std::string(name) + " is out of range"};
    return static_cast<int>(v);
}

int int_arg(PyObject *o, const char *name) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused{std::string(name) + " must be an integer"};
    }
    return to_int32(v, name);
}

float float_arg(PyObject *o, const char *name) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw Refused{std::string(name) + " must be a number"};
    }
    return static_cast<float>(v);
}

// Address of a contiguous [n] tensor of the type on `device`; None: NULL
template <typename T>
T *vector(PyObject *o, at::ScalarType type, int64_t n, const at::Device &device, const char *name) {
    if (o == Py_None) return nullptr;
    const Tensor &t = tensor(o, name);
    if (t.scalar_type() != type || t.dim() != 1 || t.size(0) != n || !t.is_contiguous() || t.device() != device)
        throw Refused{std::string(name) + " must be a contiguous " + c10::toString(type) + " [" + std::to_string(n) + "] on " + device.str()};
    return static_cast<T *>(t.data_ptr());
}

uint32_t *status_word(PyObject *o, const at::Device &device) {
    if (o == Py_None) return nullptr;
    const Tensor &t = tensor(o, "status");
    need(t.element_size() == 4 && t.numel() >= 1 && t.device() == device, "status must be a 32-bit word on the device of the other tensors");
    return static_cast<uint32_t *>(t.data_ptr());
}

// The stride of a dimension of one is of no meaning and may be anything: a multiple of 8 in its place
int64_t stride_of(const Tensor &t, int64_t dim) { return t.size(dim) > 1 ? t.stride(dim) : t.size(-1) & ~int64_t(7); }

bool same_strides(const Tensor &a, const Tensor &b) {
    for (int64_t i = 0; i < a.dim(); ++i)
        if (stride_of(a, i) != stride_of(b, i)) return false;
    return true;
}

kraken_paged_cache paged_cache(const Tensor &k, const Tensor &v, const Tensor &table) {
    need(k.is_cuda() && is_16bit(k) && k.dim() == 4 && k.stride(3) == 1,
         "the caches must be 16-bit CUDA tensors [pages, key/value heads, page size, head_dim], contiguous in the last dimension");
    need(v.device() == k.device() && v.scalar_type() == k.scalar_type() && v.sizes() == k.sizes() && v.stride(3) == 1 && same_strides(k, v),
         "k_cache and v_cache must have the same shape, strides, type and device");
    need(table.device() == k.device() && table.scalar_type() == at::kInt && table.dim() == 2 && (table.stride(1) == 1 || table.size(1) <= 1),
         "page_table must be int32 [sequences, pages] on the caches' device, contiguous in the last dimension");
    kraken_paged_cache c;
    c.k = k.data_ptr();
    c.v = v.data_ptr();
    c.page_table = static_cast<const int32_t *>(table.data_ptr());
    c.page_stride = stride_of(k, 0);
    c.head_stride = stride_of(k, 1);
    c.slot_stride = stride_of(k, 2);
    c.table_stride = table.size(0) > 1 ? table.stride(0) : table.size(1);
    c.n_pages = to_int32(k.size(0), "the number of pages");
    c.n_kv_head = to_int32(k.size(1), "the number of key/value heads");
    c.page_size = to_int32(k.size(2), "the page size");
    c.head_dim = to_int32(k.size(3), "head_dim");
    c.n_seqs = to_int32(table.size(0), "the number of sequences");
    c.max_pages = to_int32(table.size(1), "the number of pages of a sequence");
    return c;
}

struct Rows {
    void *p;
    int64_t row, head;
};

// A 16-bit [rows, heads, head_dim] tensor like the caches
Rows rows_of(const Tensor &t, int64_t rows, int64_t heads, const Tensor &like, const char *name) {
    if (t.dim() != 3 || t.size(0) != rows || t.size(1) != heads || t.size(2) != like.size(3) || t.scalar_type() != like.scalar_type() ||
        t.device() != like.device() || t.stride(2) != 1)
        throw Refused{std::string(name) + " must be [" + std::to_string(rows) + ", " + std::to_string(heads) + ", " +
                      std::to_string(like.size(3)) + "] of the caches' type and device, contiguous in the last dimension"};
    return {t.data_ptr(), stride_of(t, 0), stride_of(t, 1)};
}

// A contiguous tensor in `bytes`, from byte `at` on.  An output of its own costs 0.6 us, a part of a common one 0.1.
Tensor part(const Tensor &bytes, int64_t at, at::ScalarType type, at::IntArrayRef sizes) {
    Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(bytes.storage()), bytes.key_set(), c10::scalarTypeToTypeMeta(type));
    c10::TensorImpl *impl = t.unsafeGetTensorImpl();
    impl->set_storage_offset(at / static_cast<int64_t>(c10::elementSize(type)));
    impl->set_sizes_contiguous(sizes);
    return t;
}

PyObject *give(int code, std::initializer_list<Tensor> out) {
    PyObject *r = PyTuple_New(static_cast<Py_ssize_t>(out.size()) + 1);
    if (!r) throw python_error();
    Py_ssize_t i = 0;
    PyTuple_SET_ITEM(r, i++, PyLong_FromLong(code));
    for (const Tensor &t : out) PyTuple_SET_ITEM(r, i++, THPVariable_Wrap(t));   // an undefined tensor: None
    return r;
}

template <typename F>
PyObject *guarded(Py_ssize_t n, Py_ssize_t want, F f) {
    HANDLE_TH_ERRORS
    try {
        need(n == want, "wrong number of arguments");
        return f();
    } catch (const Refused &e) {
        PyErr_SetString(PyExc_ValueError, e.what.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// (k, v, k_cache, v_cache, page_table, positions, row_seq, q, q_out, inv_freq, interleaved, status) -> (code, q_out)
PyObject *paged_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 12, [&] {
        const Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v"), &kc = tensor(a[2], "k_cache"), &vc = tensor(a[3], "v_cache");
        const kraken_paged_cache c = paged_cache(kc, vc, tensor(a[4], "page_table"));
        const at::Device device = kc.device();
        need(k.dim() == 3, "k must be [rows, key/value heads, head_dim]");
        const int64_t rows = k.size(0);
        const Rows kr = rows_of(k, rows, c.n_kv_head, kc, "k"), vr = rows_of(v, rows, c.n_kv_head, kc, "v");
        kraken_paged_append_args g = {};
        g.k = kr.p;
        g.v = vr.p;
        g.k_row_stride = kr.row;
        g.k_head_stride = kr.head;
        g.v_row_stride = vr.row;
        g.v_head_stride = vr.head;
        need(a[5] != Py_None, "positions are needed");
        g.row_pos = vector<const int32_t>(a[5], at::kInt, rows, device, "positions");
        g.row_seq = vector<const int32_t>(a[6], at::kInt, rows, device, "row_seq");
        Tensor out;
        if (a[7] != Py_None) {
            const Tensor &q = tensor(a[7], "q");
            need(q.dim() == 3, "q must be [rows, heads, head_dim]");
            const Rows qr = rows_of(q, rows, q.size(1), kc, "q");
            c10::cuda::CUDAGuard guard(device);
            out = a[8] == Py_None ? at::zeros({rows, q.size(1), q.size(2)}, q.options()) : tensor(a[8], "q_out");
            const Rows outr = rows_of(out, rows, q.size(1), kc, "q_out");
            g.q = qr.p;
            g.q_row_stride = qr.row;
            g.q_head_stride = qr.head;
            g.q_out = outr.p;
            g.q_out_row_stride = outr.row;
            g.q_out_head_stride = outr.head;
            g.n_head = to_int32(q.size(1), "the number of heads");
        }
        if (a[9] != Py_None) {
            const Tensor &f = tensor(a[9], "inv_freq");
            need(f.dim() == 1, "inv_freq must be a vector");
            g.inv_freq = vector<const float>(a[9], at::kFloat, f.size(0), device, "inv_freq");
            g.rot_dim = to_int32(2 * f.size(0), "the rotated width");
        }
        const int interleaved = PyObject_IsTrue(a[10]);
        if (interleaved < 0) throw python_error();
        g.interleaved = interleaved;
        g.rows = to_int32(rows, "the number of rows");
        uint32_t *status = status_word(a[11], device);
        const Image &im = images[kc.scalar_type() == at::kHalf];
        if (!im.append) return give(NOT_BOUND, {Tensor()});
        c10::cuda::CUDAGuard guard(device);
        return give(im.append(&c, &g, status, c10::cuda::getCurrentCUDAStream(device.index()).stream()), {out});
    });
}

// (q, k_cache, v_cache, page_table, n_keys, row_seq, scale or None, score_cap, window, slopes, out, lse, workspace, status)
// -> (code, out, lse)
PyObject *paged_attention(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 14, [&] {
        const Tensor &q = tensor(a[0], "q"), &kc = tensor(a[1], "k_cache"), &vc = tensor(a[2], "v_cache");
        const kraken_paged_cache c = paged_cache(kc, vc, tensor(a[3], "page_table"));
        const at::Device device = kc.device();
        need(q.dim() == 3, "q must be [rows, heads, head_dim]");
        const int64_t rows = q.size(0), heads = q.size(1);
        const Rows qr = rows_of(q, rows, heads, kc, "q");
        const Image &im = images[kc.scalar_type() == at::kHalf];
        if (!im.attention) return give(NOT_BOUND, {Tensor(), Tensor()});
        kraken_paged_attention_args g = {};
        g.q = qr.p;
        g.q_row_stride = qr.row;
        g.q_head_stride = qr.head;
        need(a[4] != Py_None, "n_keys are needed");
        g.n_keys = vector<const int32_t>(a[4], at::kInt, rows, device, "n_keys");
        g.row_seq = vector<const int32_t>(a[5], at::kInt, rows, device, "row_seq");
        g.scale = a[6] == Py_None ? static_cast<float>(1.0 / std::sqrt(static_cast<double>(c.head_dim))) : float_arg(a[6], "scale");
        g.score_cap = float_arg(a[7], "score_cap");
        need(g.score_cap != 0.f || PyFloat_AsDouble(a[7]) == 0.0, "score_cap is too small for 32 bits");   // (0 is no cap)
        g.window = int_arg(a[8], "window");
        g.slopes = vector<const float>(a[9], at::kFloat, heads, device, "slopes");
        g.rows = to_int32(rows, "the number of rows");
        g.n_head = to_int32(heads, "the number of heads");
        uint32_t *status = status_word(a[13], device);
        c10::cuda::CUDAGuard guard(device);
        // out and lse where the caller brings neither: parts of one tensor
        const int64_t out_bytes = rows * heads * q.size(2) * 2;
        Tensor both;
        if (a[10] == Py_None && a[11] == Py_None) both = at::empty({out_bytes + rows * heads * 4}, q.options().dtype(at::kByte));
        const Tensor out = a[10] != Py_None ? tensor(a[10], "out")
                           : both.defined() ? part(both, 0, q.scalar_type(), {rows, heads, q.size(2)})
                                            : at::empty({rows, heads, q.size(2)}, q.options());
        const Rows outr = rows_of(out, rows, heads, kc, "out");
        g.out = outr.p;
        g.out_row_stride = outr.row;
        g.out_head_stride = outr.head;
        const Tensor lse = a[11] != Py_None ? tensor(a[11], "lse")
                           : both.defined() ? part(both, out_bytes, at::kFloat, {rows, heads})
                                            : at::empty({rows, heads}, q.options().dtype(at::kFloat));
        need(lse.device() == device && lse.scalar_type() == at::kFloat && lse.dim() == 2 && lse.size(0) == rows && lse.size(1) == heads &&
                 (lse.stride(1) == 1 || heads <= 1), "lse must be float32 [rows, heads] on the caches' device, contiguous in the last dimension");
        g.lse = static_cast<float *>(lse.data_ptr());
        g.lse_row_stride = lse.stride(0);
        Tensor workspace;
        if (a[12] == Py_None) {
            size_t bytes = 0;
            const int code = im.workspace(g.n_head, c.n_kv_head, c.head_dim, &bytes);
            if (code) return give(code, {Tensor(), Tensor()});
            workspace = at::empty({static_cast<int64_t>(bytes)}, q.options().dtype(at::kByte));
        } else {
            workspace = tensor(a[12], "workspace");
            need(workspace.device() == device && workspace.is_contiguous(), "workspace must be contiguous, on the caches' device");
        }
        g.workspace = workspace.data_ptr();
        g.workspace_bytes = workspace.nbytes();
        return give(im.attention(&c, &g, status, c10::cuda::getCurrentCUDAStream(device.index()).stream()), {out, lse});
    });
}

// (logits, targets, top, scale, status, image for float32) -> (code, logprob, entropy, lse, top_ids, top_logprobs)
PyObject *token_logprobs(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 6, [&] {
        const Tensor &x = tensor(a[0], "logits");
        need(x.is_cuda() && x.dim() == 2 && (x.scalar_type() == at::kFloat || is_16bit(x)),
             "logits must be a CUDA tensor [rows, vocab] of float32 or a 16-bit type");
        need(x.stride(1) == 1 || x.size(1) <= 1, "logits must be contiguous in the last dimension");
        const at::Device device = x.device();
        const int64_t rows = x.size(0);
        kraken_logprobs_args g = {};
        g.logits = x.data_ptr();
        g.row_stride = x.stride(0);
        g.targets = vector<const int32_t>(a[1], at::kInt, rows, device, "targets");
        g.top = int_arg(a[2], "top");
        need(g.top >= 0, "top must not be negative");
        g.scale = float_arg(a[3], "scale");
        g.rows = to_int32(rows, "the number of rows");
        g.vocab = to_int32(x.size(1), "the vocabulary");
        g.dtype = x.scalar_type() != at::kFloat;
        uint32_t *status = status_word(a[4], device);
        const Image &im = images[g.dtype ? x.scalar_type() == at::kHalf : int_arg(a[5], "image") != 0];
        if (!im.logprobs) return give(NOT_BOUND, {Tensor(), Tensor(), Tensor(), Tensor(), Tensor()});
        c10::cuda::CUDAGuard guard(device);
        // 4 rows bytes each: entropy, lse, and logprob where asked for; then the alternatives
        // (no room for lists longer than the library makes: it refuses them before it writes)
        const int64_t row = 4 * rows, numbers = g.targets ? 3 : 2, list = g.top <= KRAKEN_LOGPROBS_MAX_TOP ? row * g.top : 0;
        const Tensor bytes = at::empty({row * numbers + 2 * list}, x.options().dtype(at::kByte));
        const Tensor entropy = part(bytes, 0, at::kFloat, {rows}), lse = part(bytes, row, at::kFloat, {rows});
        Tensor logprob, ids, best;
        if (g.targets) {
            logprob = part(bytes, 2 * row, at::kFloat, {rows});
            g.logprob = static_cast<float *>(logprob.data_ptr());
        }
        if (g.top > 0) {
            best = part(bytes, numbers * row, at::kFloat, {rows, g.top});
            ids = part(bytes, numbers * row + list, at::kInt, {rows, g.top});
            g.top_logprobs = static_cast<float *>(best.data_ptr());
            g.top_ids = static_cast<int32_t *>(ids.data_ptr());
        }
        g.entropy = static_cast<float *>(entropy.data_ptr());
        g.lse = static_cast<float *>(lse.data_ptr());
        return give(im.logprobs(&g, status, c10::cuda::getCurrentCUDAStream(device.index()).stream()), {logprob, entropy, lse, ids, best});
    });
}

// (image, addresses of kraken_op_paged_append, kraken_op_paged_attention, kraken_paged_attention_workspace,
// kraken_op_token_logprobs)
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
    return guarded(n, 5, [&]() -> PyObject * {
        Image im;
        im.append = reinterpret_cast<decltype(im.append)>(PyLong_AsVoidPtr(a[1]));
        im.attention = reinterpret_cast<decltype(im.attention)>(PyLong_AsVoidPtr(a[2]));
        im.workspace = reinterpret_cast<decltype(im.workspace)>(PyLong_AsVoidPtr(a[3]));
        im.logprobs = reinterpret_cast<decltype(im.logprobs)>(PyLong_AsVoidPtr(a[4]));
        if (PyErr_Occurred()) throw python_error();
        images[int_arg(a[0], "image") != 0] = im;
        Py_RETURN_NONE;
    });
}

PyMethodDef methods[] = {
    {"paged_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(paged_append)), METH_FASTCALL, nullptr},
    {"paged_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(paged_attention)), METH_FASTCALL, nullptr},
    {"token_logprobs", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(token_logprobs)), METH_FASTCALL, nullptr},
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(bind)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
    PyObject *m = PyModule_Create(&module);
    if (m) PyModule_AddIntConstant(m, "NOT_BOUND", NOT_BOUND);
    return m;
}
