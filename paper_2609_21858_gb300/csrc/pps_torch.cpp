// pps_torch.cpp -- the binding's fast path for the target-side calls: checks torch tensors and calls the C ABI.
//
// A decoding step makes these calls once per layer, some of them for a few tokens: 3 us of GPU work behind 10 to 30 us
// of Python checks and ctypes marshalling.  Each function here takes the arguments of its namesake in pps.py in order, and
// returns the result (a tensor, or a dict of them), a status code, or None where anything about the arguments is not as
// the common case has it: pps.py then takes its own way, which says what is wrong or makes the call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cmath>
#include <cstring>

#include <ATen/ATen.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "pps.h"

namespace {

// the library's entry points, handed over by pps.py when it loads a build of libpps
struct Api {
    decltype(&pps_kv_append) append;
    decltype(&pps_paged_attention) attention;
    decltype(&pps_verify_chain) chain;
    decltype(&pps_attention_workspace_size) attention_ws;
    decltype(&pps_chain_workspace_size) chain_ws;
} api = {};

struct NotCommon {};  // left to pps.py

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) throw NotCommon();
    return THPVariable_Unpack(o);
}
// a tensor on device di of type st
const at::Tensor& on(PyObject* o, int di, at::ScalarType st) {
    const at::Tensor& t = tensor(o);
    if (!t.is_cuda() || t.get_device() != di || t.scalar_type() != st) throw NotCommon();
    return t;
}
// address of a contiguous tensor of at least n elements; null for None
template <typename P>
P* flat(PyObject* o, int di, at::ScalarType st, int64_t n) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = on(o, di, st);
    if (t.numel() < n || !t.is_contiguous()) throw NotCommon();
    return static_cast<P*>(t.data_ptr());
}
pps_heads heads(const at::Tensor& t, int64_t n, int64_t h, int64_t d) {
    if (t.dim() != 3 || t.size(0) != n || t.size(1) != h || t.size(2) != d || t.stride(2) != 1) throw NotCommon();
    return {t.data_ptr(), t.stride(0), t.stride(1)};
}
pps_kv_cache cache(PyObject* ko, PyObject* vo, int di, at::ScalarType st, int64_t d) {
    const at::Tensor &k = on(ko, di, st), &v = on(vo, di, st);
    if (k.dim() != 4 || k.size(3) != d || k.stride(3) != 1 || k.sizes() != v.sizes() || k.strides() != v.strides()) throw NotCommon();
    if (k.size(1) > INT32_MAX || k.size(2) > INT32_MAX || d > INT32_MAX) throw NotCommon();
    return {k.data_ptr(), v.data_ptr(), k.size(0), (int32_t)k.size(1), (int32_t)k.size(2), (int32_t)d, k.stride(0), k.stride(1), k.stride(2)};
}
int32_t small(int64_t x) {
    if (x < INT32_MIN || x > INT32_MAX) throw NotCommon();
    return (int32_t)x;
}
double number(PyObject* o) {
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw NotCommon();
    }
    return x;
}
int64_t integer(PyObject* o) {
    if (!PyLong_Check(o)) throw NotCommon();
    const long long x = PyLong_AsLongLong(o);
    if (x == -1 && PyErr_Occurred()) {
        PyErr_Clear();
        throw NotCommon();
    }
    return x;
}
// the queries' device and type; the device has to be the current one
int current_device_of(const at::Tensor& q) {
    if (!q.is_cuda() || q.get_device() != c10::cuda::current_device()) throw NotCommon();
    return (int)q.get_device();
}
int32_t half_code(const at::Tensor& q) {
    if (q.scalar_type() == at::kBFloat16) return PPS_BF16;
    if (q.scalar_type() == at::kHalf) return PPS_F16;
    throw NotCommon();
}

// memory of the caching allocator for the work queued on a stream while it is held
struct Scratch {
    void* p;
    Scratch(size_t n, cudaStream_t s) : p(c10::cuda::CUDACachingAllocator::raw_alloc_with_stream(n ? n : 1, s)) {}
    ~Scratch() { c10::cuda::CUDACachingAllocator::raw_delete(p); }
    Scratch(const Scratch&) = delete;
};

PyObject* new_ref(PyObject* o) {
    Py_INCREF(o);
    return o;
}
// runs f; None where it leaves the call to pps.py
template <class F>
PyObject* common(PyObject* const* a, Py_ssize_t n, Py_ssize_t want, F f) {
    HANDLE_TH_ERRORS
    if (n != want || api.append == nullptr) return new_ref(Py_None);
    try {
        return f(a);
    } catch (const NotCommon&) {
        return new_ref(Py_None);
    }
    END_HANDLE_TH_ERRORS
}

// q, k, v, pos, slot, k_cache, v_cache, rope, q_norm, k_norm, eps, interleaved, out, status
PyObject* kv_append(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return common(args, n_args, 14, [](PyObject* const* a) -> PyObject* {
        const at::Tensor& q = tensor(a[0]);
        const int di = current_device_of(q);
        const at::ScalarType st = q.scalar_type();
        pps_append_args x;
        std::memset(&x, 0, sizeof(x));
        x.size = sizeof(x);
        x.dtype = half_code(q);
        if (q.dim() != 3) throw NotCommon();
        const int64_t n = q.size(0), h = q.size(1), d = q.size(2);
        x.n_tok = n;
        x.n_heads = small(h);
        x.cache = cache(a[5], a[6], di, st, d);
        x.q = heads(q, n, h, d);
        x.k = heads(on(a[1], di, st), n, x.cache.n_kv_heads, d);
        x.v = heads(on(a[2], di, st), n, x.cache.n_kv_heads, d);
        if (a[7] != Py_None) {
            const at::Tensor& r = on(a[7], di, at::kFloat);
            if (r.dim() != 2 || !r.is_contiguous() || a[3] == Py_None) throw NotCommon();
            x.rope = static_cast<const float*>(r.data_ptr());
            x.max_pos = r.size(0);
            x.rot = small(r.size(1));
            x.pos = flat<int32_t>(a[3], di, at::kInt, n);
        }
        if (a[4] == Py_None) throw NotCommon();
        x.slot = flat<int64_t>(a[4], di, at::kLong, n);
        x.q_norm = flat<void>(a[8], di, st, d);
        x.k_norm = flat<void>(a[9], di, st, d);
        x.eps = (float)number(a[10]);
        x.interleaved = a[11] == Py_True ? 1 : a[11] == Py_False ? 0 : throw NotCommon();
        x.status = flat<uint32_t>(a[13], di, at::kInt, 1);
        at::Tensor made;
        if (a[12] == Py_None) {
            made = at::empty({n, h, d}, q.options());
            x.out_q = heads(made, n, h, d);
        } else
            x.out_q = heads(on(a[12], di, st), n, h, d);
        const pps_status code = api.append(&x, (pps_stream_t)c10::cuda::getCurrentCUDAStream(di).stream());
        if (code != PPS_OK) return PyLong_FromLong(code);
        return made.defined() ? THPVariable_Wrap(made) : new_ref(a[12]);
    });
}

// q, k_cache, v_cache, pages, kv_len, q_off, mask, scale, out, lse, ws, status
PyObject* paged_attention(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return common(args, n_args, 12, [](PyObject* const* a) -> PyObject* {
        const at::Tensor& q = tensor(a[0]);
        const int di = current_device_of(q);
        const at::ScalarType st = q.scalar_type();
        pps_attention_args x;
        std::memset(&x, 0, sizeof(x));
        x.size = sizeof(x);
        x.dtype = half_code(q);
        if (q.dim() != 3) throw NotCommon();
        const int64_t n = q.size(0), h = q.size(1), d = q.size(2);
        x.n_tok = n;
        x.n_heads = small(h);
        x.cache = cache(a[1], a[2], di, st, d);
        x.q = heads(q, n, h, d);
        if (a[4] == Py_None || a[5] == Py_None) throw NotCommon();
        const at::Tensor& lens = on(a[4], di, at::kInt);
        const int64_t n_seq = lens.numel();
        x.kv_len = flat<int32_t>(a[4], di, at::kInt, 0);
        x.q_off = flat<int32_t>(a[5], di, at::kInt, n_seq + 1);
        x.n_seq = small(n_seq);
        const at::Tensor& pages = on(a[3], di, at::kInt);
        if (pages.dim() != 2 || pages.size(0) != n_seq || (pages.size(1) > 1 && pages.stride(1) != 1)) throw NotCommon();
        x.pages = static_cast<const int32_t*>(pages.data_ptr());
        x.max_pages = small(pages.size(1));
        x.pages_stride = n_seq > 1 ? pages.stride(0) : pages.size(1);
        if (a[6] != Py_None) {
            const at::Tensor& m = on(a[6], di, at::kInt);
            if (m.dim() != 2 || m.size(0) != n || m.size(1) < 1 || !m.is_contiguous()) throw NotCommon();
            x.mask = static_cast<const uint32_t*>(m.data_ptr());
            x.mask_words = small(m.size(1));
        }
        x.scale = a[7] == Py_None ? (float)(1.0 / std::sqrt((double)d)) : (float)number(a[7]);
        x.out_lse = flat<float>(a[9], di, at::kFloat, n * h);
        x.status = flat<uint32_t>(a[11], di, at::kInt, 1);
        at::Tensor made;
        if (a[8] == Py_None) {
            made = at::empty({n, h, d}, q.options());
            x.out = heads(made, n, h, d);
        } else
            x.out = heads(on(a[8], di, st), n, h, d);
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(di).stream();
        pps_status code;
        if (a[10] != Py_None) {
            x.ws = flat<void>(a[10], di, at::kByte, 0);
            x.ws_bytes = (size_t)tensor(a[10]).numel();
            code = api.attention(&x, (pps_stream_t)stream);
        } else {
            x.ws_bytes = api.attention_ws(n, x.n_heads, x.cache.n_kv_heads, x.cache.head_dim);
            const Scratch ws(x.ws_bytes, stream);
            x.ws = ws.p;
            code = api.attention(&x, (pps_stream_t)stream);
        }
        if (code != PPS_OK) return PyLong_FromLong(code);
        return made.defined() ? THPVariable_Wrap(made) : new_ref(a[8]);
    });
}

// p_logits, q_logits, gamma, seq_off, node_draft_row, draft_tok, u, noise, temperature, ws, status (and outputs of its own)
PyObject* verify_chain(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return common(args, n_args, 11, [](PyObject* const* a) -> PyObject* {
        const at::Tensor& p = tensor(a[0]);
        const int di = current_device_of(p);
        const at::ScalarType st = p.scalar_type();
        pps_chain_args x;
        std::memset(&x, 0, sizeof(x));
        x.size = sizeof(x);
        x.dtype = st == at::kBFloat16 ? PPS_BF16 : st == at::kFloat ? PPS_F32 : throw NotCommon();
        const at::Tensor &q = on(a[1], di, st), &noise = on(a[7], di, at::kFloat);
        if (p.dim() != 2 || q.dim() != 2 || noise.dim() != 2) throw NotCommon();
        const int64_t n = p.size(0), n_draft = q.size(0), V = p.size(1), gamma = integer(a[2]);
        if (q.size(1) != V || noise.size(1) < V || p.stride(1) != 1 || q.stride(1) != 1 || noise.stride(1) != 1) throw NotCommon();
        if (a[3] == Py_None || a[4] == Py_None || a[5] == Py_None || a[6] == Py_None) throw NotCommon();
        const int64_t n_seq = on(a[3], di, at::kInt).numel() - 1;
        if (n_seq < 0 || noise.size(0) < n_seq || gamma < 0) throw NotCommon();
        x.seq_off = flat<int32_t>(a[3], di, at::kInt, n_seq + 1);
        x.node_draft_row = flat<int32_t>(a[4], di, at::kInt, n);
        x.draft_tok = flat<int32_t>(a[5], di, at::kInt, n_draft);
        x.u = flat<float>(a[6], di, at::kFloat, n_draft);
        x.p_logits = p.data_ptr();
        x.q_logits = q.data_ptr();
        x.noise = static_cast<const float*>(noise.data_ptr());
        x.n_nodes = n;
        x.n_draft = n_draft;
        x.vocab = V;
        // of one row, the stride has no meaning
        x.p_stride = n > 1 ? p.stride(0) : V;
        x.q_stride = n_draft > 1 ? q.stride(0) : V;
        x.noise_stride = n_seq > 1 ? noise.stride(0) : V;
        x.n_seq = small(n_seq);
        x.gamma = small(gamma);
        x.temperature = (float)number(a[8]);
        x.status = flat<uint32_t>(a[10], di, at::kInt, 1);
        const auto ints = p.options().dtype(at::kInt);
        at::Tensor acc = at::empty({n_seq}, ints), ne = at::empty({n_seq}, ints), em = at::empty({n_seq, gamma + 1}, ints),
                   prob = at::empty({n_draft}, p.options().dtype(at::kFloat));
        x.out_accept_len = static_cast<int32_t*>(acc.data_ptr());
        x.out_n_emitted = static_cast<int32_t*>(ne.data_ptr());
        x.out_emitted = static_cast<int32_t*>(em.data_ptr());
        x.out_accept_prob = static_cast<float*>(prob.data_ptr());
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(di).stream();
        pps_status code;
        if (a[9] != Py_None) {
            x.ws = flat<void>(a[9], di, at::kByte, 0);
            x.ws_bytes = (size_t)tensor(a[9]).numel();
            code = api.chain(&x, (pps_stream_t)stream);
        } else {
            x.ws_bytes = api.chain_ws(n, n_draft, x.n_seq);
            const Scratch ws(x.ws_bytes, stream);
            x.ws = ws.p;
            code = api.chain(&x, (pps_stream_t)stream);
        }
        if (code != PPS_OK) return PyLong_FromLong(code);
        PyObject* d = PyDict_New();
        if (d == nullptr) return nullptr;
        const std::pair<const char*, at::Tensor*> outs[] = {{"accept_len", &acc}, {"n_emitted", &ne}, {"emitted", &em}, {"accept_prob", &prob}};
        for (const auto& [name, t] : outs) {
            PyObject* o = THPVariable_Wrap(*t);
            const int bad = o == nullptr ? -1 : PyDict_SetItemString(d, name, o);
            Py_XDECREF(o);
            if (bad) {
                Py_DECREF(d);
                return nullptr;
            }
        }
        return d;
    });
}

// the addresses of pps_kv_append, pps_paged_attention, pps_verify_chain and the two workspace sizes
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* p[5];
    if (n != 5) return PyErr_Format(PyExc_TypeError, "five addresses are needed");
    for (int i = 0; i < 5; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (p[i] == nullptr && PyErr_Occurred()) return nullptr;
    }
    api = {reinterpret_cast<decltype(api.append)>(p[0]), reinterpret_cast<decltype(api.attention)>(p[1]),
           reinterpret_cast<decltype(api.chain)>(p[2]), reinterpret_cast<decltype(api.attention_ws)>(p[3]),
           reinterpret_cast<decltype(api.chain_ws)>(p[4])};
    return new_ref(Py_None);
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction fast() {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F));
}

PyMethodDef methods[] = {{"kv_append", fast<kv_append>(), METH_FASTCALL, nullptr},
                         {"paged_attention", fast<paged_attention>(), METH_FASTCALL, nullptr},
                         {"verify_chain", fast<verify_chain>(), METH_FASTCALL, nullptr},
                         {"bind", fast<bind>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "pps_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_pps_torch() { return PyModule_Create(&module); }
