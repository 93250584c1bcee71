// pps_torch.cpp -- the binding's fast path for the calls of a decoding step: checks torch tensors and calls the C ABI.
//
// A decoding step makes these calls once per layer, some of them for a few tokens: 3 us of GPU work behind 10 to 30 us
// of Python checks and ctypes marshalling.  Each function here takes the arguments of its namesake in pps.py in order, and
// returns the result (a tensor, or a dict of them), a status code, or None where anything about the arguments is not as
// the common case has it: pps.py then takes its own way, which says what is wrong or makes the call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cmath>
#include <cstring>
#include <initializer_list>
#include <type_traits>
#include <utility>

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
    decltype(&pps_kv_append_q4) append_q4;
    decltype(&pps_kv_read_q4) read_q4;
    decltype(&pps_paged_attention_q4) attention_q4;
    decltype(&pps_attention_q4_workspace_size) attention_q4_ws;
    decltype(&pps_kv_reserve) reserve;
    decltype(&pps_kv_trim) trim;
    decltype(&pps_adjust_logits) adjust;
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

// n elements of type st in the memory of `all`, from the element `from` of its own on, as a tensor that owns that memory too
at::Tensor piece(const at::Tensor& all, at::ScalarType st, int64_t from, int64_t n) {
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(all.storage()), all.key_set(), c10::scalarTypeToTypeMeta(st));
    const int64_t size[1] = {n}, stride[1] = {1};
    t.unsafeGetTensorImpl()->set_sizes_and_strides(c10::IntArrayRef(size), c10::IntArrayRef(stride),
                                                   from * (int64_t)all.element_size() / (int64_t)c10::elementSize(st));
    return t;
}
// a dict of tensors
PyObject* dict_of(std::initializer_list<std::pair<const char*, at::Tensor*>> outs) {
    PyObject* d = PyDict_New();
    if (d == nullptr) return nullptr;
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
        return dict_of({{"accept_len", &acc}, {"n_emitted", &ne}, {"emitted", &em}, {"accept_prob", &prob}});
    });
}

// one-byte codes or scales
const at::Tensor& bytes4(PyObject* o, int di, bool scales) {
    const at::Tensor& t = tensor(o);
    if (!t.is_cuda() || t.get_device() != di || t.dim() != 4 || t.stride(3) != 1) throw NotCommon();
    if (t.scalar_type() != at::kByte && !(scales && t.scalar_type() == at::kFloat8_e4m3fn)) throw NotCommon();
    return t;
}
// the six fields of a CacheQ4 from a[0] on; d < 0: as many channels as the codes say
pps_kv_cache_q4 cache_q4(PyObject* const* a, int di, int64_t d) {
    const at::Tensor &k = bytes4(a[0], di, false), &v = bytes4(a[1], di, false), &ks = bytes4(a[2], di, true), &vs = bytes4(a[3], di, true);
    if (d < 0) d = 2 * k.size(3);
    if (k.size(3) * 2 != d || k.sizes() != v.sizes() || k.strides() != v.strides() || ks.sizes() != vs.sizes() || ks.strides() != vs.strides())
        throw NotCommon();
    if (ks.size(0) != k.size(0) || ks.size(1) != k.size(1) || ks.size(2) != k.size(2) || ks.size(3) != (d + 63) / 64 * 4) throw NotCommon();
    if (k.size(1) > INT32_MAX || k.size(2) > INT32_MAX || d > INT32_MAX) throw NotCommon();
    return {k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), flat<float>(a[4], di, at::kFloat, k.size(2)),
            flat<float>(a[5], di, at::kFloat, k.size(2)), k.size(0), (int32_t)k.size(1), (int32_t)k.size(2), (int32_t)d,
            k.stride(0), k.stride(1), k.stride(2), ks.stride(0), ks.stride(1), ks.stride(2)};
}

// q, k, v, pos, slot, cache's six fields, rope, q_norm, k_norm, eps, interleaved, out, status
PyObject* kv_append_q4(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return common(args, n_args, 18, [](PyObject* const* a) -> PyObject* {
        const at::Tensor& q = tensor(a[0]);
        const int di = current_device_of(q);
        const at::ScalarType st = q.scalar_type();
        pps_append_q4_args x;
        std::memset(&x, 0, sizeof(x));
        x.size = sizeof(x);
        x.dtype = half_code(q);
        if (q.dim() != 3) throw NotCommon();
        const int64_t n = q.size(0), h = q.size(1), d = q.size(2);
        x.n_tok = n;
        x.n_heads = small(h);
        x.cache = cache_q4(a + 5, di, d);
        x.q = heads(q, n, h, d);
        x.k = heads(on(a[1], di, st), n, x.cache.n_kv_heads, d);
        x.v = heads(on(a[2], di, st), n, x.cache.n_kv_heads, d);
        if (a[11] != Py_None) {
            const at::Tensor& r = on(a[11], di, at::kFloat);
            if (r.dim() != 2 || !r.is_contiguous() || a[3] == Py_None) throw NotCommon();
            x.rope = static_cast<const float*>(r.data_ptr());
            x.max_pos = r.size(0);
            x.rot = small(r.size(1));
            x.pos = flat<int32_t>(a[3], di, at::kInt, n);
        }
        if (a[4] == Py_None) throw NotCommon();
        x.slot = flat<int64_t>(a[4], di, at::kLong, n);
        x.q_norm = flat<void>(a[12], di, st, d);
        x.k_norm = flat<void>(a[13], di, st, d);
        x.eps = (float)number(a[14]);
        x.interleaved = a[15] == Py_True ? 1 : a[15] == Py_False ? 0 : throw NotCommon();
        x.status = flat<uint32_t>(a[17], di, at::kInt, 1);
        at::Tensor made;
        if (a[16] == Py_None) {
            made = at::empty({n, h, d}, q.options());
            x.out_q = heads(made, n, h, d);
        } else
            x.out_q = heads(on(a[16], di, st), n, h, d);
        const pps_status code = api.append_q4(&x, (pps_stream_t)c10::cuda::getCurrentCUDAStream(di).stream());
        if (code != PPS_OK) return PyLong_FromLong(code);
        return made.defined() ? THPVariable_Wrap(made) : new_ref(a[16]);
    });
}

// cache's six fields, slot, whether bfloat16 (else float16), status (and outputs of its own)
PyObject* kv_read_q4(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return common(args, n_args, 9, [](PyObject* const* a) -> PyObject* {
        const at::Tensor& slot = tensor(a[6]);
        const int di = current_device_of(slot);
        pps_read_q4_args x;
        std::memset(&x, 0, sizeof(x));
        x.size = sizeof(x);
        x.cache = cache_q4(a, di, -1);
        x.n = slot.numel();
        x.slot = flat<int64_t>(a[6], di, at::kLong, x.n);
        x.status = flat<uint32_t>(a[8], di, at::kInt, 1);
        x.dtype = a[7] == Py_True ? PPS_BF16 : PPS_F16;
        const auto like = slot.options().dtype(a[7] == Py_True ? at::kBFloat16 : at::kHalf);
        const int64_t h = x.cache.n_kv_heads, d = x.cache.head_dim;
        at::Tensor k = at::empty({x.n, h, d}, like), v = at::empty({x.n, h, d}, like);
        x.k = heads(k, x.n, h, d);
        x.v = heads(v, x.n, h, d);
        const pps_status code = api.read_q4(&x, (pps_stream_t)c10::cuda::getCurrentCUDAStream(di).stream());
        if (code != PPS_OK) return PyLong_FromLong(code);
        PyObject *pk = THPVariable_Wrap(k), *pv = pk ? THPVariable_Wrap(v) : nullptr, *both = pv ? PyTuple_Pack(2, pk, pv) : nullptr;
        Py_XDECREF(pk);
        Py_XDECREF(pv);
        return both;
    });
}

// q, cache's six fields, pages, kv_len, q_off, mask, scale, out, lse, ws, status
PyObject* paged_attention_q4(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return common(args, n_args, 16, [](PyObject* const* a) -> PyObject* {
        const at::Tensor& q = tensor(a[0]);
        const int di = current_device_of(q);
        const at::ScalarType st = q.scalar_type();
        pps_attention_q4_args x;
        std::memset(&x, 0, sizeof(x));
        x.size = sizeof(x);
        x.dtype = half_code(q);
        if (q.dim() != 3) throw NotCommon();
        const int64_t n = q.size(0), h = q.size(1), d = q.size(2);
        x.n_tok = n;
        x.n_heads = small(h);
        x.cache = cache_q4(a + 1, di, d);
        x.q = heads(q, n, h, d);
        if (a[8] == Py_None || a[9] == Py_None) throw NotCommon();
        const int64_t n_seq = on(a[8], di, at::kInt).numel();
        x.kv_len = flat<int32_t>(a[8], di, at::kInt, 0);
        x.q_off = flat<int32_t>(a[9], di, at::kInt, n_seq + 1);
        x.n_seq = small(n_seq);
        const at::Tensor& pages = on(a[7], di, at::kInt);
        if (pages.dim() != 2 || pages.size(0) != n_seq || (pages.size(1) > 1 && pages.stride(1) != 1)) throw NotCommon();
        x.pages = static_cast<const int32_t*>(pages.data_ptr());
        x.max_pages = small(pages.size(1));
        x.pages_stride = n_seq > 1 ? pages.stride(0) : pages.size(1);
        if (a[10] != Py_None) {
            const at::Tensor& m = on(a[10], di, at::kInt);
            if (m.dim() != 2 || m.size(0) != n || m.size(1) < 1 || !m.is_contiguous()) throw NotCommon();
            x.mask = static_cast<const uint32_t*>(m.data_ptr());
            x.mask_words = small(m.size(1));
        }
        x.scale = a[11] == Py_None ? (float)(1.0 / std::sqrt((double)d)) : (float)number(a[11]);
        x.out_lse = flat<float>(a[13], di, at::kFloat, n * h);
        x.status = flat<uint32_t>(a[15], di, at::kInt, 1);
        at::Tensor made;
        if (a[12] == Py_None) {
            made = at::empty({n, h, d}, q.options());
            x.out = heads(made, n, h, d);
        } else
            x.out = heads(on(a[12], di, st), n, h, d);
        const cudaStream_t stream = c10::cuda::getCurrentCUDAStream(di).stream();
        pps_status code;
        if (a[14] != Py_None) {
            x.ws = flat<void>(a[14], di, at::kByte, 0);
            x.ws_bytes = (size_t)tensor(a[14]).numel();
            code = api.attention_q4(&x, (pps_stream_t)stream);
        } else {
            x.ws_bytes = api.attention_q4_ws(n, x.n_heads, x.cache.n_kv_heads, x.cache.head_dim);
            const Scratch ws(x.ws_bytes, stream);
            x.ws = ws.p;
            code = api.attention_q4(&x, (pps_stream_t)stream);
        }
        if (code != PPS_OK) return PyLong_FromLong(code);
        return made.defined() ? THPVariable_Wrap(made) : new_ref(a[12]);
    });
}

// pages, held, free_list, free_count into a reserve's or trim's arguments
template <typename A>
int pool(A& x, PyObject* const* a) {
    const at::Tensor& pages = tensor(a[0]);
    const int di = current_device_of(pages);
    std::memset(&x, 0, sizeof(x));
    x.size = sizeof(x);
    if (pages.scalar_type() != at::kInt || pages.dim() != 2 || (pages.size(1) > 1 && pages.stride(1) != 1)) throw NotCommon();
    x.pages = static_cast<int32_t*>(pages.data_ptr());
    x.n_seq = small(pages.size(0));
    x.columns = small(pages.size(1));
    x.pages_stride = pages.size(0) > 1 ? pages.stride(0) : pages.size(1);
    for (int i = 1; i < 4; ++i)
        if (a[i] == Py_None) throw NotCommon();
    x.held = flat<int32_t>(a[1], di, at::kInt, x.n_seq);
    x.free_list = flat<int32_t>(a[2], di, at::kInt, 0);
    x.free_cap = small(tensor(a[2]).numel());
    x.free_count = flat<int32_t>(a[3], di, at::kInt, 1);
    return di;
}

// pages, held, free_list, free_count, kv_len, n_new, page_size, n_tok, pos_off, status (and outputs of its own)
PyObject* kv_reserve(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return common(args, n_args, 10, [](PyObject* const* a) -> PyObject* {
        pps_reserve_args x;
        const int di = pool(x, a);
        if (a[4] == Py_None || a[5] == Py_None) throw NotCommon();
        x.kv_len = flat<int32_t>(a[4], di, at::kInt, x.n_seq);
        x.n_new = flat<int32_t>(a[5], di, at::kInt, x.n_seq);
        x.page_size = small(integer(a[6]));
        x.n_tok = integer(a[7]);
        if (x.n_tok < 0 || x.n_tok > INT32_MAX) throw NotCommon();
        x.pos_off = flat<int32_t>(a[8], di, at::kInt, x.n_tok);
        x.status = flat<uint32_t>(a[9], di, at::kInt, 1);
        const auto ints = tensor(a[0]).options();
        // the outputs share one allocation, each from a 16-byte boundary on: five take longer than the rest of the call
        const int64_t seqs = (x.n_seq + (int64_t)4) / 4 * 4, toks = (x.n_tok + 3) / 4 * 4;
        const at::Tensor all = at::empty({2 * toks + 2 * seqs + 2 * toks}, ints);
        at::Tensor slot = piece(all, at::kLong, 0, x.n_tok), off = piece(all, at::kInt, 2 * toks, x.n_seq + (int64_t)1),
                   len = piece(all, at::kInt, 2 * toks + seqs, x.n_seq), pos = piece(all, at::kInt, 2 * toks + 2 * seqs, x.n_tok),
                   seq = piece(all, at::kInt, 3 * toks + 2 * seqs, x.n_tok);
        x.out_q_off = static_cast<int32_t*>(off.data_ptr());
        x.out_kv_len = static_cast<int32_t*>(len.data_ptr());
        x.out_slot = static_cast<int64_t*>(slot.data_ptr());
        x.out_pos = static_cast<int32_t*>(pos.data_ptr());
        x.out_seq = static_cast<int32_t*>(seq.data_ptr());
        const pps_status code = api.reserve(&x, (pps_stream_t)c10::cuda::getCurrentCUDAStream(di).stream());
        if (code != PPS_OK) return PyLong_FromLong(code);
        return dict_of({{"q_off", &off}, {"kv_len", &len}, {"slot", &slot}, {"pos", &pos}, {"seq", &seq}});
    });
}

// pages, held, free_list, free_count, keep, page_size, status; True when done
PyObject* kv_trim(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return common(args, n_args, 7, [](PyObject* const* a) -> PyObject* {
        pps_trim_args x;
        const int di = pool(x, a);
        if (a[4] == Py_None) throw NotCommon();
        x.keep = flat<int32_t>(a[4], di, at::kInt, x.n_seq);
        x.page_size = small(integer(a[5]));
        x.status = flat<uint32_t>(a[6], di, at::kInt, 1);
        const pps_status code = api.trim(&x, (pps_stream_t)c10::cuda::getCurrentCUDAStream(di).stream());
        return code != PPS_OK ? PyLong_FromLong(code) : new_ref(Py_True);
    });
}

// logits, seq_off, text, text_len, prompt_len, node_tok, node_mask, repetition, frequency, presence, bias_off, bias_tok, bias_val,
// allowed, out, status
PyObject* adjust_logits(PyObject*, PyObject* const* args, Py_ssize_t n_args) {
    return common(args, n_args, 16, [](PyObject* const* a) -> PyObject* {
        const at::Tensor& l = tensor(a[0]);
        const int di = current_device_of(l);
        const at::ScalarType st = l.scalar_type();
        pps_adjust_args x;
        std::memset(&x, 0, sizeof(x));
        x.size = sizeof(x);
        x.dtype = st == at::kBFloat16 ? PPS_BF16 : st == at::kFloat ? PPS_F32 : throw NotCommon();
        if (l.dim() != 2 || l.stride(1) != 1 || a[1] == Py_None) throw NotCommon();
        const int64_t n = l.size(0), V = l.size(1), n_seq = on(a[1], di, at::kInt).numel() - 1;
        x.seq_off = flat<int32_t>(a[1], di, at::kInt, 1);
        x.n_seq = small(n_seq);
        x.logits = l.data_ptr();
        x.n_rows = n;
        x.vocab = V;
        x.in_stride = n > 1 ? l.stride(0) : V;
        if (a[2] != Py_None || a[3] != Py_None) {
            const at::Tensor& t = on(a[2], di, at::kInt);
            if (t.dim() != 2 || t.size(0) != n_seq || (t.size(1) > 1 && t.stride(1) != 1) || a[3] == Py_None) throw NotCommon();
            x.text = static_cast<const int32_t*>(t.data_ptr());
            x.text_cap = small(t.size(1));
            x.text_stride = n_seq > 1 ? t.stride(0) : t.size(1);
            x.text_len = flat<int32_t>(a[3], di, at::kInt, n_seq);
        }
        x.prompt_len = flat<int32_t>(a[4], di, at::kInt, n_seq);
        x.node_tok = flat<int32_t>(a[5], di, at::kInt, n);
        if (a[5] != Py_None && n == 0) x.node_tok = x.seq_off;  // (an empty tensor has no address: any other, of which nothing is read)
        if (a[6] != Py_None) {
            const at::Tensor& m = on(a[6], di, at::kInt);
            if (m.dim() != 2 || m.size(0) != n || m.size(1) < 1 || !m.is_contiguous()) throw NotCommon();
            x.node_mask = static_cast<const uint32_t*>(m.data_ptr());
            x.mask_words = small(m.size(1));
        }
        x.repetition = flat<float>(a[7], di, at::kFloat, n_seq);
        x.frequency = flat<float>(a[8], di, at::kFloat, n_seq);
        x.presence = flat<float>(a[9], di, at::kFloat, n_seq);
        if (a[10] != Py_None || a[11] != Py_None || a[12] != Py_None) {
            if (a[10] == Py_None || a[11] == Py_None || a[12] == Py_None) throw NotCommon();
            x.n_bias = small(tensor(a[11]).numel());
            x.bias_off = flat<int32_t>(a[10], di, at::kInt, n_seq + 1);
            x.bias_tok = flat<int32_t>(a[11], di, at::kInt, 0);
            x.bias_val = flat<float>(a[12], di, at::kFloat, x.n_bias);
        }
        if (a[13] != Py_None) {
            const at::Tensor& m = on(a[13], di, at::kInt);
            if (m.dim() != 2 || m.size(0) != n || m.size(1) < (V + 31) / 32 || (m.size(1) > 1 && m.stride(1) != 1)) throw NotCommon();
            x.allowed = static_cast<const uint32_t*>(m.data_ptr());
            x.allowed_stride = n > 1 ? m.stride(0) : m.size(1);
        }
        x.status = flat<uint32_t>(a[15], di, at::kInt, 1);
        at::Tensor made;
        const at::Tensor* out = &made;
        if (a[14] == Py_None)
            made = at::empty({n, V}, l.options());
        else
            out = &on(a[14], di, st);
        if (out->dim() != 2 || out->size(0) != n || out->size(1) != V || out->stride(1) != 1) throw NotCommon();
        x.out = out->data_ptr();
        x.out_stride = n > 1 ? out->stride(0) : V;
        const pps_status code = api.adjust(&x, (pps_stream_t)c10::cuda::getCurrentCUDAStream(di).stream());
        if (code != PPS_OK) return PyLong_FromLong(code);
        return made.defined() ? THPVariable_Wrap(made) : new_ref(a[14]);
    });
}

// the addresses of the calls, in the order of Api
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    constexpr int kCalls = 12;
    void* p[kCalls];
    if (n != kCalls) return PyErr_Format(PyExc_TypeError, "%d addresses are needed", kCalls);
    for (int i = 0; i < kCalls; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (p[i] == nullptr && PyErr_Occurred()) return nullptr;
    }
    int i = 0;
    auto take = [&](auto& f) { f = reinterpret_cast<std::remove_reference_t<decltype(f)>>(p[i++]); };
    Api x = {};
    take(x.append);
    take(x.attention);
    take(x.chain);
    take(x.attention_ws);
    take(x.chain_ws);
    take(x.append_q4);
    take(x.read_q4);
    take(x.attention_q4);
    take(x.attention_q4_ws);
    take(x.reserve);
    take(x.trim);
    take(x.adjust);
    api = x;
    return new_ref(Py_None);
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyCFunction fast() {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F));
}

PyMethodDef methods[] = {{"kv_append", fast<kv_append>(), METH_FASTCALL, nullptr},
                         {"paged_attention", fast<paged_attention>(), METH_FASTCALL, nullptr},
                         {"verify_chain", fast<verify_chain>(), METH_FASTCALL, nullptr},
                         {"kv_append_q4", fast<kv_append_q4>(), METH_FASTCALL, nullptr},
                         {"kv_read_q4", fast<kv_read_q4>(), METH_FASTCALL, nullptr},
                         {"paged_attention_q4", fast<paged_attention_q4>(), METH_FASTCALL, nullptr},
                         {"kv_reserve", fast<kv_reserve>(), METH_FASTCALL, nullptr},
                         {"kv_trim", fast<kv_trim>(), METH_FASTCALL, nullptr},
                         {"adjust_logits", fast<adjust_logits>(), METH_FASTCALL, nullptr},
                         {"bind", fast<bind>(), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "pps_torch", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_pps_torch() { return PyModule_Create(&module); }
