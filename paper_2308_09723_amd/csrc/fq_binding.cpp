// The calls of the torch-tensor layer that a program makes over and over (products, activation and weight quantiser), in
// native code: argument checks, output allocation, the current stream and the call of the library.
//
// A product of one kernel takes the GPU 4 - 8 us, and issuing it from Python took as long: 6.5 us, of which the launch itself
// is 2.7; here it takes 3.5.  The integer path's two calls: 14.7 us from Python, now 9.7 (which the GPU takes); fq.quantize 9.2
// -> 5.6.
//
// Every function returns None, having launched nothing, where anything is out of the ordinary: objects that are not plain
// CUDA tensors, torch function modes, other types than the listed ones, arguments or a workspace that the library refuses.  fq.py
// then takes its own way, which reports the error or does what it always did.  An error of the runtime (FQ_ERR_HIP) may follow
// launches that were enqueued, so it is raised here and the call is not made again.  Only arguments are looked at; nothing is
// kept between calls.
#include <Python.h>

#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/generated/variable_factories.h>
#include <torch/csrc/autograd/python_variable.h>

#include <limits.h>
#include <string.h>


#include "../../include/fq.h"

namespace {

// the library's functions, as addresses that fq.py hands over (bind): one copy of the library per process
struct {
    decltype(&fq_gemm_sf) gemm_sf;
    decltype(&fq_gemm_workspace_bytes) gemm_workspace_bytes;
    decltype(&fq_gemm_grouped_sf) gemm_grouped_sf;
    decltype(&fq_gemm_w4a8) gemm_w4a8;
    decltype(&fq_gemm_w4a8_workspace_bytes) gemm_w4a8_workspace_bytes;
    decltype(&fq_quantize_act_i8) quantize_act_i8;
    decltype(&fq_quantize_sf) quantize_sf;
    decltype(&fq_quantize_w4a8) quantize_w4a8;
    decltype(&fq_codes_bytes) codes_bytes;
    decltype(&fq_scales_bytes) scales_bytes;
    decltype(&fq_zscale_bytes) zscale_bytes;
    decltype(&fq_qk_norm_rope) qk_norm_rope;
    decltype(&fq_attention_prompt) attention_prompt;
    decltype(&fq_attention_prompt_workspace_bytes) attention_prompt_workspace_bytes;
    decltype(&fq_attention_tree) attention_tree;
    decltype(&fq_attention_tree_workspace_bytes) attention_tree_workspace_bytes;
    decltype(&fq_kv4_page_bytes) kv4_page_bytes;
    decltype(&fq_kv4_write) kv4_write;
    decltype(&fq_kv4_read) kv4_read;
    decltype(&fq_attention_tree_kv4) attention_tree_kv4;
    decltype(&fq_attention_tree_kv4_workspace_bytes) attention_tree_kv4_workspace_bytes;
    decltype(&fq_pages_take) pages_take;
    decltype(&fq_pages_fork) pages_fork;
    decltype(&fq_pages_fork_workspace_bytes) pages_fork_workspace_bytes;
    decltype(&fq_pages_free) pages_free;
    decltype(&fq_pages_compact) pages_compact;
    decltype(&fq_pages_compact_workspace_bytes) pages_compact_workspace_bytes;
    decltype(&fq_adapters) adapters;
    decltype(&fq_adapters_workspace_bytes) adapters_workspace_bytes;
} lib;

PyObject* fq_error;       // fq.FqError

struct not_plain {};      // thrown: the Python way
struct runtime_error {    // thrown: FqError(FQ_ERR_HIP, where)
    const char* where;
};

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o)) throw not_plain();
    const at::Tensor& t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.layout() != at::kStrided) throw not_plain();
    return t;
}

int integer(PyObject* o) {
    if (!PyLong_CheckExact(o)) throw not_plain();
    int overflow = 0;
    const long v = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow != 0 || v < INT_MIN || v > INT_MAX) throw not_plain();
    return (int)v;
}

// 0 for binary16, 1 for bfloat16: the library's activation types and its scale formats alike
int type16(at::ScalarType s) {
    if (s == at::kHalf) return 0;
    if (s == at::kBFloat16) return 1;
    throw not_plain();
}

int scalar16(PyObject* o) {
    if (!THPDtype_Check(o)) throw not_plain();
    return type16(reinterpret_cast<THPDtype*>(o)->scalar_type);
}

at::Tensor empty(at::IntArrayRef size, at::ScalarType type, const at::Tensor& like) {
    return torch::empty(size, at::TensorOptions().dtype(type).device(like.device()));
}

void* stream() { return (void*)c10::hip::getCurrentHIPStream(c10::hip::current_device()).stream(); }

void arguments(Py_ssize_t got, Py_ssize_t want) {
    if (got != want || at::impl::torch_function_mode_enabled()) throw not_plain();
}

// runs `f` (a call of the library's function `where`) without the interpreter's lock
template <typename F>
void call(const char* where, F f) {
    int status;
    Py_BEGIN_ALLOW_THREADS
    status = f();
    Py_END_ALLOW_THREADS
    if (status == FQ_ERR_HIP) throw runtime_error{where};
    if (status != FQ_OK) throw not_plain();
}

// a caller's workspace (None: one of `need()` bytes) as address and size
template <typename F>
void* scratch(PyObject* o, const at::Tensor& like, F need, size_t* size, at::Tensor* own) {
    if (o != Py_None) {
        const at::Tensor& t = tensor(o);
        *size = (size_t)t.numel() * t.element_size();
        return t.data_ptr();
    }
    *size = need();
    if (*size == 0) return nullptr;
    *own = empty({(int64_t)*size}, at::kByte, like);
    return own->data_ptr();
}

// the output a caller gave, or a new one
PyObject* result(PyObject* given, at::Tensor&& made) {
    if (given == Py_None) return THPVariable_Wrap(std::move(made));
    Py_INCREF(given);
    return given;
}

template <typename F>
PyObject* guarded(F f) {
    try {
        return f();
    } catch (const runtime_error& e) {
        PyObject* raised = PyObject_CallFunction(fq_error, "is", (int)FQ_ERR_HIP, e.where);
        if (raised) PyErr_SetObject(fq_error, raised);
        Py_XDECREF(raised);
        return nullptr;
    } catch (...) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// gemm(A, codes, scales, bits, group_size, out, workspace)
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 7);
        const at::Tensor &A = tensor(a[0]), &codes = tensor(a[1]), &scales = tensor(a[2]);
        if (A.dim() != 2 || scales.dim() != 2 || !A.is_contiguous()) throw not_plain();
        const int act = type16(A.scalar_type()), format = type16(scales.scalar_type()), bits = integer(a[3]), g = integer(a[4]);
        const int64_t M = A.size(0), K = A.size(1), N = scales.size(1);
        const void *Ap = A.data_ptr(), *cp = codes.data_ptr(), *sp = scales.data_ptr();
        at::Tensor C = a[5] != Py_None ? tensor(a[5]) : empty({M, N}, A.scalar_type(), A), own;
        size_t size = 0;
        void* ws = scratch(a[6], A, [&] { return lib.gemm_workspace_bytes(M, N, K, bits, g); }, &size, &own);
        void *Cp = C.data_ptr(), *s = stream();
        call("fq_gemm_sf", [&] { return lib.gemm_sf(Ap, act, M, N, K, cp, sp, format, bits, g, Cp, ws, size, s); });
        return result(a[5], std::move(C));
    });
}

// gemm_grouped(A, offsets, codes, scales, bits, group_size, N, out)
PyObject* gemm_grouped(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 8);
        const at::Tensor &A = tensor(a[0]), &codes = tensor(a[2]), &scales = tensor(a[3]);
        if (A.dim() != 2 || !(PyList_CheckExact(a[1]) || PyTuple_CheckExact(a[1]))) throw not_plain();
        const Py_ssize_t count = PySequence_Fast_GET_SIZE(a[1]);
        if (count < 1 || count > 257) throw not_plain();
        int32_t offsets[257];
        for (Py_ssize_t i = 0; i < count; ++i) offsets[i] = integer(PySequence_Fast_GET_ITEM(a[1], i));
        const int act = type16(A.scalar_type()), format = type16(scales.scalar_type()), bits = integer(a[4]), g = integer(a[5]);
        const int64_t K = A.size(1), N = integer(a[6]);
        const void *Ap = A.data_ptr(), *cp = codes.data_ptr(), *sp = scales.data_ptr();
        at::Tensor C = a[7] != Py_None ? tensor(a[7]) : empty({A.size(0), N}, A.scalar_type(), A);
        void *Cp = C.data_ptr(), *s = stream();
        call("fq_gemm_grouped_sf", [&] {
            return lib.gemm_grouped_sf(Ap, act, offsets, (int)count - 1, N, K, cp, sp, format, bits, g, Cp, nullptr, 0, s);
        });
        return result(a[7], std::move(C));
    });
}

// quantize_act_i8(A)
PyObject* quantize_act_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 1);
        const at::Tensor& A = tensor(a[0]);
        if (A.dim() != 2 || !A.is_contiguous()) throw not_plain();
        const int act = type16(A.scalar_type());
        const int64_t M = A.size(0), K = A.size(1);
        const void* Ap = A.data_ptr();
        at::Tensor Aq = empty({M, K}, at::kChar, A), alpha = empty({M}, at::kFloat, A);
        int8_t* qp = (int8_t*)Aq.data_ptr();
        float* alp = (float*)alpha.data_ptr();
        void* s = stream();
        call("fq_quantize_act_i8", [&] { return lib.quantize_act_i8(Ap, act, M, K, qp, alp, s); });
        return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(Aq)), THPVariable_Wrap(std::move(alpha)));
    });
}

// gemm_w4a8(Aq, alpha, codes, z, t, group_size, out_dtype, out, workspace)
PyObject* gemm_w4a8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 9);
        const at::Tensor &Aq = tensor(a[0]), &alpha = tensor(a[1]), &codes = tensor(a[2]), &z = tensor(a[3]), &t = tensor(a[4]);
        if (Aq.dim() != 2 || t.dim() != 1) throw not_plain();
        const int g = integer(a[5]), type = scalar16(a[6]);
        const int64_t M = Aq.size(0), K = Aq.size(1), N = t.size(0);
        const int8_t* qp = (const int8_t*)Aq.data_ptr();
        const float* alp = (const float*)alpha.data_ptr();
        const void *cp = codes.data_ptr(), *tp = t.data_ptr();
        const uint8_t* zp = (const uint8_t*)z.data_ptr();
        at::Tensor C = a[7] != Py_None ? tensor(a[7]) : empty({M, N}, type == 0 ? at::kHalf : at::kBFloat16, Aq), own;
        size_t size = 0;
        void* ws = scratch(a[8], Aq, [&] { return lib.gemm_w4a8_workspace_bytes(M, N, K, g); }, &size, &own);
        void *Cp = C.data_ptr(), *s = stream();
        call("fq_gemm_w4a8", [&] { return lib.gemm_w4a8(qp, alp, M, N, K, cp, zp, tp, g, Cp, type, ws, size, s); });
        return result(a[7], std::move(C));
    });
}

// quantize(W, bits, group_size, scale_format)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 4);
        const at::Tensor& W = tensor(a[0]);
        if (W.dim() != 2 || W.scalar_type() != at::kHalf || !W.is_contiguous()) throw not_plain();
        const int bits = integer(a[1]), g = integer(a[2]), format = integer(a[3]);
        const int64_t K = W.size(0), N = W.size(1);
        const size_t cb = lib.codes_bytes(K, N, bits), sb = lib.scales_bytes(K, N, g);
        if (cb == 0 || sb == 0 || (format != FQ_SCALE_F16 && format != FQ_SCALE_BF16)) throw not_plain();
        const void* Wp = W.data_ptr();
        at::Tensor codes = empty({(int64_t)cb}, at::kByte, W);
        at::Tensor scales = empty({g == 0 ? 1 : K / g, N}, format == FQ_SCALE_BF16 ? at::kBFloat16 : at::kHalf, W);
        void *cp = codes.data_ptr(), *sp = scales.data_ptr(), *s = stream();
        call("fq_quantize_sf", [&] { return lib.quantize_sf(Wp, K, N, bits, g, format, cp, sp, s); });
        return Py_BuildValue("(NN)", THPVariable_Wrap(std::move(codes)), THPVariable_Wrap(std::move(scales)));
    });
}

// quantize_w4a8(W, group_size)
PyObject* quantize_w4a8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 2);
        const at::Tensor& W = tensor(a[0]);
        if (W.dim() != 2 || W.scalar_type() != at::kHalf || !W.is_contiguous()) throw not_plain();
        const int g = integer(a[1]);
        const int64_t K = W.size(0), N = W.size(1);
        if (lib.zscale_bytes(K, N, g) == 0) throw not_plain();
        const void* Wp = W.data_ptr();
        at::Tensor codes = empty({(int64_t)lib.codes_bytes(K, N, 4)}, at::kByte, W), z = empty({g == 0 ? 1 : K / g, N}, at::kByte, W),
                   t = empty({N}, at::kHalf, W);
        void *cp = codes.data_ptr(), *tp = t.data_ptr(), *s = stream();
        uint8_t* zp = (uint8_t*)z.data_ptr();
        call("fq_quantize_w4a8", [&] { return lib.quantize_w4a8(Wp, K, N, g, cp, zp, tp, s); });
        return Py_BuildValue("(NNN)", THPVariable_Wrap(std::move(codes)), THPVariable_Wrap(std::move(z)), THPVariable_Wrap(std::move(t)));
    });
}

// ------------------------------------------------------------------------------------------ attention
void require(bool condition) {
    if (!condition) throw not_plain();
}

double number(PyObject* o) {
    if (PyFloat_CheckExact(o)) return PyFloat_AS_DOUBLE(o);
    return integer(o);
}

bool truth(PyObject* o) {
    require(PyBool_Check(o));
    return o == Py_True;
}

// a contiguous tensor of this type beside `like`
const at::Tensor& plain(PyObject* o, at::ScalarType type, const at::Tensor& like) {
    const at::Tensor& t = tensor(o);
    require(t.scalar_type() == type && t.device() == like.device() && t.is_contiguous());
    return t;
}

at::Tensor output(PyObject* o, at::IntArrayRef size, const at::Tensor& like) {
    if (o == Py_None) return empty(size, like.scalar_type(), like);
    const at::Tensor& t = plain(o, like.scalar_type(), like);
    require(t.sizes() == size);
    return t;
}

fq_kv_pages pages(PyObject* ko, PyObject* vo, const at::Tensor& like, int64_t kv_heads, int64_t head_dim) {
    const at::Tensor &k = tensor(ko), &v = tensor(vo);
    for (const at::Tensor* t : {&k, &v})
        require(t->dim() == 4 && t->scalar_type() == like.scalar_type() && t->device() == like.device() && t->stride(3) == 1 &&
                t->size(2) == kv_heads && t->size(3) == head_dim);
    require(k.sizes() == v.sizes() && k.strides() == v.strides() && k.size(1) <= INT_MAX);
    return {k.data_ptr(), v.data_ptr(), k.size(0), (int)k.size(1), k.stride(0), k.stride(1), k.stride(2)};
}

fq_heads heads(const at::Tensor& t) {
    require(t.dim() == 3 && t.stride(2) == 1 && t.size(1) <= INT_MAX && t.size(2) <= INT_MAX);
    return {t.data_ptr(), t.stride(0), t.stride(1)};
}

// qk_norm_rope(qkv, heads, kv_heads, table, positions, q_weight, k_weight, eps, interleaved, q_out, k_out, k_cache, v_cache, slots)
PyObject* qk_norm_rope(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 14);
        const at::Tensor& qkv = tensor(a[0]);
        const int hq = integer(a[1]), hk = integer(a[2]), act = type16(qkv.scalar_type());
        require(qkv.dim() == 2 && hq > 0 && hk > 0 && qkv.stride(1) == 1 && qkv.size(1) % ((int64_t)hq + 2 * (int64_t)hk) == 0);
        const int64_t tokens = qkv.size(0), D = qkv.size(1) / ((int64_t)hq + 2 * (int64_t)hk);
        require(tokens > 0 && D <= INT_MAX);
        const void* weight[2] = {};
        for (int i = 0; i < 2; ++i)
            if (a[5 + i] != Py_None) {
                const at::Tensor& w = plain(a[5 + i], qkv.scalar_type(), qkv);
                require(w.numel() == D);
                weight[i] = w.data_ptr();
            }
        const float* table = nullptr;
        const int32_t* positions = nullptr;
        int64_t rows = 0, rot = 0;
        if (a[3] != Py_None) {
            const at::Tensor &t = plain(a[3], at::kFloat, qkv), &p = plain(a[4], at::kInt, qkv);
            require(t.dim() == 2 && p.numel() == tokens && t.size(1) > 0 && t.size(1) <= INT_MAX);
            table = (const float*)t.data_ptr();
            positions = (const int32_t*)p.data_ptr();
            rows = t.size(0);
            rot = t.size(1);
        }
        fq_kv_pages cache = {};
        const int64_t* slots = nullptr;
        const bool cached = a[11] != Py_None;
        require(cached == (a[12] != Py_None) && cached == (a[13] != Py_None));
        if (cached) {
            cache = pages(a[11], a[12], qkv, hk, D);
            const at::Tensor& s = plain(a[13], at::kLong, qkv);
            require(s.numel() == tokens);
            slots = (const int64_t*)s.data_ptr();
        }
        const float eps = (float)number(a[7]);
        const int interleaved = truth(a[8]);
        at::Tensor q = output(a[9], {tokens, hq, D}, qkv), k;
        const bool keys = !cached || a[10] != Py_None;
        if (keys) k = output(a[10], {tokens, hk, D}, qkv);
        const void* from = qkv.data_ptr();
        const int64_t stride = qkv.stride(0);
        void *qp = q.data_ptr(), *kp = keys ? k.data_ptr() : nullptr, *s = stream();
        call("fq_qk_norm_rope", [&] {
            return lib.qk_norm_rope(from, act, tokens, stride, hq, hk, (int)D, weight[0], weight[1], eps, table, rows, (int)rot, interleaved, positions, qp,
                                    kp, cached ? &cache : nullptr, slots, s);
        });
        PyObject* first = result(a[9], std::move(q));
        if (keys) return Py_BuildValue("(NN)", first, result(a[10], std::move(k)));
        return Py_BuildValue("(NO)", first, Py_None);
    });
}

// host offsets of up to 1024 sequences, as int32
struct offsets32 {
    int32_t at[1025];
    int count = 0;
    explicit offsets32(PyObject* o) {
        require(PyList_CheckExact(o) || PyTuple_CheckExact(o));
        const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
        require(n >= 1 && n <= 1025);
        for (Py_ssize_t i = 0; i < n; ++i) at[i] = integer(PySequence_Fast_GET_ITEM(o, i));
        count = (int)n;
    }
};

// a scale that was given; 0 for the library's own
float given_scale(PyObject* o) {
    if (o == Py_None) return 0.0f;
    const float x = (float)number(o);
    require(x > 0.0f);
    return x;
}

// a caller's workspace beside `like` where it is large enough, or a new one of `need` bytes
void* scratch_of(PyObject* o, const at::Tensor& like, size_t need, size_t* size, at::Tensor* own) {
    if (o != Py_None) {
        const at::Tensor& t = tensor(o);
        require(t.device() == like.device() && t.is_contiguous());
        *size = (size_t)t.numel() * t.element_size();
        if (*size >= need) return t.data_ptr();
    }
    *size = need;
    if (need == 0) return nullptr;
    *own = empty({(int64_t)need}, at::kByte, like);
    return own->data_ptr();
}

// attention_prompt(q, k, v, q_offsets, k_offsets, scale, out, workspace)
PyObject* attention_prompt(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 8);
        const at::Tensor &q = tensor(a[0]), &k = tensor(a[1]), &v = tensor(a[2]);
        const int act = type16(q.scalar_type());
        const fq_heads qh = heads(q), kh = heads(k), vh = heads(v);
        for (const at::Tensor* t : {&k, &v})
            require(t->sizes() == k.sizes() && t->size(2) == q.size(2) && t->scalar_type() == q.scalar_type() && t->device() == q.device());
        const int hq = (int)q.size(1), hk = (int)k.size(1), D = (int)q.size(2);
        const offsets32 qo(a[3]);
        const bool own_keys = a[4] != Py_None;
        const offsets32 ko(own_keys ? a[4] : a[3]);
        require(ko.count == qo.count && qo.at[qo.count - 1] == q.size(0) && ko.at[ko.count - 1] == k.size(0));
        const int32_t* kp = own_keys ? ko.at : nullptr;
        const float scale = given_scale(a[5]);
        at::Tensor out = output(a[6], q.sizes(), q), own;
        size_t size = 0;
        void* ws = scratch_of(a[7], q, lib.attention_prompt_workspace_bytes(hq, hk, D, qo.at, kp, qo.count - 1), &size, &own);
        void *op = out.data_ptr(), *s = stream();
        call("fq_attention_prompt",
             [&] { return lib.attention_prompt(&qh, &kh, &vh, act, hq, hk, D, qo.at, kp, qo.count - 1, scale, op, ws, size, s); });
        return result(a[6], std::move(out));
    });
}

// the row stride of drafted tokens' queries [sequences, nodes, heads, head_dim] (of one token, or one sequence, the tensor's says nothing)
int64_t drafted_rows(const at::Tensor& q) {
    require(q.dim() == 4 && q.stride(3) == 1);
    const int64_t B = q.size(0), nodes = q.size(1), row = B * nodes <= 1 ? 0 : nodes == 1 ? q.stride(0) : q.stride(1);
    require((q.stride(0) == nodes * row || B <= 1) && q.size(2) <= INT_MAX && q.size(3) <= INT_MAX);
    return row;
}

// page table, lengths and masks of them
struct tree_inputs {
    const int32_t *table, *lens;
    int64_t width, stride = 0;
    const uint64_t* mask = nullptr;
    tree_inputs(PyObject* to, PyObject* lo, PyObject* mo, const at::Tensor& q) {
        const at::Tensor &t = plain(to, at::kInt, q), &l = plain(lo, at::kInt, q);
        const int64_t B = q.size(0), nodes = q.size(1), words = (nodes + 63) / 64;
        require(t.dim() == 2 && t.size(0) == B && l.numel() == B);
        table = (const int32_t*)t.data_ptr();
        lens = (const int32_t*)l.data_ptr();
        width = t.size(1);
        if (mo == Py_None) return;
        const at::Tensor& m = plain(mo, at::kLong, q);
        const bool shared = m.dim() == 2;
        require(shared ? m.size(0) == nodes && m.size(1) == words : m.dim() == 3 && m.size(0) == B && m.size(1) == nodes && m.size(2) == words);
        mask = (const uint64_t*)m.data_ptr();
        stride = shared ? 0 : nodes * words;
    }
};

// attention_tree(q, k_cache, v_cache, page_table, context_lens, mask, scale, out, workspace)
PyObject* attention_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 9);
        const at::Tensor& q = tensor(a[0]);
        const int act = type16(q.scalar_type());
        const int64_t row = drafted_rows(q), B = q.size(0), nodes = q.size(1), hq = q.size(2), D = q.size(3);
        const at::Tensor& kc = tensor(a[1]);
        const int64_t hk = kc.dim() == 4 ? kc.size(2) : 0;
        require(hk <= INT_MAX);
        const fq_kv_pages cache = pages(a[1], a[2], q, hk, D);
        const tree_inputs in(a[3], a[4], a[5], q);
        const float scale = given_scale(a[6]);
        at::Tensor out = output(a[7], q.sizes(), q), own;
        size_t size = 0;
        void* ws = scratch_of(a[8], q, lib.attention_tree_workspace_bytes(B, nodes, (int)hq, (int)hk, (int)D, in.width, cache.page_size), &size, &own);
        const fq_heads qh = {q.data_ptr(), row, q.stride(2)};
        void *op = out.data_ptr(), *s = stream();
        call("fq_attention_tree", [&] {
            return lib.attention_tree(&qh, act, B, nodes, (int)hq, (int)hk, (int)D, &cache, in.table, in.width, in.lens, in.mask, in.stride, scale, op, ws, size, s);
        });
        return result(a[7], std::move(out));
    });
}

// Whether a call's tensors lie on the device whose stream it goes to
void here(const at::Tensor& t) { require(t.device().index() == c10::hip::current_device()); }

// ------------------------------------------------------------------------------------------ a cache held in 4 bits
fq_kv4_pages kv4_pages(PyObject* o, int page_size, int64_t kv_heads, int64_t head_dim, const at::Device& device) {
    const at::Tensor& t = tensor(o);
    require(t.dim() == 2 && t.scalar_type() == at::kByte && t.device() == device && t.stride(1) == 1 && kv_heads <= INT_MAX && head_dim <= INT_MAX);
    const size_t bytes = lib.kv4_page_bytes(page_size, (int)kv_heads, (int)head_dim);
    require(bytes > 0 && t.size(1) == (int64_t)bytes);
    return {t.data_ptr(), t.size(0), page_size, t.stride(0)};
}

// kv4_write(k, v, cache, page_size, slots)
PyObject* kv4_write(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 5);
        const at::Tensor &k = tensor(a[0]), &v = tensor(a[1]);
        const int act = type16(k.scalar_type());
        const fq_heads kh = heads(k), vh = heads(v);
        require(v.sizes() == k.sizes() && v.scalar_type() == k.scalar_type() && v.device() == k.device() && k.size(0) > 0);
        here(k);
        const fq_kv4_pages cache = kv4_pages(a[2], integer(a[3]), k.size(1), k.size(2), k.device());
        const at::Tensor& slots = plain(a[4], at::kLong, k);
        require(slots.numel() == k.size(0));
        const int64_t* at = (const int64_t*)slots.data_ptr();
        const int64_t tokens = k.size(0);
        const int hk = (int)k.size(1), D = (int)k.size(2);
        void* s = stream();
        call("fq_kv4_write", [&] { return lib.kv4_write(&kh, &vh, act, tokens, hk, D, &cache, at, s); });
        Py_RETURN_TRUE;
    });
}

// kv4_read(cache, page_size, kv_heads, head_dim, slots, dtype, k_out, v_out)
PyObject* kv4_read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 8);
        const at::Tensor& slots = tensor(a[4]);
        here(slots);
        const int hk = integer(a[2]), D = integer(a[3]), act = scalar16(a[5]);
        const fq_kv4_pages cache = kv4_pages(a[0], integer(a[1]), hk, D, slots.device());
        require(slots.scalar_type() == at::kLong && slots.is_contiguous() && slots.numel() > 0);
        const at::ScalarType type = act == 0 ? at::kHalf : at::kBFloat16;
        const int64_t tokens = slots.numel();
        at::Tensor out[2];
        void* p[2];
        for (int i = 0; i < 2; ++i) {
            out[i] = a[6 + i] != Py_None ? plain(a[6 + i], type, slots) : empty({tokens, hk, D}, type, slots);
            require(out[i].dim() == 3 && out[i].size(0) == tokens && out[i].size(1) == hk && out[i].size(2) == D);
            p[i] = out[i].data_ptr();
        }
        const int64_t* at = (const int64_t*)slots.data_ptr();
        void* s = stream();
        call("fq_kv4_read", [&] { return lib.kv4_read(&cache, act, tokens, hk, D, at, p[0], p[1], s); });
        PyObject* first = result(a[6], std::move(out[0]));
        return Py_BuildValue("(NN)", first, result(a[7], std::move(out[1])));
    });
}

// attention_tree_kv4(q, cache, page_size, kv_heads, page_table, context_lens, mask, scale, out, workspace)
PyObject* attention_tree_kv4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 10);
        const at::Tensor& q = tensor(a[0]);
        here(q);
        const int act = type16(q.scalar_type()), hk = integer(a[3]);
        const int64_t row = drafted_rows(q), B = q.size(0), nodes = q.size(1), hq = q.size(2), D = q.size(3);
        const fq_kv4_pages cache = kv4_pages(a[1], integer(a[2]), hk, D, q.device());
        const tree_inputs in(a[4], a[5], a[6], q);
        const float scale = given_scale(a[7]);
        at::Tensor out = output(a[8], q.sizes(), q), own;
        size_t size = 0;
        void* ws = scratch_of(a[9], q, lib.attention_tree_kv4_workspace_bytes(B, nodes, (int)hq, hk, (int)D, in.width, cache.page_size), &size, &own);
        const fq_heads qh = {q.data_ptr(), row, q.stride(2)};
        void *op = out.data_ptr(), *s = stream();
        call("fq_attention_tree_kv4", [&] {
            return lib.attention_tree_kv4(&qh, act, B, nodes, (int)hq, hk, (int)D, &cache, in.table, in.width, in.lens, in.mask, in.stride, scale, op, ws, size, s);
        });
        return result(a[8], std::move(out));
    });
}

// ------------------------------------------------------------------------------------------ pages that sequences share
// refs, table and lengths of a pool
struct pool {
    int32_t *refs, *table, *lens;
    int64_t pages, rows, width;
    at::Tensor like;
    pool(PyObject* ro, PyObject* to, PyObject* lo) {
        const at::Tensor& r = tensor(ro);
        here(r);
        const at::Tensor &t = plain(to, at::kInt, r), &l = plain(lo, at::kInt, r);
        require(r.scalar_type() == at::kInt && r.is_contiguous() && r.dim() == 1 && t.dim() == 2 && l.numel() == t.size(0));
        refs = (int32_t*)r.data_ptr();
        table = (int32_t*)t.data_ptr();
        lens = (int32_t*)l.data_ptr();
        pages = r.size(0);
        rows = t.size(0);
        width = t.size(1);
        like = r;
    }
};

// one tensor [tensors, pages, ...], or a list or tuple of up to 256 tensors [pages, ...]
struct page_buffers {
    fq_page_buffer at[256];
    int count = 0;
    void add(const at::Tensor& t, int dims, const pool& p) {
        require(t.dim() > dims && t.size(dims - 1) == p.pages && t.device() == p.like.device());
        const int64_t size = t.element_size();
        int64_t expected = 1;
        for (int64_t d = t.dim() - 1; d >= dims; --d) {
            require(t.size(d) == 1 || t.stride(d) == expected);
            expected *= t.size(d);
        }
        at[count++] = {t.data_ptr(), dims == 2 ? t.size(0) : 1, dims == 2 ? t.stride(0) * size : 0, t.stride(dims - 1) * size, expected * size};
    }
    page_buffers(PyObject* o, const pool& p) {
        if (PyList_CheckExact(o) || PyTuple_CheckExact(o)) {
            const Py_ssize_t n = PySequence_Fast_GET_SIZE(o);
            require(n <= 256);
            for (Py_ssize_t i = 0; i < n; ++i) add(tensor(PySequence_Fast_GET_ITEM(o, i)), 1, p);
        } else {
            add(tensor(o), 2, p);
        }
    }
};

// pages_take(refs, page_size, page_table, lens, wanted)
PyObject* pages_take(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 5);
        const pool p(a[0], a[2], a[3]);
        const int page = integer(a[1]);
        const at::Tensor& wanted = plain(a[4], at::kInt, p.like);
        require(wanted.numel() == p.rows);
        const int32_t* w = (const int32_t*)wanted.data_ptr();
        void* s = stream();
        call("fq_pages_take", [&] { return lib.pages_take(p.refs, p.pages, page, p.table, p.rows, p.width, p.lens, w, s); });
        Py_RETURN_TRUE;
    });
}

// pages_fork(refs, page_size, page_table, lens, parents, buffers, release, table_out, lens_out, workspace)
PyObject* pages_fork(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 10);
        const pool p(a[0], a[2], a[3]);
        const int page = integer(a[1]), release = truth(a[6]);
        const at::Tensor& parents = plain(a[4], at::kInt, p.like);
        const page_buffers buffers(a[5], p);
        const int64_t children = parents.numel();
        at::Tensor table = output(a[7], {children, p.width}, p.like), lens = output(a[8], {children}, p.like), own;
        size_t size = 0;
        void* ws = scratch_of(a[9], p.like, lib.pages_fork_workspace_bytes(p.rows, children), &size, &own);
        const int32_t* from = (const int32_t*)parents.data_ptr();
        int32_t *t = (int32_t*)table.data_ptr(), *l = (int32_t*)lens.data_ptr();
        void* s = stream();
        call("fq_pages_fork", [&] {
            return lib.pages_fork(p.refs, p.pages, page, p.table, p.rows, p.width, p.lens, from, children, release, t, l, buffers.at, buffers.count, ws, size, s);
        });
        PyObject* first = result(a[7], std::move(table));
        return Py_BuildValue("(NN)", first, result(a[8], std::move(lens)));
    });
}

// pages_free(refs, page_size, page_table, lens, rows)
PyObject* pages_free(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 5);
        const pool p(a[0], a[2], a[3]);
        const int page = integer(a[1]);
        const int32_t* which = nullptr;
        int64_t count = 0;
        if (a[4] != Py_None) {
            const at::Tensor& w = plain(a[4], at::kInt, p.like);
            count = w.numel();
            require(count > 0);
            which = (const int32_t*)w.data_ptr();
        }
        void* s = stream();
        call("fq_pages_free", [&] { return lib.pages_free(p.refs, p.pages, page, p.table, p.rows, p.width, p.lens, which, count, s); });
        Py_RETURN_TRUE;
    });
}

// pages_compact(refs, page_size, page_table, lens, buffers, workspace)
PyObject* pages_compact(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 6);
        const pool p(a[0], a[2], a[3]);
        const int page = integer(a[1]);
        const page_buffers buffers(a[4], p);
        at::Tensor own;
        size_t size = 0;
        void* ws = scratch_of(a[5], p.like, lib.pages_compact_workspace_bytes(p.pages), &size, &own);
        void* s = stream();
        call("fq_pages_compact",
             [&] { return lib.pages_compact(p.refs, p.pages, page, p.table, p.rows, p.width, p.lens, buffers.at, buffers.count, ws, size, s); });
        Py_RETURN_TRUE;
    });
}

// ------------------------------------------------------------------------------------------ low-rank adapters
// adapters(x, a, b, ids, out, scales, workspace)
PyObject* adapters(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded([&]() -> PyObject* {
        arguments(n, 7);
        const at::Tensor &x = tensor(a[0]), &out = tensor(a[4]);
        here(x);
        const int act = type16(x.scalar_type());
        const at::Tensor &A = plain(a[1], x.scalar_type(), x), &B = plain(a[2], x.scalar_type(), x), &ids = plain(a[3], at::kInt, x);
        require(x.dim() == 2 && out.dim() == 2 && A.dim() == 3 && B.dim() == 3 && x.stride(1) == 1 && out.stride(1) == 1);
        const int64_t rows = x.size(0), K = x.size(1), count = A.size(0), rank = A.size(1), N = B.size(1);
        require(out.scalar_type() == x.scalar_type() && out.device() == x.device() && A.size(2) == K && B.size(0) == count && B.size(2) == rank &&
                out.size(0) == rows && out.size(1) == N && ids.numel() == rows && rank <= INT_MAX);
        const float* scales = nullptr;
        if (a[5] != Py_None) {
            const at::Tensor& t = plain(a[5], at::kFloat, x);
            require(t.numel() == count);
            scales = (const float*)t.data_ptr();
        }
        at::Tensor own;
        size_t size = 0;
        void* ws = scratch_of(a[6], x, lib.adapters_workspace_bytes(rows, count, (int)rank, N, K), &size, &own);
        const void *xp = x.data_ptr(), *ap = A.data_ptr(), *bp = B.data_ptr();
        const int32_t* ip = (const int32_t*)ids.data_ptr();
        const int64_t xs = x.stride(0), os = out.stride(0);
        void *op = out.data_ptr(), *s = stream();
        call("fq_adapters", [&] { return lib.adapters(xp, xs, act, rows, N, K, ap, bp, count, (int)rank, ip, scales, op, os, ws, size, s); });
        Py_INCREF(a[4]);
        return a[4];
    });
}

// bind(FqError, addresses of the functions of `lib`, in its order)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    constexpr Py_ssize_t count = sizeof(lib) / sizeof(void*);
    if (n != 1 + count) {
        PyErr_SetString(PyExc_TypeError, "bind: wrong number of functions");
        return nullptr;
    }
    void* p[count];
    for (Py_ssize_t i = 0; i < count; ++i) {
        p[i] = PyLong_AsVoidPtr(a[1 + i]);
        if (!p[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind: no address");
            return nullptr;
        }
    }
    memcpy(&lib, p, sizeof(lib));
    Py_INCREF(a[0]);
    Py_XSETREF(fq_error, a[0]);
    Py_RETURN_NONE;
}

#define FQ_METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FQ_METHOD(gemm),     FQ_METHOD(gemm_grouped),  FQ_METHOD(quantize_act_i8), FQ_METHOD(gemm_w4a8),
                         FQ_METHOD(quantize), FQ_METHOD(quantize_w4a8), FQ_METHOD(qk_norm_rope),    FQ_METHOD(attention_prompt),
                         FQ_METHOD(attention_tree), FQ_METHOD(kv4_write),     FQ_METHOD(kv4_read),        FQ_METHOD(attention_tree_kv4),
                         FQ_METHOD(pages_take), FQ_METHOD(pages_fork),   FQ_METHOD(pages_free),      FQ_METHOD(pages_compact),
                         FQ_METHOD(adapters), FQ_METHOD(bind),           {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fqcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fqcall(void) { return PyModule_Create(&module); }
