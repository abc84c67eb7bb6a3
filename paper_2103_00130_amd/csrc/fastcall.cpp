// The calls that a serving loop makes for every layer, every lookup and every decoding step, marshalled natively: the operands of
// abft_gemm_u8s8s32_checked, abft_eb_u8_checked, abft_w4_gemv, abft_kv_plan, abft_kv_append, abft_kv_append_rotary, abft_kv_read,
// abft_kv_attention, abft_lora_gemv and abft_logprobs are unpacked from torch tensors here and handed to the C ABI, whose addresses bind() receives.  What binding.py checks is checked here too, and whatever does not pass - another type, a wrong
// shape, a tensor subclass - is left to it: the function returns None, and the Python code that follows raises what it
// always raised.  A call took 9.3-10 us of host time through ctypes, more than most of the kernels it launches run.
// The interpreter lock is released around the library call, as ctypes does.
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/abft_eb.h"
#include "../../include/abft_gemm.h"

namespace {

decltype(&abft_gemm_u8s8s32_checked) g_gemm = nullptr;
decltype(&abft_eb_u8_checked) g_eb = nullptr;
decltype(&abft_w4_gemv) g_w4 = nullptr;
decltype(&abft_kv_plan) g_plan = nullptr;
decltype(&abft_kv_append) g_append = nullptr;
decltype(&abft_kv_read) g_read = nullptr;
decltype(&abft_kv_attention) g_attention = nullptr;
decltype(&abft_kv_append_rotary) g_append_rotary = nullptr;
decltype(&abft_lora_gemv) g_lora = nullptr;
decltype(&abft_logprobs) g_logprobs = nullptr;
PyObject* g_current_device = nullptr;  // () -> int
PyObject* g_raw_stream = nullptr;      // (device) -> the current stream of that device, as an integer
PyObject* g_cuda_stream = nullptr;     // the attribute name of an explicit stream

struct Leave {};  // "not mine": the caller's Python code takes over

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o)) throw Leave{};
    return THPVariable_Unpack(o);
}

// a device tensor of the given type, or null for None
const at::Tensor* operand(PyObject* o, at::ScalarType type) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o);
    if (!t.is_cuda() || t.scalar_type() != type || t.layout() != at::kStrided) throw Leave{};
    return &t;
}
const at::Tensor& needed(PyObject* o, at::ScalarType type) {
    const at::Tensor* t = operand(o, type);
    if (!t) throw Leave{};
    return *t;
}

template <typename T>
T* ptr(const at::Tensor* t) {
    return t ? static_cast<T*>(t->data_ptr()) : nullptr;
}

// leading dimension of a matrix with unit column stride
int64_t leading(const at::Tensor& t) {
    if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1)) throw Leave{};
    return t.size(0) > 1 ? t.stride(0) : std::max(t.stride(0), t.size(1));
}

void entries(const at::Tensor* t, int64_t at_least, bool contiguous) {
    if (t && (t->numel() < at_least || (contiguous && !t->is_contiguous()))) throw Leave{};
}

long long integer(PyObject* o) {
    if (!PyLong_CheckExact(o)) throw Leave{};
    int over = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &over);
    if (over) throw Leave{};
    return v;
}

void* handle(PyObject* o) {
    if (!PyLong_CheckExact(o)) throw Leave{};
    void* const h = PyLong_AsVoidPtr(o);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        throw Leave{};
    }
    return h;
}

void* stream(PyObject* o) {
    PyObject* v = nullptr;
    if (o == Py_None) {
        PyObject* const dev = PyObject_CallNoArgs(g_current_device);
        if (dev) {
            v = PyObject_CallOneArg(g_raw_stream, dev);
            Py_DECREF(dev);
        }
    } else {
        v = PyObject_GetAttr(o, g_cuda_stream);
    }
    if (!v || !PyLong_Check(v)) {
        Py_XDECREF(v);
        PyErr_Clear();
        throw Leave{};
    }
    void* const s = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        throw Leave{};
    }
    return s;
}

// gemm(A, handle, K, N, C, row_flags, err_count, rq, Cq, inj, n_inj, flags, workspace, stream) -> return code, or None.
// rq: an abft_requant_t of the binding (its bytes are the struct), or None
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    Py_buffer rq_bytes;
    bool have_rq = false;
    int rc = 0;
    try {
        if (n != 14 || !g_gemm) throw Leave{};
        const at::Tensor& A = needed(a[0], at::kByte);
        const int64_t lda = leading(A), M = A.size(0), K = integer(a[2]), N = integer(a[3]);
        if (A.size(1) != K || M > 0x7fffffff) throw Leave{};
        const at::Tensor *C = operand(a[4], at::kInt), *flags_out = operand(a[5], at::kInt), *count = operand(a[6], at::kInt);
        const at::Tensor *Cq = operand(a[8], at::kByte), *inj = operand(a[9], at::kInt);
        int64_t ldc = 0, ldcq = 0;
        if (C) {
            ldc = leading(*C);
            if (C->size(0) != M || C->size(1) != N) throw Leave{};
        }
        if (Cq) {
            ldcq = leading(*Cq);
            if (Cq->size(0) != M || Cq->size(1) != N) throw Leave{};
        }
        const long long n_inj = integer(a[10]), flags = integer(a[11]);
        if (n_inj < -0x80000000ll || n_inj > 0x7fffffffll || flags < 0 || flags > 0xffffffffll) throw Leave{};
        entries(flags_out, M, false);
        entries(inj, 3 * n_inj, false);
        void* ws = nullptr;
        size_t ws_bytes = 0;
        if (a[12] != Py_None) {
            const at::Tensor& w = tensor(a[12]);
            if (!w.is_cuda() || !w.is_contiguous()) throw Leave{};
            ws = w.data_ptr();
            ws_bytes = (size_t)w.numel() * w.element_size();
        }
        void* const Bp = handle(a[1]);
        void* const s = stream(a[13]);
        if (a[7] != Py_None) {
            if (PyObject_GetBuffer(a[7], &rq_bytes, PyBUF_SIMPLE) != 0) {
                PyErr_Clear();
                throw Leave{};
            }
            have_rq = true;
            if (rq_bytes.len != (Py_ssize_t)sizeof(abft_requant_t)) throw Leave{};
        }
        const uint8_t* const A_ptr = ptr<uint8_t>(&A);
        int32_t *const C_ptr = ptr<int32_t>(C), *const flags_ptr = ptr<int32_t>(flags_out), *const count_ptr = ptr<int32_t>(count);
        uint8_t* const Cq_ptr = ptr<uint8_t>(Cq);
        const abft_inject_t* const inj_ptr = ptr<abft_inject_t>(inj);
        const abft_requant_t* const rq = have_rq ? static_cast<const abft_requant_t*>(rq_bytes.buf) : nullptr;
        Py_BEGIN_ALLOW_THREADS
        rc = g_gemm(A_ptr, lda, (int)M, static_cast<const abft_packed_b*>(Bp), C_ptr, ldc, flags_ptr, count_ptr, rq, Cq_ptr, ldcq,
                    inj_ptr, (int)n_inj, (uint32_t)flags, ws, ws_bytes, s);
        Py_END_ALLOW_THREADS
    } catch (...) {   // (a tensor without storage throws from data_ptr)
        if (have_rq) PyBuffer_Release(&rq_bytes);
        Py_RETURN_NONE;
    }
    if (have_rq) PyBuffer_Release(&rq_bytes);
    return PyLong_FromLong(rc);
}

// eb(handle, d, indices, offsets, R, bag_flags, weights, rsum, csum, rel_bound, flags, stream) -> return code, or None
PyObject* eb(PyObject*, PyObject* const* a, Py_ssize_t n) {
    int rc = 0;
    try {
        if (n != 12 || !g_eb) throw Leave{};
        const at::Tensor &indices = needed(a[2], at::kLong), &offsets = needed(a[3], at::kLong), &R = needed(a[4], at::kFloat);
        const int64_t n_bags = offsets.numel() - 1, n_indices = indices.numel();
        if (n_bags < 0 || !offsets.is_contiguous() || !indices.is_contiguous()) throw Leave{};
        const int64_t ldr = leading(R);
        if (R.size(0) < n_bags || R.size(1) != integer(a[1])) throw Leave{};
        const at::Tensor *bag_flags = operand(a[5], at::kInt), *weights = operand(a[6], at::kFloat);
        const at::Tensor *rsum = operand(a[7], at::kDouble), *csum = operand(a[8], at::kDouble);
        entries(bag_flags, n_bags, true);
        entries(rsum, n_bags, true);
        entries(csum, n_bags, true);
        if (weights && (weights->numel() != n_indices || !weights->is_contiguous())) throw Leave{};
        if (!PyFloat_CheckExact(a[9])) throw Leave{};
        const double bound = PyFloat_AS_DOUBLE(a[9]);
        const long long flags = integer(a[10]);
        if (flags < 0 || flags > 0xffffffffll) throw Leave{};
        void* const Tp = handle(a[0]);
        void* const s = stream(a[11]);
        const int64_t *const idx_ptr = ptr<int64_t>(&indices), *const off_ptr = ptr<int64_t>(&offsets);
        const float* const w_ptr = ptr<float>(weights);
        float* const R_ptr = ptr<float>(&R);
        int32_t* const f_ptr = ptr<int32_t>(bag_flags);
        double *const rs_ptr = ptr<double>(rsum), *const cs_ptr = ptr<double>(csum);
        Py_BEGIN_ALLOW_THREADS
        rc = g_eb(static_cast<const abft_eb_table*>(Tp), idx_ptr, n_indices, off_ptr, n_bags, w_ptr, R_ptr, ldr, f_ptr, rs_ptr, cs_ptr,
                  bound, (unsigned)flags, s);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

// ABFT_TYPE_* of a device tensor of activations
int value_type(const at::Tensor& t) {
    if (!t.is_cuda() || t.layout() != at::kStrided) throw Leave{};
    switch (t.scalar_type()) {
        case at::kFloat: return ABFT_TYPE_F32;
        case at::kHalf: return ABFT_TYPE_F16;
        case at::kBFloat16: return ABFT_TYPE_BF16;
        default: throw Leave{};
    }
}
int small(PyObject* o) {
    const long long v = integer(o);
    if (v < -0x80000000ll || v > 0x7fffffffll) throw Leave{};
    return (int)v;
}
// the address of a contiguous tensor of at least n entries
template <typename T>
T* vec(PyObject* o, at::ScalarType type, int64_t n) {
    const at::Tensor& t = needed(o, type);
    entries(&t, n, true);
    return ptr<T>(&t);
}
// tokens x heads x head_dim values, columns side by side
struct Rows {
    void* at;
    int64_t token, head;
    int type;
};
Rows rows(PyObject* o, int64_t n, int64_t heads, int64_t dim) {
    const at::Tensor& t = tensor(o);
    Rows r;
    r.type = value_type(t);
    if (t.dim() != 3 || t.size(0) != n || t.size(1) != heads || t.size(2) != dim || (dim > 1 && t.stride(2) != 1)) throw Leave{};
    r.at = t.data_ptr();
    r.token = t.stride(0);
    r.head = t.stride(1);
    return r;
}

// w4(X, handle, N, K, Y, stream) -> return code, or None
PyObject* w4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    int rc = 0;
    try {
        if (n != 6 || !g_w4) throw Leave{};
        const at::Tensor &X = tensor(a[0]), &Y = tensor(a[4]);
        const int type = value_type(X);
        if (value_type(Y) != type) throw Leave{};
        const int64_t ldx = leading(X), ldy = leading(Y), M = X.size(0);
        if (X.size(1) != integer(a[3]) || Y.size(1) != integer(a[2]) || Y.size(0) != M || M > 0x7fffffff) throw Leave{};
        void* const Wp = handle(a[1]);
        void* const s = stream(a[5]);
        void *const x = X.data_ptr(), *const y = Y.data_ptr();
        Py_BEGIN_ALLOW_THREADS
        rc = g_w4(x, ldx, type, (int)M, static_cast<const abft_w4*>(Wp), y, ldy, s);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

// plan(ctx_len, new_len, block_tokens, table, free_blocks, seq_len, cu_new, slots, req_flags, taken, stream) -> return code, or None
PyObject* plan(PyObject*, PyObject* const* a, Py_ssize_t n) {
    int rc = 0;
    try {
        if (n != 11 || !g_plan) throw Leave{};
        const int64_t R = needed(a[0], at::kInt).numel();
        const at::Tensor &table = needed(a[3], at::kInt), &free_blocks = needed(a[4], at::kInt), &slots_t = needed(a[7], at::kLong);
        if (R > 0x7fffffff || table.dim() != 2 || table.size(0) != R || table.size(1) > 0x7fffffff || free_blocks.numel() > 0x7fffffff) throw Leave{};
        const int64_t ldt = std::max(leading(table), table.size(1)), n_slots = slots_t.numel();
        const int32_t *const ctx = vec<int32_t>(a[0], at::kInt, R), *const fresh = vec<int32_t>(a[1], at::kInt, R);
        const int block = small(a[2]), width = (int)table.size(1), n_free = (int)free_blocks.numel();
        int32_t* const tab = ptr<int32_t>(&table);
        const int32_t* const free_at = vec<int32_t>(a[4], at::kInt, 0);
        int32_t *const seq = vec<int32_t>(a[5], at::kInt, R), *const cu = vec<int32_t>(a[6], at::kInt, R + 1);
        int64_t* const slots = vec<int64_t>(a[7], at::kLong, 0);
        int32_t *const flags = vec<int32_t>(a[8], at::kInt, R), *const taken = vec<int32_t>(a[9], at::kInt, 1);
        void* const s = stream(a[10]);
        Py_BEGIN_ALLOW_THREADS
        rc = g_plan(ctx, fresh, (int)R, block, tab, ldt, width, free_at, n_free, seq, cu, slots, n_slots, flags, taken, s);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

// append(cache struct, heads, head_dim, K, V, slots, stream) -> return code, or None
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    int rc = 0;
    try {
        if (n != 7 || !g_append) throw Leave{};
        const int64_t heads = integer(a[1]), dim = integer(a[2]), T = needed(a[5], at::kLong).numel();
        const Rows k = rows(a[3], T, heads, dim), v = rows(a[4], T, heads, dim);
        if (k.type != v.type) throw Leave{};
        const int64_t* const slots = vec<int64_t>(a[5], at::kLong, T);
        const abft_kv_cache_t* const cache = static_cast<const abft_kv_cache_t*>(handle(a[0]));
        void* const s = stream(a[6]);
        Py_BEGIN_ALLOW_THREADS
        rc = g_append(cache, k.at, k.token, k.head, v.at, v.token, v.head, k.type, slots, T, s);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

// read(cache struct, heads, head_dim, slots, K, V, stream) -> return code, or None
PyObject* read(PyObject*, PyObject* const* a, Py_ssize_t n) {
    int rc = 0;
    try {
        if (n != 7 || !g_read) throw Leave{};
        const int64_t heads = integer(a[1]), dim = integer(a[2]), T = needed(a[3], at::kLong).numel();
        const Rows k = rows(a[4], T, heads, dim), v = rows(a[5], T, heads, dim);
        if (k.type != v.type) throw Leave{};
        const int64_t* const slots = vec<int64_t>(a[3], at::kLong, T);
        const abft_kv_cache_t* const cache = static_cast<const abft_kv_cache_t*>(handle(a[0]));
        void* const s = stream(a[6]);
        Py_BEGIN_ALLOW_THREADS
        rc = g_read(cache, slots, T, k.at, k.token, k.head, v.at, v.token, v.head, k.type, s);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

// attention(cache struct, head_dim, Q, table, seq_len, cu_new, O, max_new, max_len, scale, lse, req_flags, workspace, stream) -> return code, or None
PyObject* attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
    int rc = 0;
    try {
        if (n != 14 || !g_attention) throw Leave{};
        const at::Tensor &Q = tensor(a[2]), &table = needed(a[3], at::kInt);
        const int64_t dim = integer(a[1]), R = needed(a[4], at::kInt).numel();
        if (Q.dim() != 3 || table.dim() != 2 || R > 0x7fffffff || table.size(0) != R || table.size(1) > 0x7fffffff || Q.size(1) > 0x7fffffff) throw Leave{};
        const Rows q = rows(a[2], Q.size(0), Q.size(1), dim), o = rows(a[6], Q.size(0), Q.size(1), dim);
        if (q.type != o.type || !PyFloat_CheckExact(a[9])) throw Leave{};
        const int64_t n_rows = Q.size(0), ldt = std::max(leading(table), table.size(1));
        const int32_t* const tab = ptr<int32_t>(&table);
        const int32_t *const seq = vec<int32_t>(a[4], at::kInt, R), *const cu = vec<int32_t>(a[5], at::kInt, R + 1);
        const int q_heads = (int)Q.size(1), width = (int)table.size(1), max_new = small(a[7]), max_len = small(a[8]);
        const float scale = (float)PyFloat_AS_DOUBLE(a[9]);
        float* const lse = a[10] == Py_None ? nullptr : vec<float>(a[10], at::kFloat, n_rows * q_heads);
        int32_t* const flags = a[11] == Py_None ? nullptr : vec<int32_t>(a[11], at::kInt, R);
        void* ws = nullptr;
        size_t ws_bytes = 0;
        if (a[12] != Py_None) {
            const at::Tensor& w = tensor(a[12]);
            if (!w.is_cuda() || !w.is_contiguous()) throw Leave{};
            ws = w.data_ptr();
            ws_bytes = (size_t)w.numel() * w.element_size();
        }
        const abft_kv_cache_t* const cache = static_cast<const abft_kv_cache_t*>(handle(a[0]));
        void* const s = stream(a[13]);
        Py_BEGIN_ALLOW_THREADS
        rc = g_attention(cache, q.at, q.token, q.head, q.type, n_rows, q_heads, tab, ldt, width, seq, cu, (int)R, max_new, max_len, scale,
                         o.at, o.token, o.head, lse, flags, ws, ws_bytes, s);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

// memory that a caller lends: a contiguous device tensor of any type, or none
struct Lent {
    void* at = nullptr;
    size_t bytes = 0;
};
Lent lent(PyObject* o) {
    Lent l;
    if (o == Py_None) return l;
    const at::Tensor& w = tensor(o);
    if (!w.is_cuda() || !w.is_contiguous()) throw Leave{};
    l.at = w.data_ptr();
    l.bytes = (size_t)w.numel() * w.element_size();
    return l;
}

// append_rotary(cache struct, heads, head_dim, Q, K, V, slots, positions, table, QR, neighbours, stream) -> return code, or None
PyObject* append_rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    int rc = 0;
    try {
        if (n != 12 || !g_append_rotary || !PyBool_Check(a[10])) throw Leave{};
        const int64_t heads = integer(a[1]), dim = integer(a[2]), T = needed(a[6], at::kLong).numel();
        const Rows k = rows(a[4], T, heads, dim), v = rows(a[5], T, heads, dim);
        Rows q = {nullptr, 0, 0, k.type}, r = q;
        int64_t q_heads = 0;
        if (a[3] != Py_None) {
            const at::Tensor& Q = tensor(a[3]);
            if (Q.dim() != 3 || Q.size(1) > 0x7fffffff) throw Leave{};
            q_heads = Q.size(1);
            q = rows(a[3], T, q_heads, dim);
            r = rows(a[9], T, q_heads, dim);
        } else if (a[9] != Py_None) {
            throw Leave{};
        }
        if (k.type != v.type || q.type != k.type || r.type != k.type) throw Leave{};
        const at::Tensor& table = needed(a[8], at::kFloat);
        if (table.dim() != 2 || !table.is_contiguous() || table.size(1) > 0x7fffffff) throw Leave{};
        const int64_t* const slots = vec<int64_t>(a[6], at::kLong, T);
        const int32_t* const positions = vec<int32_t>(a[7], at::kInt, T);
        const abft_kv_cache_t* const cache = static_cast<const abft_kv_cache_t*>(handle(a[0]));
        const float* const angles = ptr<float>(&table);
        const int64_t n_positions = table.size(0), rot = table.size(1);
        const int pairs = a[10] == Py_True ? ABFT_ROTARY_NEIGHBOURS : ABFT_ROTARY_HALVES;
        void* const s = stream(a[11]);
        Py_BEGIN_ALLOW_THREADS
        rc = g_append_rotary(cache, q.at, q.token, q.head, (int)q_heads, r.at, r.token, r.head, k.at, k.token, k.head, v.at, v.token, v.head, k.type, slots,
                             positions, T, angles, n_positions, (int)rot, pairs, s);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

// lora(X, pool struct, K, N, type, ids, base, Y, workspace, stream) -> return code, or None
PyObject* lora(PyObject*, PyObject* const* a, Py_ssize_t n) {
    int rc = 0;
    try {
        if (n != 10 || !g_lora) throw Leave{};
        const at::Tensor &X = tensor(a[0]), &base = tensor(a[6]), &Y = tensor(a[7]);
        const int64_t K = integer(a[2]), N = integer(a[3]), type = integer(a[4]);
        if (value_type(X) != type || value_type(base) != type || value_type(Y) != type) throw Leave{};
        const int64_t ldx = leading(X), ldb = leading(base), ldy = leading(Y), M = X.size(0);
        if (X.size(1) != K || base.size(0) != M || base.size(1) != N || Y.size(0) != M || Y.size(1) != N || M > 0x7fffffff) throw Leave{};
        const int32_t* const ids = vec<int32_t>(a[5], at::kInt, M);
        const Lent ws = lent(a[8]);
        const abft_lora_t* const pool = static_cast<const abft_lora_t*>(handle(a[1]));
        void* const s = stream(a[9]);
        void *const x = X.data_ptr(), *const b = base.data_ptr(), *const y = Y.data_ptr();
        Py_BEGIN_ALLOW_THREADS
        rc = g_lora(x, ldx, (int)M, pool, ids, b, ldb, y, ldy, ws.at, ws.bytes, s);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

// logprobs(logits, targets, logprob, rank, entropy, lse, top_logprob, top_index, scale, workspace, stream) -> return code, or None
PyObject* logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
    int rc = 0;
    try {
        if (n != 11 || !g_logprobs || !PyFloat_CheckExact(a[8]) || (a[6] == Py_None) != (a[7] == Py_None)) throw Leave{};
        const at::Tensor& x = tensor(a[0]);
        const int type = value_type(x);
        const int64_t ldl = leading(x), M = x.size(0), V = x.size(1);
        if (V > 0x7fffffff) throw Leave{};
        int64_t top = 0;
        if (a[7] != Py_None) {
            const at::Tensor &value = needed(a[6], at::kFloat), &index = needed(a[7], at::kLong);
            if (index.dim() != 2 || index.size(0) != M || value.sizes() != index.sizes() || index.size(1) > 0x7fffffff) throw Leave{};
            top = index.size(1);
        }
        const auto f = [&](PyObject* o, int64_t count) { return o == Py_None ? nullptr : vec<float>(o, at::kFloat, count); };
        const int64_t* const targets = a[1] == Py_None ? nullptr : vec<int64_t>(a[1], at::kLong, M);
        float *const logprob = f(a[2], M), *const entropy = f(a[4], M), *const lse = f(a[5], M), *const top_logprob = f(a[6], M * top);
        int32_t* const rank = a[3] == Py_None ? nullptr : vec<int32_t>(a[3], at::kInt, M);
        int64_t* const top_index = a[7] == Py_None ? nullptr : vec<int64_t>(a[7], at::kLong, M * top);
        const float scale = (float)PyFloat_AS_DOUBLE(a[8]);
        const Lent ws = lent(a[9]);
        void* const s = stream(a[10]);
        void* const logits = x.data_ptr();
        Py_BEGIN_ALLOW_THREADS
        rc = g_logprobs(logits, ldl, type, M, (int)V, scale, targets, logprob, rank, entropy, lse, (int)top, top_logprob, top_index, ws.at, ws.bytes, s);
        Py_END_ALLOW_THREADS
    } catch (...) {
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

template <typename F>
bool address(PyObject* list, Py_ssize_t i, F* f) {
    PyObject* const o = PyList_GetItem(list, i);
    void* const at = o ? PyLong_AsVoidPtr(o) : nullptr;
    if (PyErr_Occurred()) return false;
    *f = reinterpret_cast<F>(at);
    return true;
}

// bind([addresses of abft_gemm_u8s8s32_checked, abft_eb_u8_checked, abft_w4_gemv, abft_kv_plan, abft_kv_append, abft_kv_read, abft_kv_attention,
// abft_kv_append_rotary, abft_lora_gemv, abft_logprobs], current_device, raw_stream)
PyObject* bind(PyObject*, PyObject* args) {
    PyObject *list, *device, *raw;
    if (!PyArg_ParseTuple(args, "O!OO", &PyList_Type, &list, &device, &raw)) return nullptr;
    if (!address(list, 0, &g_gemm) || !address(list, 1, &g_eb) || !address(list, 2, &g_w4) || !address(list, 3, &g_plan) ||
        !address(list, 4, &g_append) || !address(list, 5, &g_read) || !address(list, 6, &g_attention) ||
        !address(list, 7, &g_append_rotary) || !address(list, 8, &g_lora) || !address(list, 9, &g_logprobs))
        return nullptr;
    Py_INCREF(device);
    Py_INCREF(raw);
    Py_XSETREF(g_current_device, device);
    Py_XSETREF(g_raw_stream, raw);
    Py_RETURN_NONE;
}

PyMethodDef g_methods[] = {
    {"gemm", (PyCFunction)(void (*)(void))gemm, METH_FASTCALL, "abft_gemm_u8s8s32_checked on torch tensors; None when the operands are not what it takes"},
    {"eb", (PyCFunction)(void (*)(void))eb, METH_FASTCALL, "abft_eb_u8_checked on torch tensors; None when the operands are not what it takes"},
#define ABFT_FAST(name, what) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, what " on torch tensors; None when the operands are not what it takes"}
    ABFT_FAST(w4, "abft_w4_gemv"),
    ABFT_FAST(plan, "abft_kv_plan"),
    ABFT_FAST(append, "abft_kv_append"),
    ABFT_FAST(read, "abft_kv_read"),
    ABFT_FAST(attention, "abft_kv_attention"),
    ABFT_FAST(append_rotary, "abft_kv_append_rotary"),
    ABFT_FAST(lora, "abft_lora_gemv"),
    ABFT_FAST(logprobs, "abft_logprobs"),
#undef ABFT_FAST
    {"bind", bind, METH_VARARGS, "addresses of the library's functions, and where to ask for the current device and stream"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_fastcall", "native marshalling of the calls of a serving loop", -1, g_methods,
                        nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fastcall(void) {
    g_cuda_stream = PyUnicode_InternFromString("cuda_stream");
    return g_cuda_stream ? PyModule_Create(&g_module) : nullptr;
}
