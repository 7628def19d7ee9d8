// CPython side of the step calls: reads the tensor bundles of binding.py and makes the C call, without building ctypes
// structures in Python (a step's three calls took 55 us of host time that way, more than the GPU needs for a small
// tree).  Only the CPython API is used: a tensor is asked for its `data_ptr`, `stride` and `size` like any object, so
// the module does not depend on torch's C++ interface.  Every function returns the hs_status as an int.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <stddef.h>

#include "../../include/heterospec.h"

extern "C" int hs_context_device(const hs_ctx* ctx);        // (of the library, not of its interface)

namespace {

PyObject *n_data_ptr, *n_contiguous, *n_get_device, *n_numel, *n_stride, *n_size, *n_dtype, *o_zero, *o_one, *o_two, *t_f32, *t_bf16, *t_i32;

struct Name {
    const char* text;
    PyObject* str;
};
Name k_tree[] = {{"batch"}, {"n_nodes_total"}, {"node_off"}, {"parent"}, {"token"}};
Name k_quant[] = {{"row_max"}, {"row_lse"}, {"h_full"}, {"i_topk"}, {"i_trunc"}, {"topk_val"}, {"topk_idx"},
                  {"logc"}, {"score"}, {"phi"}, {"depth"}, {"pstar_node"}, {"phi_star"}, {"status"}};
Name k_pruned[] = {{"bin"}, {"d_prime"}, {"n_prime"}, {"n_keep"}, {"keep_off"}, {"keep_idx"}, {"new_parent"},
                   {"new_depth"}, {"keep_rank"}, {"anc_mask"}, {"status"}};
Name k_accept[] = {{"accept_len"}, {"path_nodes"}, {"path_compact"}, {"path_tokens"}, {"bonus_token"},
                   {"terminal_rank"}, {"status"}, {"path_cap"}, {"max_kept_rows"}};
Name k_expand[] = {{"batch"}, {"cap"}, {"top_k"}, {"n_cand"}, {"parent"}, {"token"}, {"depth"}, {"logc"}, {"score"},
                   {"frontier"}, {"n_frontier"}, {"status"}};
Name k_policy[] = {{"thresholds"}, {"d_base"}, {"alpha"}, {"n_default"}, {"top_k"}, {"gamma_pct"}, {"phi_mode"},
                   {"pstar_mode"}, {"entropy_mode"}};
Name k_cache[] = {{"batch"}, {"hkv"}, {"head_dim"}, {"page_size"}, {"n_pages"}, {"max_pages"}, {"k"}, {"v"}, {"k_scale"},
                  {"v_scale"}, {"page_table"}, {"kv_len"}, {"device_index"}};
Name k_rope[] = {{"address"}};

// fields of k_pruned and k_accept, as bits
enum : unsigned int { PRUNED_N_KEEP = 1u << 3, PRUNED_KEEP_OFF = 1u << 4, PRUNED_KEEP_IDX = 1u << 5, PRUNED_NEW_DEPTH = 1u << 7, PRUNED_ANC_MASK = 1u << 9,
                      PRUNED_STATUS = 1u << 10, ACCEPT_LEN = 1u << 0, ACCEPT_PATHS = 3u << 1, ACCEPT_STATUS = 1u << 6 };
const char* const k_batch = "the trees and the cache are of one batch";
const char* const k_offsets = "offsets have an entry more than the batch has sequences";
const char* const k_entries = "an entry for every sequence of the batch is expected";

bool intern_all(Name* k, size_t n) {
    for (size_t i = 0; i < n; ++i)
        if (!(k[i].str = PyUnicode_InternFromString(k[i].text))) return false;
    return true;
}

// Reads arguments and fields; after a failed read `bad` stays set, the Python error with it, and reads return 0.
struct Reader {
    bool bad = false;
    long long device = -2;          // of the tensors that were asked for theirs: -2 none yet, -1 host memory, -3 several

    long long integer(PyObject* o) {
        if (bad) return 0;
        const unsigned long long v = PyLong_AsUnsignedLongLongMask(o);
        if (v == (unsigned long long)-1 && PyErr_Occurred()) bad = true;
        return (long long)v;
    }
    double real(PyObject* o) {
        if (bad) return 0.0;
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) bad = true;
        return v;
    }
    // device pointer of a tensor, NULL for None
    void* ptr(PyObject* o) {
        if (bad || o == Py_None) return nullptr;
        PyObject* args[] = {nullptr, o};                             // (the call may use the slot ahead of its arguments)
        PyObject* r = PyObject_VectorcallMethod(n_data_ptr, args + 1, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr);
        if (!r) { bad = true; return nullptr; }
        void* p = (void*)(uintptr_t)PyLong_AsUnsignedLongLongMask(r);
        Py_DECREF(r);
        return p;
    }
    long long dim(PyObject* name, PyObject* t, PyObject* index) {
        if (bad) return 0;
        PyObject* args[] = {nullptr, t, index};
        PyObject* r = PyObject_VectorcallMethod(name, args + 1, 2 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr);
        if (!r) { bad = true; return 0; }
        const long long v = integer(r);
        Py_DECREF(r);
        return v;
    }
    long long size(PyObject* t, PyObject* index) { return dim(n_size, t, index); }
    long long stride(PyObject* t, PyObject* index) { return dim(n_stride, t, index); }
    hs_dtype dtype(PyObject* t, const char* what = "logits") {
        if (bad) return HS_F32;
        PyObject* d = PyObject_GetAttr(t, n_dtype);
        if (!d) { bad = true; return HS_F32; }
        Py_DECREF(d);
        if (d == t_bf16) return HS_BF16;
        if (d == t_f32) return HS_F32;
        bad = true;
        PyErr_Format(PyExc_TypeError, "%s must be float32 or bfloat16, got %S", what, d);
        return HS_F32;
    }
    void* field_ptr(PyObject* o, const Name& k) {
        if (bad) return nullptr;
        PyObject* v = PyObject_GetAttr(o, k.str);
        if (!v) { bad = true; return nullptr; }
        void* p = ptr(v);
        Py_DECREF(v);
        return p;
    }
    int field_int(PyObject* o, const Name& k) {
        if (bad) return 0;
        PyObject* v = PyObject_GetAttr(o, k.str);
        if (!v) { bad = true; return 0; }
        const int i = (int)integer(v);
        Py_DECREF(v);
        return i;
    }
    // n pointers in declaration order (the C structs start with, or consist of, an unbroken run of pointers)
    void pointers(PyObject* o, const Name* k, int n, void* dst) {
        void** out = (void**)dst;
        for (int i = 0; i < n; ++i) out[i] = field_ptr(o, k[i]);
    }
    // only the pointers that a call reads (bits of `which`), the others NULL: a field costs a quarter of a microsecond
    void some(PyObject* o, const Name* k, int n, unsigned int which, void* dst) {
        void** out = (void**)dst;
        for (int i = 0; i < n; ++i) out[i] = which >> i & 1u ? field_ptr(o, k[i]) : nullptr;
    }
    // the three sizes or strides of a tensor
    void three(PyObject* name, PyObject* t, long long* out) {
        if (bad) return;
        PyObject* args[] = {nullptr, t};
        PyObject* r = PyObject_VectorcallMethod(name, args + 1, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr);
        if (!r) { bad = true; return; }
        if (!PyTuple_Check(r) || PyTuple_GET_SIZE(r) != 3) fail("a tensor [rows, heads, values] is expected");
        else for (int i = 0; i < 3; ++i) out[i] = integer(PyTuple_GET_ITEM(r, i));
        Py_DECREF(r);
    }
    void met(long long d) { device = device == -2 || device == d ? d : -3; }
    void locate(PyObject* t) {
        if (bad) return;
        PyObject* args[] = {nullptr, t};
        PyObject* r = PyObject_VectorcallMethod(n_get_device, args + 1, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr);
        if (!r) { bad = true; return; }
        met(integer(r));
        Py_DECREF(r);
    }
    // (a pointer into host memory, or another device's, would fault the context's)
    void here(const hs_ctx* ctx) {
        if (!bad && ctx && device != hs_context_device(ctx)) fail("the tensors of a call are on the context's device");
    }
    bool contiguous(PyObject* t) {
        if (bad) return false;
        PyObject* args[] = {nullptr, t};
        PyObject* r = PyObject_VectorcallMethod(n_contiguous, args + 1, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr);
        if (!r) { bad = true; return false; }
        Py_DECREF(r);
        return r == Py_True;
    }
    // entries of a tensor (a third of what size(0) costs)
    long long numel(PyObject* t) {
        if (bad) return 0;
        PyObject* args[] = {nullptr, t};
        PyObject* r = PyObject_VectorcallMethod(n_numel, args + 1, 1 | PY_VECTORCALL_ARGUMENTS_OFFSET, nullptr);
        if (!r) { bad = true; return 0; }
        const long long v = integer(r);
        Py_DECREF(r);
        return v;
    }
    // a tensor of `count` entries, or None
    void* list(PyObject* t, long long count, const char* why, PyObject* type = t_i32) {
        if (bad || t == Py_None) return nullptr;
        if (numel(t) != count && !bad) return fail(why);
        PyObject* d = bad ? nullptr : PyObject_GetAttr(t, n_dtype);
        if (!d) { bad = true; return nullptr; }
        Py_DECREF(d);
        if (d != type) {
            bad = true;
            PyErr_Format(PyExc_TypeError, "a tensor of %S is expected, got %S", type, d);
            return nullptr;
        }
        if (!contiguous(t) && !bad) return fail("a contiguous tensor is expected");      // (the calls take the entries to lie side by side)
        locate(t);
        return ptr(t);
    }
    // a bundle's `status` has an entry for each of `batch` sequences
    void batch_of(PyObject* o, const Name& status, long long batch, const char* why) {
        if (bad) return;
        PyObject* v = PyObject_GetAttr(o, status.str);
        if (!v) { bad = true; return; }
        if (numel(v) != batch && !bad) fail(why);
        Py_DECREF(v);
    }
    void tree(PyObject* o, hs_tree_batch* t) {
        t->batch = field_int(o, k_tree[0]);
        t->n_nodes_total = field_int(o, k_tree[1]);
        t->node_off = (const int32_t*)field_ptr(o, k_tree[2]);
        t->parent = (const int32_t*)field_ptr(o, k_tree[3]);
        t->token = (const int32_t*)field_ptr(o, k_tree[4]);
    }
    void expand(PyObject* o, hs_expand_state* s) {
        s->batch = field_int(o, k_expand[0]);
        s->cap = field_int(o, k_expand[1]);
        s->top_k = field_int(o, k_expand[2]);
        pointers(o, k_expand + 3, 9, &s->n_cand);
    }
    void cache(PyObject* o, hs_kv_cache* c) {
        int32_t* ints = &c->batch;
        for (int i = 0; i < 6; ++i) ints[i] = field_int(o, k_cache[i]);
        pointers(o, k_cache + 6, 6, &c->k);
        met(field_int(o, k_cache[12]));
    }
    const hs_rope* rope(PyObject* o) {
        if (bad) return nullptr;
        PyObject* v = PyObject_GetAttr(o, k_rope[0].str);
        if (!v) { bad = true; return nullptr; }
        const hs_rope* p = (const hs_rope*)(uintptr_t)integer(v);
        Py_DECREF(v);
        return p;
    }
    // [rows, heads, values] with the values of a head side by side; `whole`: the rows and heads too.  Sizes as the caller needs them.
    void* heads(PyObject* t, bool whole, hs_dtype want, long long* rows, long long* n_heads, long long* dim, int64_t* token_stride,
                int64_t* head_stride) {
        if (bad) return nullptr;
        const hs_dtype dt = dtype(t, "heads");
        if (bad) return nullptr;
        long long sizes[3] = {0, 0, 0}, strides[3] = {0, 0, 1};
        three(n_size, t, sizes);
        if (bad) return nullptr;
        *rows = sizes[0]; *n_heads = sizes[1]; *dim = sizes[2];
        if (contiguous(t)) {
            strides[0] = sizes[1] * sizes[2];
            strides[1] = sizes[2];
        } else {
            three(n_stride, t, strides);
            if (whole && !bad) return fail("a contiguous tensor [rows, heads, values] is expected");
        }
        if (bad) return nullptr;
        *token_stride = strides[0]; *head_stride = strides[1];
        if (dt != want) return fail("tensors of one call have one type");
        if (*rows > 0 && strides[2] != 1) return fail("the values of a head lie side by side");
        if (*n_heads == 1) *head_stride = *dim;              // (of a single head the stride means nothing)
        if (*rows <= 1 && *token_stride < *n_heads * *dim) *token_stride = *n_heads * *dim;
        locate(t);
        return ptr(t);
    }
    void* fail(const char* why) {
        bad = true;
        PyErr_SetString(PyExc_ValueError, why);
        return nullptr;
    }
    PyObject* item(PyObject* dict, const Name& k) {                  // borrowed
        if (bad) return nullptr;
        PyObject* v = PyDict_GetItemWithError(dict, k.str);
        if (!v) {
            bad = true;
            if (!PyErr_Occurred()) PyErr_SetObject(PyExc_KeyError, k.str);
        }
        return v;
    }
    void policy(PyObject* d, hs_policy* p) {
        for (int which = 0; which < 2 && !bad; ++which) {
            PyObject* v = item(d, k_policy[which ? 5 : 0]);
            if (bad) return;
            PyObject* s = PySequence_Fast(v, "the policy's thresholds and gamma_pct are sequences");
            if (!s) { bad = true; return; }
            const Py_ssize_t n = PySequence_Fast_GET_SIZE(s), want = which ? 3 : 7;
            for (Py_ssize_t i = 0; i < want; ++i) {                  // (missing entries are zero)
                PyObject* x = i < n ? PySequence_Fast_GET_ITEM(s, i) : nullptr;
                if (which) p->gamma_pct[i] = x ? (int)integer(x) : 0;
                else p->thresholds[i] = x ? (float)real(x) : 0.f;
            }
            Py_DECREF(s);
            if (n > want && !bad) { bad = true; PyErr_SetString(PyExc_IndexError, "invalid index"); }
        }
        int* at[] = {&p->d_base, &p->alpha, &p->n_default, &p->top_k};
        for (int i = 0; i < 4; ++i) if (PyObject* v = item(d, k_policy[1 + i])) *at[i] = (int)integer(v);
        int* modes[] = {&p->phi_mode, &p->pstar_mode, &p->entropy_mode};
        for (int i = 0; i < 3; ++i) if (PyObject* v = item(d, k_policy[6 + i])) *modes[i] = (int)integer(v);
    }
    hs_ctx* ctx(PyObject* o) { return (hs_ctx*)(uintptr_t)integer(o); }
    hs_stream stream(PyObject* o) { return (hs_stream)(uintptr_t)integer(o); }
};

static_assert(offsetof(hs_kv_cache, k) == 6 * sizeof(int32_t), "hs_kv_cache is six integers and six pointers");
static_assert(sizeof(hs_quant_out) == 14 * sizeof(void*), "hs_quant_out is fourteen pointers");
static_assert(sizeof(hs_pruned_tree) == 11 * sizeof(void*), "hs_pruned_tree is eleven pointers");

bool arity(Py_ssize_t got, Py_ssize_t want) {
    if (got == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, got);
    return false;
}

#define HS_NATIVE(name) PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n)
// the C call, with the interpreter lock released (a launch may wait for room in the driver's queue)
#define HS_DONE(call)                                   \
    do {                                                \
        hs_ctx* ctx = r.ctx(a[0]);                      \
        hs_stream stream = r.stream(a[n - 1]);          \
        if (r.bad) return nullptr;                      \
        hs_status st;                                   \
        Py_BEGIN_ALLOW_THREADS                          \
        st = call;                                      \
        Py_END_ALLOW_THREADS                            \
        return PyLong_FromLong((long)st);               \
    } while (0)

// the same for calls whose tensors were asked for their device
#define HS_DONE_HERE(call)                              \
    do {                                                \
        r.here(r.ctx(a[0]));                            \
        HS_DONE(call);                                  \
    } while (0)

// (ctx, tree, logits, policy, quant, stream)
HS_NATIVE(entropy_quantify) {
    if (!arity(n, 6)) return nullptr;
    Reader r;
    hs_tree_batch t; hs_policy p; hs_quant_out q;
    r.tree(a[1], &t); r.policy(a[3], &p); r.pointers(a[4], k_quant, 14, &q);
    const void* x = r.ptr(a[2]);
    const hs_dtype dt = r.dtype(a[2]);
    const long long rs = r.stride(a[2], o_zero), v = r.size(a[2], o_one);
    HS_DONE(hs_entropy_quantify(ctx, &t, x, dt, rs, (int)v, &p, &q, stream));
}
// (ctx, tree, logits, policy, quant, pruned, stream)
HS_NATIVE(entropy_quantify_prune) {
    if (!arity(n, 7)) return nullptr;
    Reader r;
    hs_tree_batch t; hs_policy p; hs_quant_out q; hs_pruned_tree k;
    r.tree(a[1], &t); r.policy(a[3], &p); r.pointers(a[4], k_quant, 14, &q); r.pointers(a[5], k_pruned, 11, &k);
    const void* x = r.ptr(a[2]);
    const hs_dtype dt = r.dtype(a[2]);
    const long long rs = r.stride(a[2], o_zero), v = r.size(a[2], o_one);
    HS_DONE(hs_entropy_quantify_prune(ctx, &t, x, dt, rs, (int)v, &p, &q, &k, stream));
}
// (ctx, tree, quant, policy, pruned, stream)
HS_NATIVE(stratify_prune) {
    if (!arity(n, 6)) return nullptr;
    Reader r;
    hs_tree_batch t; hs_policy p; hs_quant_out q; hs_pruned_tree k;
    r.tree(a[1], &t); r.pointers(a[2], k_quant, 14, &q); r.policy(a[3], &p); r.pointers(a[4], k_pruned, 11, &k);
    HS_DONE(hs_stratify_prune(ctx, &t, &q, &p, &k, stream));
}
// (ctx, tree, quant, policy, slo_class, budget, pruned, stream)
HS_NATIVE(stratify_prune_budget) {
    if (!arity(n, 8)) return nullptr;
    Reader r;
    hs_tree_batch t; hs_policy p; hs_quant_out q; hs_pruned_tree k;
    r.tree(a[1], &t); r.pointers(a[2], k_quant, 14, &q); r.policy(a[3], &p); r.pointers(a[6], k_pruned, 11, &k);
    const int32_t* slo = (const int32_t*)r.ptr(a[4]);
    const int budget = (int)r.integer(a[5]);
    HS_DONE(hs_stratify_prune_budget(ctx, &t, &q, &p, slo, budget, &k, stream));
}
// (ctx, pruned, q, k_tree, v_tree, k_cache, v_cache, kv_off, batch, max_nodes, max_kv_len, layout, node_off | None,
//  sm_scale | None, out, lse | None, stream)
HS_NATIVE(tree_verify_attention) {
    if (!arity(n, 17)) return nullptr;
    Reader r;
    hs_pruned_tree k; hs_attn_desc d;
    r.pointers(a[1], k_pruned, 11, &k);
    d.batch = (int)r.integer(a[8]);
    d.max_rows = (int)r.size(a[2], o_zero);
    d.max_nodes = (int)r.integer(a[9]);
    d.kv_total = (int)r.size(a[5], o_zero);
    d.max_kv_len = (int)r.integer(a[10]);
    d.hq = (int)r.size(a[2], o_one);
    d.hkv = (int)r.size(a[3], o_one);
    d.head_dim = (int)r.size(a[2], o_two);
    d.layout = (int)r.integer(a[11]);
    d.node_off = (const int32_t*)r.ptr(a[12]);
    d.kv_off = (const int32_t*)r.ptr(a[7]);
    d.kv_token_stride = d.kv_total ? r.stride(a[5], o_zero) : (int64_t)d.hkv * d.head_dim;
    d.kv_head_stride = d.kv_total ? r.stride(a[5], o_one) : d.head_dim;
    if (a[13] == Py_None) {
        // 1 / sqrt(head_dim), the default (for the one supported head size a constant)
        d.sm_scale = d.head_dim == HS_HEAD_DIM ? 0.08838834764831845f : 1.f;
    } else {
        d.sm_scale = (float)r.real(a[13]);
    }
    const void *q = r.ptr(a[2]), *kt = r.ptr(a[3]), *vt = r.ptr(a[4]), *kc = r.ptr(a[5]), *vc = r.ptr(a[6]);
    void* out = r.ptr(a[14]);
    float* lse = (float*)r.ptr(a[15]);
    HS_DONE(hs_tree_verify_attention(ctx, &k, &d, q, kt, vt, kc, vc, out, lse, stream));
}
// (ctx, tree, pruned, target, target_layout, draft | None, mode, temperature, seed, offset, uniforms | None, accept, stream)
HS_NATIVE(accept_path) {
    if (!arity(n, 13)) return nullptr;
    Reader r;
    hs_tree_batch t; hs_pruned_tree k; hs_accept_out o;
    r.tree(a[1], &t); r.pointers(a[2], k_pruned, 11, &k); r.pointers(a[11], k_accept, 7, &o);
    o.path_cap = r.field_int(a[11], k_accept[7]);
    o.max_kept_rows = r.field_int(a[11], k_accept[8]);
    const void *x = r.ptr(a[3]), *q = r.ptr(a[5]);
    const hs_dtype dt = r.dtype(a[3]);
    const long long rs = r.stride(a[3], o_zero), v = r.size(a[3], o_one);
    const int layout = (int)r.integer(a[4]);
    const int32_t* mode = (const int32_t*)r.ptr(a[6]);
    const float *temp = (const float*)r.ptr(a[7]), *u = (const float*)r.ptr(a[10]);
    const uint64_t seed = (uint64_t)r.integer(a[8]), offset = (uint64_t)r.integer(a[9]);
    HS_DONE(hs_accept_path(ctx, &t, &k, x, layout, q, dt, rs, (int)v, mode, temp, seed, offset, u, &o, stream));
}
// (ctx, state, stream)
HS_NATIVE(expand_init) {
    if (!arity(n, 3)) return nullptr;
    Reader r;
    hs_expand_state s;
    r.expand(a[1], &s);
    HS_DONE(hs_expand_init(ctx, &s, stream));
}
// (ctx, state, topk_val, topk_idx, row_lse, stream)
HS_NATIVE(expand_level) {
    if (!arity(n, 6)) return nullptr;
    Reader r;
    hs_expand_state s;
    r.expand(a[1], &s);
    const float* tv = (const float*)r.ptr(a[2]);
    const int32_t* ti = (const int32_t*)r.ptr(a[3]);
    const float* lse = (const float*)r.ptr(a[4]);
    const int stride = (int)r.size(a[2], o_one);
    HS_DONE(hs_expand_level(ctx, &s, tv, ti, lse, stride, stream));
}
// (ctx, state, n_top | None, n_default, node_off, parent, token, cand_id, depth, stream)
HS_NATIVE(rerank) {
    if (!arity(n, 10)) return nullptr;
    Reader r;
    hs_expand_state s;
    r.expand(a[1], &s);
    const int32_t* top = (const int32_t*)r.ptr(a[2]);
    const int def = (int)r.integer(a[3]);
    int32_t* o[5];
    for (int i = 0; i < 5; ++i) o[i] = (int32_t*)r.ptr(a[4 + i]);
    HS_DONE(hs_rerank(ctx, &s, top, def, o[0], o[1], o[2], o[3], o[4], stream));
}

// (ctx, cache, k, v, row_off, len_out | None, stream)
HS_NATIVE(kv_append) {
    if (!arity(n, 7)) return nullptr;
    Reader r;
    hs_kv_cache c;
    r.cache(a[1], &c);
    const hs_dtype dt = r.dtype(a[2], "heads");
    long long rows = 0, heads = 0, dim = 0, rows2 = 0, heads2 = 0, dim2 = 0;
    int64_t ts = 0, hs = 0, ts2 = 0, hs2 = 0;
    const void* k = r.heads(a[2], false, dt, &rows, &heads, &dim, &ts, &hs);
    const void* v = r.heads(a[3], false, dt, &rows2, &heads2, &dim2, &ts2, &hs2);
    if (!r.bad && (rows != rows2 || heads != heads2 || dim != dim2 || ts != ts2 || hs != hs2)) r.fail("k and v have one shape and one stride");
    if (!r.bad && (heads != c.hkv || dim != c.head_dim || rows > 0x7fffffffll)) r.fail("k and v are [rows, hkv, head_dim] of the cache");
    const int32_t* off = (const int32_t*)r.list(a[4], c.batch + 1ll, k_offsets);
    int32_t* len = (int32_t*)r.list(a[5], c.batch, k_entries);
    HS_DONE_HERE(hs_kv_append(ctx, &c, k, v, dt, ts, hs, off, (int)rows, len, stream));
}
// (ctx, cache, pruned, accept, layout, node_off | None, k_tree, v_tree, len_out | None, stream)
HS_NATIVE(kv_append_path) {
    if (!arity(n, 10)) return nullptr;
    Reader r;
    hs_kv_cache c; hs_pruned_tree t; hs_accept_out o;
    const int layout = (int)r.integer(a[4]);
    r.cache(a[1], &c);
    r.some(a[2], k_pruned, 11, PRUNED_N_KEEP | PRUNED_KEEP_OFF | PRUNED_STATUS, &t);
    r.some(a[3], k_accept, 7, ACCEPT_LEN | ACCEPT_PATHS | ACCEPT_STATUS, &o);
    r.batch_of(a[2], k_pruned[10], c.batch, k_batch);
    r.batch_of(a[3], k_accept[6], c.batch, k_batch);
    o.path_cap = r.field_int(a[3], k_accept[7]);
    o.max_kept_rows = 0;                                             // (not read)
    const int32_t* node_off = (const int32_t*)r.list(a[5], c.batch + 1ll, k_offsets);
    long long rows = 0, heads = 0, dim = 0, rows2 = 0, heads2 = 0, dim2 = 0;
    int64_t ts, hs;
    const void* k = r.heads(a[6], true, HS_BF16, &rows, &heads, &dim, &ts, &hs);
    const void* v = r.heads(a[7], true, HS_BF16, &rows2, &heads2, &dim2, &ts, &hs);
    if (!r.bad && (rows != rows2 || heads != heads2 || dim != dim2 || heads != c.hkv || dim != c.head_dim)) r.fail("k_tree and v_tree are [rows, hkv, head_dim] of the cache");
    int32_t* len = (int32_t*)r.list(a[8], c.batch, k_entries);
    HS_DONE_HERE(hs_kv_append_path(ctx, &c, &t, &o, layout, node_off, k, v, (int)rows, len, stream));
}
// (ctx, cache, row_off, first | None, k_out, v_out, stream)
HS_NATIVE(kv_read) {
    if (!arity(n, 7)) return nullptr;
    Reader r;
    hs_kv_cache c;
    r.cache(a[1], &c);
    const int32_t *off = (const int32_t*)r.list(a[2], c.batch + 1ll, k_offsets), *first = (const int32_t*)r.list(a[3], c.batch, k_entries);
    const hs_dtype dt = r.dtype(a[4], "heads");
    long long rows = 0, heads = 0, dim = 0, rows2 = 0, heads2 = 0, dim2 = 0;
    int64_t ts = 0, hs = 0, ts2 = 0, hs2 = 0;
    void* k = r.heads(a[4], false, dt, &rows, &heads, &dim, &ts, &hs);
    void* v = r.heads(a[5], false, dt, &rows2, &heads2, &dim2, &ts2, &hs2);
    if (!r.bad && (rows != rows2 || heads != heads2 || dim != dim2 || ts != ts2 || hs != hs2)) r.fail("k_out and v_out have one shape and one stride");
    if (!r.bad && (heads != c.hkv || dim != c.head_dim || rows > 0x7fffffffll)) r.fail("k_out and v_out are [rows, hkv, head_dim] of the cache");
    HS_DONE_HERE(hs_kv_read(ctx, &c, off, first, (int)rows, k, v, dt, ts, hs, stream));
}
// (ctx, pruned, cache, q, k_tree, v_tree, max_nodes, max_kv_len, layout, node_off | None, sm_scale | None, out, lse | None, stream)
HS_NATIVE(tree_verify_attention_paged) {
    if (!arity(n, 14)) return nullptr;
    Reader r;
    hs_pruned_tree t; hs_kv_cache c; hs_paged_attn_desc d;
    r.some(a[1], k_pruned, 11, PRUNED_N_KEEP | PRUNED_KEEP_OFF | PRUNED_KEEP_IDX | PRUNED_ANC_MASK | PRUNED_STATUS, &t);
    r.cache(a[2], &c);
    r.batch_of(a[1], k_pruned[10], c.batch, k_batch);
    long long rows[4] = {0, 0, 0, 0}, heads[4] = {0, 0, 0, 0}, dim[4] = {0, 0, 0, 0};
    int64_t ts, hs;
    const int at[4] = {3, 4, 5, 11};
    void* x[4];
    for (int i = 0; i < 4; ++i) x[i] = r.heads(a[at[i]], true, HS_BF16, &rows[i], &heads[i], &dim[i], &ts, &hs);
    if (!r.bad && (heads[1] != c.hkv || heads[2] != c.hkv || heads[3] != heads[0] || rows[3] != rows[0] || rows[1] != rows[0] || rows[2] != rows[0] ||
                   dim[0] != c.head_dim || dim[1] != c.head_dim || dim[2] != c.head_dim || dim[3] != c.head_dim))
        r.fail("q and out are [rows, hq, head_dim], k_tree and v_tree [rows, hkv, head_dim]");
    d.max_rows = (int)rows[0];
    d.max_nodes = (int)r.integer(a[6]);
    d.max_kv_len = (int)r.integer(a[7]);
    d.hq = (int)heads[0];
    d.layout = (int)r.integer(a[8]);
    d.node_off = (const int32_t*)r.list(a[9], c.batch + 1ll, k_offsets);
    d.sm_scale = a[10] == Py_None ? 0.08838834764831845f : (float)r.real(a[10]);      // 1 / sqrt(128)
    float* lse = (float*)r.list(a[12], rows[0] * heads[0], "lse_out is [rows, hq]", t_f32);
    if (lse && r.size(a[12], o_one) != heads[0] && !r.bad) r.fail("lse_out is [rows, hq]");
    HS_DONE_HERE(hs_tree_verify_attention_paged(ctx, &t, &c, &d, x[0], x[1], x[2], x[3], lse, stream));
}
// q or k with its output, as hs_heads
void head_pair(Reader& r, PyObject* in, PyObject* out, hs_dtype dt, hs_heads* x, long long* rows, long long* dim) {
    long long heads = 0, rows2 = 0, heads2 = 0, dim2 = 0;
    x->in = r.heads(in, false, dt, rows, &heads, dim, &x->in_token_stride, &x->in_head_stride);
    x->out = r.heads(out, false, dt, &rows2, &heads2, &dim2, &x->out_token_stride, &x->out_head_stride);
    if (!r.bad && (*rows != rows2 || heads != heads2 || *dim != dim2)) r.fail("an output has the shape of its input");
    x->heads = (int)heads;
}
// (ctx, rope, pos, q, q_out, k | None, k_out | None, stream)
HS_NATIVE(rotary) {
    if (!arity(n, 8)) return nullptr;
    Reader r;
    const hs_rope* rope = r.rope(a[1]);
    const hs_dtype dt = r.dtype(a[3], "heads");
    hs_heads q = {}, k = {};
    long long rows = 0, dim = 0, rows2 = 0, dim2 = 0;
    head_pair(r, a[3], a[4], dt, &q, &rows, &dim);
    const bool with_k = a[5] != Py_None;
    if (with_k) {
        head_pair(r, a[5], a[6], dt, &k, &rows2, &dim2);
        if (!r.bad && (rows2 != rows || dim2 != dim)) r.fail("k has the rows and the head size of q");
    }
    const int32_t* pos = (const int32_t*)r.list(a[2], rows, "one position for each row");
    if (!r.bad && rows > 0x7fffffffll) r.fail("one position for each row");
    if (!r.bad && dim != rope->head_dim) r.fail("the head size is not the one of the frequencies");
    HS_DONE_HERE(hs_rotary(ctx, rope, pos, (int)rows, &q, with_k ? &k : nullptr, dt, stream));
}
// (ctx, rope, pruned, kv_len, max_nodes, layout, node_off | None, q, q_out, k | None, k_out | None, stream)
HS_NATIVE(rotary_tree) {
    if (!arity(n, 12)) return nullptr;
    Reader r;
    const hs_rope* rope = r.rope(a[1]);
    hs_pruned_tree t;
    r.some(a[2], k_pruned, 11, PRUNED_N_KEEP | PRUNED_KEEP_OFF | PRUNED_KEEP_IDX | PRUNED_NEW_DEPTH | PRUNED_STATUS, &t);
    const long long batch = r.numel(a[3]);
    const int32_t* kv_len = (const int32_t*)r.list(a[3], batch, k_entries);
    r.batch_of(a[2], k_pruned[10], batch, k_batch);
    const int max_nodes = (int)r.integer(a[4]), layout = (int)r.integer(a[5]);
    const int32_t* node_off = (const int32_t*)r.list(a[6], batch + 1, k_offsets);
    const hs_dtype dt = r.dtype(a[7], "heads");
    hs_heads q = {}, k = {};
    long long rows = 0, dim = 0, rows2 = 0, dim2 = 0;
    head_pair(r, a[7], a[8], dt, &q, &rows, &dim);
    const bool with_k = a[9] != Py_None;
    if (with_k) {
        head_pair(r, a[9], a[10], dt, &k, &rows2, &dim2);
        if (!r.bad && (rows2 != rows || dim2 != dim)) r.fail("k has the rows and the head size of q");
    }
    if (!r.bad && dim != rope->head_dim) r.fail("the head size is not the one of the frequencies");
    HS_DONE_HERE(hs_rotary_tree(ctx, rope, &t, kv_len, (int)batch, max_nodes, (int)rows, layout, node_off, &q, with_k ? &k : nullptr, dt, stream));
}

// setup(torch.float32, torch.bfloat16, torch.int32)
HS_NATIVE(setup) {
    if (!arity(n, 3)) return nullptr;
    t_f32 = Py_NewRef(a[0]);
    t_bf16 = Py_NewRef(a[1]);
    t_i32 = Py_NewRef(a[2]);
    Py_RETURN_NONE;
}

#define HS_METHOD(f) {#f, (PyCFunction)(void (*)(void))f, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {HS_METHOD(setup), HS_METHOD(entropy_quantify), HS_METHOD(entropy_quantify_prune),
                         HS_METHOD(stratify_prune), HS_METHOD(stratify_prune_budget), HS_METHOD(tree_verify_attention),
                         HS_METHOD(accept_path), HS_METHOD(expand_init), HS_METHOD(expand_level), HS_METHOD(rerank),
                         HS_METHOD(kv_append), HS_METHOD(kv_append_path), HS_METHOD(kv_read),
                         HS_METHOD(tree_verify_attention_paged), HS_METHOD(rotary), HS_METHOD(rotary_tree),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) {
    n_data_ptr = PyUnicode_InternFromString("data_ptr");
    n_contiguous = PyUnicode_InternFromString("is_contiguous");
    n_get_device = PyUnicode_InternFromString("get_device");
    n_numel = PyUnicode_InternFromString("numel");
    n_stride = PyUnicode_InternFromString("stride");
    n_size = PyUnicode_InternFromString("size");
    n_dtype = PyUnicode_InternFromString("dtype");
    o_zero = PyLong_FromLong(0);
    o_one = PyLong_FromLong(1);
    o_two = PyLong_FromLong(2);
    if (!n_data_ptr || !n_contiguous || !n_get_device || !n_numel || !n_stride || !n_size || !n_dtype || !o_zero || !o_one || !o_two ||
        !intern_all(k_tree, 5) || !intern_all(k_quant, 14) || !intern_all(k_pruned, 11) || !intern_all(k_accept, 9) ||
        !intern_all(k_expand, 12) || !intern_all(k_policy, 9) || !intern_all(k_cache, 13) || !intern_all(k_rope, 1))
        return nullptr;
    return PyModule_Create(&module);
}
