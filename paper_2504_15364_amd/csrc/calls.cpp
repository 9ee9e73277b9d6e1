// Python's side of norm_rope, branch_append, branch_attention and of the calls that go with them: checks of the tensors, allocation of what the caller does not give, and the
// call of the C ABI (include/keydiff.h), whose entry points the package hands over once (`bind`).  No arithmetic lives here.  A function returns
// its tensors, or the error code of the C ABI as a number.
//
// A generation step makes such calls for every layer, and its kernels take 3 to 15 us.  Calls in a row, host time of each: norm_rope 5.7 us,
// branch_append 4.1, branch_attention (two launches) 9.2; marshalled in Python through ctypes 11.3, 11.5 and 14.9.  The functions take all arguments by position; their defaults and documentation are binding.py's.
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ops/empty.h>
#include <c10/core/DeviceGuard.h>

#include <stdexcept>
#include <string>
#include <type_traits>

#include "../../include/keydiff.h"

namespace {

decltype(&keydiff_norm_rope) norm_rope_abi;
decltype(&keydiff_branch_append) append_abi;
decltype(&keydiff_branch_workspace_bytes) workspace_abi;
decltype(&keydiff_branch_attention) attention_abi;
decltype(&keydiff_cache_branch_attention) cache_attention_abi;
decltype(&keydiff_branch_chunk_workspace_bytes) chunk_workspace_abi;
decltype(&keydiff_branch_chunk_attention) chunk_abi;
decltype(&keydiff_cache_branch_chunk_attention) cache_chunk_abi;
decltype(&keydiff_branch_weights_workspace_bytes) weights_workspace_abi;
decltype(&keydiff_branch_weights) weights_abi;
decltype(&keydiff_branch_evict_workspace_bytes) evict_workspace_abi;
decltype(&keydiff_branch_evict) evict_abi;
PyObject *current_stream;   // torch's function: device index -> handle of the current stream

struct Refused : std::runtime_error {   // becomes a ValueError
    using std::runtime_error::runtime_error;
};

std::string shape_of(at::IntArrayRef s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + (s.size() == 1 ? ",)" : ")");
}
std::string what_is(const at::Tensor &t) { return shape_of(t.sizes()) + " " + c10::toString(t.scalar_type()) + ", strides " + shape_of(t.strides()); }

const at::Tensor &tensor_of(PyObject *o, const char *name)
{
    if (!THPVariable_Check(o)) throw Refused(std::string(name) + " must be a tensor");
    return THPVariable_Unpack(o);
}

// Four dimensions, whose sizes the C ABI takes as int32
void four(const char *name, const at::Tensor &t)
{
    if (t.dim() != 4) throw Refused(std::string(name) + " must have four dimensions, got " + what_is(t));
    for (const int64_t s : t.sizes())
        if (s > INT32_MAX) throw Refused(std::string(name) + " is too large: " + what_is(t));
}

// Checks against the first tensor's device
struct Checked {
    c10::Device device;

    void here(const char *name, const at::Tensor &t) const
    {
        if (t.device() != device)
            throw Refused("the tensors must live on one device, got " + device.str() + " and " + t.device().str() + " for " + name);
    }
    // rows [n][heads][tokens][d]: bf16, the innermost dimension contiguous, other strides free
    keydiff_rows_t rows(const char *name, const at::Tensor &t, int64_t n, int64_t heads, int64_t tokens, int64_t d) const
    {
        if (t.scalar_type() != at::kBFloat16 || t.sizes() != at::IntArrayRef({n, heads, tokens, d}) || t.stride(3) != 1)
            throw Refused(std::string(name) + " must be a bf16 tensor of shape " + shape_of({n, heads, tokens, d}) +
                          " with a contiguous last dimension, got " + what_is(t));
        here(name, t);
        return {t.data_ptr(), n > 1 ? t.stride(0) : 0, heads > 1 ? t.stride(1) : 0, tokens > 1 ? t.stride(2) : 0};
    }
    // a contiguous tensor of this shape and type
    void *dense(const char *name, const at::Tensor &t, at::IntArrayRef shape, at::ScalarType type) const
    {
        if (t.scalar_type() != type || t.sizes() != shape || !t.is_contiguous())
            throw Refused(std::string(name) + " must be a contiguous " + c10::toString(type) + " tensor of shape " + shape_of(shape) + ", got " + what_is(t));
        here(name, t);
        return t.data_ptr();
    }
    void *dense_or_null(const char *name, PyObject *o, at::IntArrayRef shape, at::ScalarType type) const
    {
        return o == Py_None ? nullptr : dense(name, tensor_of(o, name), shape, type);
    }
    void weight(const char *name, PyObject *o, int64_t heads, int64_t d, const void **at, int64_t *stride) const
    {
        const at::Tensor &w = tensor_of(o, name);
        const bool one = w.dim() == 1;
        if (w.scalar_type() != at::kBFloat16 || (one ? w.sizes() != at::IntArrayRef({d}) : w.sizes() != at::IntArrayRef({heads, d})) ||
            w.stride(-1) != 1)
            throw Refused(std::string(name) + " must be a bf16 tensor of shape " + shape_of({d}) + " or " + shape_of({heads, d}) + ", got " + what_is(w));
        here(name, w);
        *at = w.data_ptr();
        *stride = one || heads == 1 ? 0 : w.stride(0);
    }
    keydiff_row_form_t form(int64_t hq, int64_t hkv, int64_t d, PyObject *cos, PyObject *sin, PyObject *q_weight, PyObject *k_weight,
                            PyObject *eps) const
    {
        keydiff_row_form_t f{};
        f.norm_eps = (float)PyFloat_AsDouble(eps);
        if (PyErr_Occurred()) throw python_error();
        if ((q_weight == Py_None) != (k_weight == Py_None)) throw Refused("q_weight and k_weight are given together or not at all");
        if ((cos == Py_None) != (sin == Py_None)) throw Refused("cos and sin are given together or not at all");
        if (q_weight != Py_None) {
            weight("q_weight", q_weight, hq, d, &f.q_weight, &f.q_weight_stride);
            weight("k_weight", k_weight, hkv, d, &f.k_weight, &f.k_weight_stride);
        }
        if (cos != Py_None) {
            const at::Tensor &c = tensor_of(cos, "cos");
            f.table_rows = c.dim() == 2 ? c.size(0) : 0;
            f.cos_table = static_cast<const float *>(dense("cos", c, {f.table_rows, d / 2}, at::kFloat));
            f.sin_table = static_cast<const float *>(dense("sin", tensor_of(sin, "sin"), {f.table_rows, d / 2}, at::kFloat));
        }
        return f;
    }
    keydiff_branches_t branches(int64_t n, int64_t hq, int64_t hkv, int64_t d, PyObject *k_pages, PyObject *v_pages, PyObject *table_, PyObject *lens,
                                PyObject *n_new) const
    {
        const at::Tensor &pages = tensor_of(k_pages, "k_pages"), &table = tensor_of(table_, "table");
        if (pages.dim() != 4 || pages.size(1) != hkv || pages.size(3) != d)
            throw Refused("k_pages must be [pages][" + std::to_string(hkv) + "][page_rows][" + std::to_string(d) + "], got " + what_is(pages));
        if (table.dim() != 2) throw Refused("table must be [" + std::to_string(n) + "][width], got " + what_is(table));
        four("k_pages", pages);
        if (table.size(1) > INT32_MAX) throw Refused("table is too large: " + what_is(table));
        keydiff_branches_t b{};
        b.k_pages = dense("k_pages", pages, pages.sizes(), at::kBFloat16);
        if (v_pages) b.v_pages = dense("v_pages", tensor_of(v_pages, "v_pages"), pages.sizes(), at::kBFloat16);
        b.table = static_cast<const int32_t *>(dense("table", table, {n, table.size(1)}, at::kInt));
        b.lens = static_cast<const int32_t *>(dense("lens", tensor_of(lens, "lens"), {n}, at::kInt));
        b.n_new = static_cast<const int32_t *>(dense_or_null("n_new", n_new, {n}, at::kInt));
        b.n_seqs = (int32_t)n;
        b.n_q_heads = (int32_t)hq;
        b.n_kv_heads = (int32_t)hkv;
        b.head_dim = (int32_t)d;
        b.page_rows = (int32_t)pages.size(2);
        b.n_pages = (int32_t)pages.size(0);
        b.table_width = (int32_t)table.size(1);
        return b;
    }
    void on_gpu() const
    {
        if (device.type() != c10::DeviceType::CUDA) throw Refused("the tensors must live on a GPU, got " + device.str());
    }
    void *stream() const
    {
        PyObject *index = PyLong_FromLong(device.index());
        PyObject *r = index ? PyObject_CallOneArg(current_stream, index) : nullptr;
        Py_XDECREF(index);
        if (!r) throw python_error();
        void *s = PyLong_AsVoidPtr(r);
        Py_DECREF(r);
        if (!s && PyErr_Occurred()) throw python_error();
        return s;
    }
};

int64_t whole(PyObject *o)
{
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw python_error();
    return v;
}

void arguments(Py_ssize_t got, Py_ssize_t want)
{
    if (got != want) throw Refused("takes " + std::to_string(want) + " arguments, got " + std::to_string(got));
}

// A tensor that the caller gave, or a new one
PyObject *given_or(PyObject *o, at::Tensor &made)
{
    if (o == Py_None) return THPVariable_Wrap(std::move(made));
    Py_INCREF(o);
    return o;
}

#define KD_TRY HANDLE_TH_ERRORS try {
#define KD_END                                            \
    }                                                     \
    catch (const Refused &e)                              \
    {                                                     \
        PyErr_SetString(PyExc_ValueError, e.what());      \
        return nullptr;                                   \
    }                                                     \
    END_HANDLE_TH_ERRORS

// q, k, cos, sin, pos0, positions, q_weight, k_weight, norm_eps, q_out, k_out, status
PyObject *norm_rope(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    KD_TRY
    arguments(n, 12);
    const at::Tensor &q = tensor_of(a[0], "q"), &k = tensor_of(a[1], "k");
    four("q", q);
    four("k", k);
    const int64_t b = q.size(0), hq = q.size(1), T = q.size(2), d = q.size(3), hkv = k.size(1);
    const Checked on{q.device()};
    const keydiff_rows_t rq = on.rows("q", q, b, hq, T, d), rk = on.rows("k", k, b, hkv, T, d);
    const int32_t *positions = static_cast<const int32_t *>(on.dense_or_null("positions", a[5], {b, T}, at::kInt));
    keydiff_row_form_t form = on.form(hq, hkv, d, a[2], a[3], a[6], a[7], a[8]);
    form.status = static_cast<int32_t *>(on.dense_or_null("status", a[11], {1}, at::kInt));
    void *q_out = on.dense_or_null("q_out", a[9], {b, hq, T, d}, at::kBFloat16), *k_out = on.dense_or_null("k_out", a[10], {b, hkv, T, d}, at::kBFloat16);
    const int64_t pos0 = whole(a[4]);
    on.on_gpu();
    const c10::DeviceGuard guard(on.device);
    at::Tensor q_new, k_new;
    if (!q_out) q_out = (q_new = at::empty({b, hq, T, d}, q.options())).data_ptr();
    if (!k_out) k_out = (k_new = at::empty({b, hkv, T, d}, q.options())).data_ptr();
    const int rc = norm_rope_abi(&rq, &rk, (int32_t)b, (int32_t)hq, (int32_t)hkv, (int32_t)d, (int32_t)T, pos0, positions, &form, q_out, k_out,
                                 on.stream());
    if (rc != KEYDIFF_OK) return PyLong_FromLong(rc);
    PyObject *x = given_or(a[9], q_new), *y = given_or(a[10], k_new), *both = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return both;
    KD_END
}

// q, k_new, v_new, k_pages, v_pages, table, lens, n_new, pos0, cos, sin, q_weight, k_weight, norm_eps, q_out, status
PyObject *branch_append(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    KD_TRY
    arguments(n_args, 16);
    const at::Tensor &k = tensor_of(a[1], "k_new"), &v = tensor_of(a[2], "v_new");
    four("k_new", k);
    const int64_t n = k.size(0), hkv = k.size(1), Bt = k.size(2), d = k.size(3);
    int64_t hq = hkv;
    const Checked on{k.device()};
    keydiff_rows_t rq{};
    const keydiff_rows_t rk = on.rows("k_new", k, n, hkv, Bt, d), rv = on.rows("v_new", v, n, hkv, Bt, d);
    void *q_out = nullptr;
    if (a[0] != Py_None) {
        const at::Tensor &q = tensor_of(a[0], "q");
        four("q", q);
        hq = q.size(1);
        rq = on.rows("q", q, n, hq, Bt, d);
        q_out = on.dense_or_null("q_out", a[14], {n, hq, Bt, d}, at::kBFloat16);
    } else if (a[14] != Py_None) {
        throw Refused("q_out without q");
    }
    const keydiff_branches_t b = on.branches(n, hq, hkv, d, a[3], a[4], a[5], a[6], a[7]);
    const int32_t *pos0 = static_cast<const int32_t *>(on.dense_or_null("pos0", a[8], {n}, at::kInt));
    keydiff_row_form_t form = on.form(hq, hkv, d, a[9], a[10], a[11], a[12], a[13]);
    form.status = static_cast<int32_t *>(on.dense_or_null("status", a[15], {1}, at::kInt));
    on.on_gpu();
    const c10::DeviceGuard guard(on.device);
    at::Tensor q_new;
    if (rq.data && !q_out) q_out = (q_new = at::empty({n, hq, Bt, d}, k.options())).data_ptr();
    const int rc = append_abi(&b, rq.data ? &rq : nullptr, &rk, &rv, (int32_t)Bt, pos0, &form, q_out, on.stream());
    if (rc != KEYDIFF_OK) return PyLong_FromLong(rc);
    if (!rq.data) Py_RETURN_NONE;
    return given_or(a[14], q_new);
    KD_END
}

// The rows that sequences share: those of a cache (its handle and batch), or tensors
struct Prefix {
    bool cached;
    const void *k = nullptr, *v = nullptr;
    int64_t prompts, rows = 0, cap = 0;

    // a: handle (None: no cache), batch, keys and values (None: no rows), rows
    Prefix(const Checked &on, PyObject *const *a, int64_t hkv, int64_t d) : cached(a[0] != Py_None), prompts(cached ? whole(a[1]) : 0)
    {
        if (a[2] == Py_None) return;
        const at::Tensor &keys = tensor_of(a[2], "prefix keys");
        four("prefix keys", keys);
        prompts = keys.size(0);
        cap = keys.size(2);
        rows = whole(a[4]);
        if (rows < 0 || rows > cap) throw Refused("the prefix has " + std::to_string(cap) + " rows a head, " + std::to_string(rows) + " are to be read");
        k = on.dense("prefix keys", keys, {prompts, hkv, cap, d}, at::kBFloat16);
        v = on.dense("prefix values", tensor_of(a[3], "prefix values"), {prompts, hkv, cap, d}, at::kBFloat16);
    }
};

double number(PyObject *o)
{
    const double x = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) throw python_error();
    return x;
}

int32_t small(const char *name, PyObject *o)
{
    const int64_t v = whole(o);
    if (v < INT32_MIN || v > INT32_MAX) throw Refused(std::string(name) + " is too large: " + std::to_string(v));
    return (int32_t)v;
}

// The caller's workspace, or a new one
at::Tensor workspace_of(const Checked &on, PyObject *o, size_t need, const at::Tensor &like)
{
    if (o == Py_None) return at::empty({(int64_t)need}, like.options().dtype(at::kByte));
    const at::Tensor &work = tensor_of(o, "workspace");
    if (work.scalar_type() != at::kByte || !work.is_contiguous() || (size_t)work.numel() < need || work.device() != on.device)
        throw Refused("workspace must be a contiguous uint8 tensor of at least " + std::to_string(need) + " elements on " + on.device.str());
    return work;
}

// q, k_pages, v_pages, table, lens, n_new, the handle of the prefix's cache (None: no cache), its batch, prefix keys and values (None: no rows), rows,
// softmax_scale, out, workspace; chunk: and lse
PyObject *attention(PyObject *const *a, bool chunk)
{
    const at::Tensor &q = tensor_of(a[0], "q"), &pages = tensor_of(a[1], "k_pages");
    four("q", q);
    four("k_pages", pages);
    const int64_t n = q.size(0), hq = q.size(1), Bt = q.size(2), d = q.size(3), hkv = pages.size(1);
    const Checked on{q.device()};
    const keydiff_rows_t rq = on.rows("q", q, n, hq, Bt, d);
    const keydiff_branches_t b = on.branches(n, hq, hkv, d, a[1], a[2], a[3], a[4], a[5]);
    void *out = on.dense_or_null("out", a[12], {n, hq, Bt, d}, at::kBFloat16);
    float *lse = chunk ? static_cast<float *>(on.dense_or_null("lse", a[14], {n, hq, Bt}, at::kFloat)) : nullptr;
    const Prefix prefix(on, a + 6, hkv, d);
    const double scale = number(a[11]);
    if (prefix.cached && !(scale <= 0)) throw Refused("softmax_scale is the cache's");
    on.on_gpu();
    const c10::DeviceGuard guard(on.device);
    size_t need = 0;
    if (const int rc = (chunk ? chunk_workspace_abi : workspace_abi)(&b, (int32_t)Bt, (int32_t)prefix.prompts, &need)) return PyLong_FromLong(rc);
    const at::Tensor work = workspace_of(on, a[13], need, q);
    at::Tensor made, made_lse;
    if (!out) out = (made = at::empty({n, hq, Bt, d}, q.options())).data_ptr();
    if (chunk && !lse) lse = static_cast<float *>((made_lse = at::empty({n, hq, Bt}, q.options().dtype(at::kFloat))).data_ptr());
    void *stream = on.stream(), *ws = work.data_ptr();
    const size_t bytes = (size_t)work.numel();
    keydiff_cache_t *cache = prefix.cached ? static_cast<keydiff_cache_t *>(PyLong_AsVoidPtr(a[6])) : nullptr;
    const int32_t T = (int32_t)Bt, prompts = (int32_t)prefix.prompts, rows = (int32_t)prefix.rows;
    int rc;
    if (chunk)
        rc = prefix.cached ? cache_chunk_abi(cache, &b, &rq, T, out, lse, ws, bytes, stream)
                           : chunk_abi(&b, &rq, T, prefix.k, prefix.v, prompts, rows, prefix.cap, (float)scale, out, lse, ws, bytes, stream);
    else
        rc = prefix.cached ? cache_attention_abi(cache, &b, &rq, T, out, ws, bytes, stream)
                           : attention_abi(&b, &rq, T, prefix.k, prefix.v, prompts, rows, prefix.cap, (float)scale, out, ws, bytes, stream);
    if (rc != KEYDIFF_OK) return PyLong_FromLong(rc);
    if (!chunk) return given_or(a[12], made);
    PyObject *x = given_or(a[12], made), *y = given_or(a[14], made_lse), *both = x && y ? PyTuple_Pack(2, x, y) : nullptr;
    Py_XDECREF(x);
    Py_XDECREF(y);
    return both;
}

PyObject *branch_attention(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    KD_TRY
    arguments(n_args, 14);
    return attention(a, false);
    KD_END
}

PyObject *branch_chunk_attention(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    KD_TRY
    arguments(n_args, 15);
    return attention(a, true);
    KD_END
}

// q, k_pages, w_pages, table, lens, lse, n_new, observe, decay, softmax_scale, workspace
PyObject *branch_weights(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    KD_TRY
    arguments(n_args, 11);
    const at::Tensor &q = tensor_of(a[0], "q"), &pages = tensor_of(a[1], "k_pages");
    four("q", q);
    four("k_pages", pages);
    const int64_t n = q.size(0), hq = q.size(1), Bt = q.size(2), d = q.size(3), hkv = pages.size(1);
    const Checked on{q.device()};
    const keydiff_rows_t rq = on.rows("q", q, n, hq, Bt, d);
    const keydiff_branches_t b = on.branches(n, hq, hkv, d, a[1], nullptr, a[3], a[4], a[6]);
    float *w = static_cast<float *>(on.dense("w_pages", tensor_of(a[2], "w_pages"), {pages.size(0), hkv, pages.size(2)}, at::kFloat));
    const float *lse = static_cast<const float *>(on.dense("lse", tensor_of(a[5], "lse"), {n, hq, Bt}, at::kFloat));
    const int32_t observe = small("observe", a[7]);
    const double decay = number(a[8]), scale = number(a[9]);
    on.on_gpu();
    const c10::DeviceGuard guard(on.device);
    size_t need = 0;
    if (const int rc = weights_workspace_abi(&b, (int32_t)Bt, observe, &need)) return PyLong_FromLong(rc);
    const at::Tensor work = workspace_of(on, a[10], need, q);
    return PyLong_FromLong(weights_abi(&b, &rq, (int32_t)Bt, lse, w, observe, (float)decay, (float)scale, work.data_ptr(), (size_t)work.numel(), on.stream()));
    KD_END
}

// k_pages, v_pages, w_pages, p_pages, table, lens, budget, Bt, n_new, pos0, window, status, workspace
PyObject *branch_evict(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    KD_TRY
    arguments(n_args, 13);
    const at::Tensor &pages = tensor_of(a[0], "k_pages"), &table = tensor_of(a[4], "table");
    four("k_pages", pages);
    if (table.dim() != 2) throw Refused("table must be [sequences][width], got " + what_is(table));
    if (table.size(0) > INT32_MAX) throw Refused("table is too large: " + what_is(table));
    const int64_t n = table.size(0), hkv = pages.size(1);
    const Checked on{pages.device()};
    const keydiff_branches_t b = on.branches(n, hkv, hkv, pages.size(3), a[0], a[1], a[4], a[5], a[8]);
    float *w = static_cast<float *>(on.dense("w_pages", tensor_of(a[2], "w_pages"), {pages.size(0), hkv, pages.size(2)}, at::kFloat));
    int32_t *positions = static_cast<int32_t *>(on.dense("p_pages", tensor_of(a[3], "p_pages"), {pages.size(0), hkv, pages.size(2)}, at::kInt));
    const int32_t budget = small("budget", a[6]), Bt = small("Bt", a[7]), window = small("window", a[10]);
    const int32_t *pos0 = static_cast<const int32_t *>(on.dense_or_null("pos0", a[9], {n}, at::kInt));
    int32_t *status = static_cast<int32_t *>(on.dense_or_null("status", a[11], {1}, at::kInt));
    on.on_gpu();
    const c10::DeviceGuard guard(on.device);
    size_t need = 0;
    if (const int rc = evict_workspace_abi(&b, budget, &need)) return PyLong_FromLong(rc);
    const at::Tensor work = workspace_of(on, a[12], need, pages);
    return PyLong_FromLong(evict_abi(&b, Bt, w, positions, pos0, budget, window, status, work.data_ptr(), (size_t)work.numel(), on.stream()));
    KD_END
}

// Addresses of the entry points in the order of their declaration above; torch's current-stream function
PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    KD_TRY
    arguments(n, 13);
    int i = 0;
    auto take = [&](auto &f) { f = reinterpret_cast<std::decay_t<decltype(f)>>(PyLong_AsVoidPtr(a[i++])); };
    take(norm_rope_abi);
    take(append_abi);
    take(workspace_abi);
    take(attention_abi);
    take(cache_attention_abi);
    take(chunk_workspace_abi);
    take(chunk_abi);
    take(cache_chunk_abi);
    take(weights_workspace_abi);
    take(weights_abi);
    take(evict_workspace_abi);
    take(evict_abi);
    if (PyErr_Occurred()) throw python_error();
    Py_INCREF(a[i]);
    Py_XDECREF(current_stream);
    current_stream = a[i];
    Py_RETURN_NONE;
    KD_END
}

// hq, hkv, d, cos, sin, q_weight, k_weight, norm_eps and a tensor on their device: the bytes of a keydiff_row_form_t
PyObject *row_form(PyObject *, PyObject *const *a, Py_ssize_t n)
{
    KD_TRY
    arguments(n, 9);
    const Checked on{tensor_of(a[8], "like").device()};
    const keydiff_row_form_t form = on.form(whole(a[0]), whole(a[1]), whole(a[2]), a[3], a[4], a[5], a[6], a[7]);
    return PyBytes_FromStringAndSize(reinterpret_cast<const char *>(&form), sizeof form);
    KD_END
}

#define KD_METHOD(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {KD_METHOD(bind), KD_METHOD(row_form), KD_METHOD(norm_rope), KD_METHOD(branch_append),
                         KD_METHOD(branch_attention),
                         KD_METHOD(branch_chunk_attention), KD_METHOD(branch_weights), KD_METHOD(branch_evict), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&module); }
