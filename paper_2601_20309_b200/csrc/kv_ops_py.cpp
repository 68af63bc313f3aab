// Python entry of the operators on the device cache: checks of tensors and argument marshalling, nothing else.  A decode step
// calls these a few times per layer; read through Python attributes, a call's dozen tensors took 13 to 30 us, several
// times what the kernels of a small call need.
#include <Python.h>
#include <ATen/core/grad_mode.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <string>

#include "../../include/duplexkv.h"

namespace {

struct Bad {
    std::string what;
};

const char *name_of(at::ScalarType t)
{
    return t == at::kBFloat16 ? "bf16" : t == at::kHalf ? "f16" : t == at::kInt ? "int32" : t == at::kFloat ? "float32" : c10::toString(t);
}

struct Call {
    int device;
    const kv_cache_t *cache;

    at::ScalarType type() const { return cache->dtype == KV_DT_F16 || cache->dtype == KV_DT_F16_Q4 ? at::kHalf : at::kBFloat16; }

    // address and outer strides of a tensor whose last dimension is contiguous; -1 in `shape`: any size
    const at::Tensor &rows(PyObject *o, at::ScalarType want, std::initializer_list<int64_t> shape, const char *what, const void **p, int64_t *strides) const
    {
        if (!THPVariable_Check(o)) throw Bad{std::string(what) + " must be a tensor"};
        const at::Tensor &t = THPVariable_Unpack(o);
        if (t.scalar_type() != want) throw Bad{std::string(what) + " must be " + name_of(want) + ", not " + name_of(t.scalar_type())};
        if (t.requires_grad() && at::GradMode::is_enabled())
            throw Bad{std::string(what) + " requires grad, and the operators have no backward pass: call them under torch.no_grad()"};
        if (!t.is_cuda() || t.get_device() != device) throw Bad{std::string(what) + " must be on cuda:" + std::to_string(device)};
        const auto have = t.sizes(), st = t.strides();
        bool ok = have.size() == shape.size();
        size_t d = 0;
        for (int64_t want_d : shape) {
            if (!ok) break;
            ok = want_d < 0 || have[d] == want_d;
            ++d;
        }
        if (!ok) {
            std::string text = std::string(what) + " must have shape (";
            for (int64_t w : shape) text += (w < 0 ? std::string("any") : std::to_string(w)) + ", ";
            text += "), not (";
            for (int64_t h : have) text += std::to_string(h) + ", ";
            throw Bad{text + ")"};
        }
        if (st.back() != 1 && have.back() > 1) throw Bad{std::string(what) + ": the last dimension must be contiguous"};
        *p = t.data_ptr();
        for (size_t k = 0; strides && k + 1 < st.size(); ++k) strides[k] = have[k] > 1 ? st[k] : 0;      // nothing steps along a dimension of size 1
        return t;
    }
    const at::Tensor &slots(PyObject *o, at::ScalarType want, std::initializer_list<int64_t> shape, int64_t least, const char *what, const void **p, int64_t *strides) const
    {
        const at::Tensor &t = rows(o, want, shape, what, p, strides);
        if (t.sizes().back() < least) throw Bad{std::string(what) + " needs " + std::to_string(least) + " slots"};
        return t;
    }
    template <typename Args> void tables(Args &a, PyObject *block_tables, PyObject *lens, int64_t n) const
    {
        const at::Tensor &t = rows(block_tables, at::kInt, {n, -1}, "block_tables", (const void **)&a.block_tables, &a.table_stride);
        a.table_width = (int32_t)std::min<int64_t>(t.size(1), INT32_MAX);
        rows(lens, at::kInt, {n}, "lens", (const void **)&a.lens, nullptr);
    }
};

int64_t size_of(PyObject *o, int d, const char *what)
{
    if (!THPVariable_Check(o)) throw Bad{std::string(what) + " must be a tensor"};
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.dim() <= d) throw Bad{std::string(what) + " has too few dimensions"};
    return t.size(d);
}

int64_t integer(PyObject *o)
{
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Bad{""};
    return v;
}
int32_t integer32(PyObject *o)
{
    const int64_t v = integer(o);
    if (v < INT32_MIN || v > INT32_MAX) throw Bad{"a number is out of range"};
    return (int32_t)v;
}
double number(PyObject *o)
{
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Bad{""};
    return v;
}

void same(const int64_t *a, const int64_t *b, int n, const char *what)
{
    if (memcmp(a, b, n * sizeof(int64_t))) throw Bad{std::string(what) + " differ in strides"};
}

// (handle, device, cache address, layer, q, block_tables, lens, max_len, out, lse, window, scale, weights_in, weights_out)
int32_t attend(PyObject *const *v)
{
    const Call c{(int)integer(v[1]), (const kv_cache_t *)integer(v[2])};
    kv_attend_args_t a;
    memset(&a, 0, sizeof(a));
    const int64_t n = size_of(v[4], 0, "q"), heads = size_of(v[4], 1, "q");
    a.layer = integer32(v[3]);
    a.num_seqs = (int32_t)n;
    a.q_heads = (int32_t)heads;
    a.max_len = integer(v[7]);
    a.window = integer32(v[10]);
    a.scale = (float)number(v[11]);
    int64_t s[2], w[2];
    c.rows(v[4], c.type(), {n, heads, c.cache->head_dim}, "q", &a.q, s);
    a.q_seq_stride = s[0];
    a.q_head_stride = s[1];
    c.rows(v[8], c.type(), {n, heads, c.cache->head_dim}, "out", (const void **)&a.out, s);
    a.out_seq_stride = s[0];
    a.out_head_stride = s[1];
    c.tables(a, v[5], v[6], n);
    if (v[9] != Py_None) {
        c.rows(v[9], at::kFloat, {n, heads}, "lse", (const void **)&a.lse, s);
        if (s[0] != heads && n > 1) throw Bad{"lse must be contiguous"};
    }
    if (v[13] != Py_None) {
        c.slots(v[13], at::kFloat, {n, c.cache->kv_heads, -1}, a.max_len, "weights_out", (const void **)&a.weights_out, w);
        a.w_seq_stride = w[0];
        a.w_head_stride = w[1];
    }
    if (v[12] != Py_None) {
        c.slots(v[12], at::kFloat, {n, c.cache->kv_heads, -1}, a.max_len, "weights_in", (const void **)&a.weights_in, s);
        if (v[13] != Py_None) same(s, w, 2, "weights_in and weights_out");
    }
    return kv_attend((kv_ops_t *)integer(v[0]), c.cache, &a);
}

// (handle, device, cache address, layer, q, k, v, block_tables, lens, positions, inv_freq, axis_of, halves, q_out, seq_starts,
//  weights, order, token_order, q_norm, k_norm, norm_eps)
int32_t append(PyObject *const *v)
{
    const Call c{(int)integer(v[1]), (const kv_cache_t *)integer(v[2])};
    kv_append_args_t a;
    memset(&a, 0, sizeof(a));
    const int64_t t = size_of(v[5], 0, "k"), n = size_of(v[8], 0, "lens"), heads = c.cache->kv_heads, dim = c.cache->head_dim;
    int64_t s[2], w[2];
    a.layer = integer32(v[3]);
    a.num_seqs = (int32_t)n;
    a.num_tokens = t;
    a.pair_style = PyObject_IsTrue(v[12]) ? 0 : 1;
    if (v[4] != Py_None) {
        const int64_t q_heads = size_of(v[4], 1, "q");
        a.q_heads = (int32_t)q_heads;
        c.rows(v[4], c.type(), {t, q_heads, dim}, "q", &a.q, s);
        a.q_token_stride = s[0];
        a.q_head_stride = s[1];
        if (v[13] != Py_None) {
            c.rows(v[13], c.type(), {t, q_heads, dim}, "q_out", (const void **)&a.q_out, s);
            a.qo_token_stride = s[0];
            a.qo_head_stride = s[1];
        }
    }
    c.rows(v[5], c.type(), {t, heads, dim}, "k", &a.k, s);
    a.k_token_stride = s[0];
    a.k_head_stride = s[1];
    c.rows(v[6], c.type(), {t, heads, dim}, "v", &a.v, s);
    a.v_token_stride = s[0];
    a.v_head_stride = s[1];
    c.tables(a, v[7], v[8], n);
    a.num_axes = (int32_t)c.rows(v[9], at::kInt, {-1, t}, "positions", (const void **)&a.positions, &a.axis_stride).size(0);
    const int64_t half = c.rows(v[10], at::kFloat, {-1}, "inv_freq", (const void **)&a.inv_freq, nullptr).size(0);
    a.rotary_dim = (int32_t)(2 * half);
    if (half > 128) throw Bad{"at most 128 frequencies"};
    if (v[11] != Py_None) {
        PyObject *of = PySequence_Fast(v[11], "axis_of must be a sequence");
        if (!of) throw Bad{""};
        bool ok = PySequence_Fast_GET_SIZE(of) == half;
        for (int64_t f = 0; ok && f < half; ++f) {
            const long axis = PyLong_AsLong(PySequence_Fast_GET_ITEM(of, f));
            ok = axis >= 0 && axis < 256;
            a.axis_of[f] = (uint8_t)axis;
        }
        Py_DECREF(of);
        if (PyErr_Occurred()) throw Bad{""};
        if (!ok) throw Bad{"axis_of must name an axis for each frequency"};
    }
    if (v[14] != Py_None) c.rows(v[14], at::kInt, {n + 1}, "seq_starts", (const void **)&a.seq_starts, nullptr);
    int64_t slots = -1;
    if (v[15] != Py_None) {
        slots = c.rows(v[15], at::kFloat, {n, heads, -1}, "weights", (const void **)&a.weights, w).size(2);
        a.m_seq_stride = w[0];
        a.m_head_stride = w[1];
    }
    if (v[16] != Py_None) {
        const int64_t have = c.rows(v[16], at::kInt, {n, heads, -1}, "order", (const void **)&a.order, s).size(2);
        if (v[15] != Py_None && have != slots) throw Bad{"weights and order differ in shape"};
        if (v[15] != Py_None) same(s, w, 2, "weights and order");
        slots = have;
        a.m_seq_stride = s[0];
        a.m_head_stride = s[1];
        if (v[17] != Py_None) c.rows(v[17], at::kInt, {t}, "token_order", (const void **)&a.token_order, nullptr);
    }
    if (slots >= 0) a.num_slots = (int32_t)std::min<int64_t>(slots, INT32_MAX);
    if (v[18] == Py_None && v[19] == Py_None) return kv_append((kv_ops_t *)integer(v[0]), c.cache, &a);
    kv_norm_args_t norms;
    memset(&norms, 0, sizeof(norms));
    norms.eps = (float)number(v[20]);
    at::ScalarType kind = at::kFloat;
    // weights of one head for all, or of each; float32 or of the cache's type, both alike
    const auto weights = [&](PyObject *o, int64_t of_heads, const char *what, bool first, const void **p, int64_t *stride) {
        if (!THPVariable_Check(o)) throw Bad{std::string(what) + " must be a tensor"};
        const at::Tensor &w = THPVariable_Unpack(o);
        if (w.scalar_type() != at::kFloat && w.scalar_type() != c.type()) throw Bad{std::string(what) + " must be float32 or " + name_of(c.type()) + ", not " + name_of(w.scalar_type())};
        if (!first && w.scalar_type() != kind) throw Bad{"q_norm and k_norm differ in type"};
        kind = w.scalar_type();
        if (w.dim() == 1) c.rows(o, kind, {dim}, what, p, nullptr);
        else c.rows(o, kind, {of_heads, dim}, what, p, stride);
    };
    if (v[18] != Py_None) {
        if (v[4] == Py_None) throw Bad{"q_norm without q"};
        weights(v[18], a.q_heads, "q_norm", true, &norms.q_weight, &norms.q_head_stride);
    }
    if (v[19] != Py_None) weights(v[19], heads, "k_norm", v[18] == Py_None, &norms.k_weight, &norms.k_head_stride);
    norms.weight_float = kind == at::kFloat;
    return kv_append_normed((kv_ops_t *)integer(v[0]), c.cache, &a, &norms);
}

// (handle, device, cache address, layer, block_tables, lens, k_out, v_out, seq_starts)
int32_t read(PyObject *const *v)
{
    const Call c{(int)integer(v[1]), (const kv_cache_t *)integer(v[2])};
    kv_read_args_t a;
    memset(&a, 0, sizeof(a));
    const int64_t n = size_of(v[5], 0, "lens"), heads = c.cache->kv_heads, dim = c.cache->head_dim;
    const bool k = v[6] != Py_None, w = v[7] != Py_None;
    if (!k && !w) throw Bad{"k_out or v_out is needed"};
    const int64_t t = size_of(v[k ? 6 : 7], 0, k ? "k_out" : "v_out");
    int64_t s[2];
    a.layer = integer32(v[3]);
    a.num_seqs = (int32_t)n;
    a.num_tokens = t;
    if (k) {
        c.rows(v[6], c.type(), {t, heads, dim}, "k_out", (const void **)&a.k, s);
        a.k_token_stride = s[0];
        a.k_head_stride = s[1];
    }
    if (w) {
        c.rows(v[7], c.type(), {t, heads, dim}, "v_out", (const void **)&a.v, s);
        a.v_token_stride = s[0];
        a.v_head_stride = s[1];
    }
    c.tables(a, v[4], v[5], n);
    if (v[8] != Py_None) c.rows(v[8], at::kInt, {n + 1}, "seq_starts", (const void **)&a.seq_starts, nullptr);
    return kv_read((kv_ops_t *)integer(v[0]), c.cache, &a);
}

// (handle, device, cache address, block_tables, lens, max_len, keep, weights, order, seen, recent, sink, weights_out, order_out,
//  lens_out, first_layer)
int32_t evict(PyObject *const *v)
{
    const Call c{(int)integer(v[1]), (const kv_cache_t *)integer(v[2])};
    kv_evict_args_t a;
    memset(&a, 0, sizeof(a));
    const int64_t n = size_of(v[4], 0, "lens"), layers = size_of(v[7], 0, "weights"), heads = c.cache->kv_heads;
    int64_t m[3], s[3];
    a.first_layer = integer32(v[15]);
    a.num_layers = (int32_t)layers;
    a.num_seqs = (int32_t)n;
    a.max_len = integer(v[5]);
    a.keep = integer32(v[6]);
    a.recent = integer32(v[10]);
    a.sink = integer32(v[11]);
    c.tables(a, v[3], v[4], n);
    c.slots(v[7], at::kFloat, {layers, n, heads, -1}, a.max_len, "weights", (const void **)&a.weights, m);
    a.m_layer_stride = m[0];
    a.m_seq_stride = m[1];
    a.m_head_stride = m[2];
    if (v[8] != Py_None) {
        c.slots(v[8], at::kInt, {layers, n, heads, -1}, a.max_len, "order", (const void **)&a.order, s);
        same(s, m, 3, "weights and order");
    }
    const int64_t kept = std::min<int64_t>(a.keep, a.max_len);
    if (v[12] != Py_None) {
        c.slots(v[12], at::kFloat, {layers, n, heads, -1}, kept, "weights_out", (const void **)&a.weights_out, m);
        a.o_layer_stride = m[0];
        a.o_seq_stride = m[1];
        a.o_head_stride = m[2];
    }
    if (v[13] != Py_None) {
        c.slots(v[13], at::kInt, {layers, n, heads, -1}, kept, "order_out", (const void **)&a.order_out, s);
        if (v[12] != Py_None) same(s, m, 3, "weights_out and order_out");
    }
    if (v[9] != Py_None) c.rows(v[9], at::kInt, {n}, "seen", (const void **)&a.seen, nullptr);
    if (v[14] != Py_None) c.rows(v[14], at::kInt, {n}, "lens_out", (const void **)&a.lens_out, nullptr);
    return kv_evict((kv_ops_t *)integer(v[0]), c.cache, &a);
}

// no C++ exception leaves for the interpreter
template <int32_t (*call)(PyObject *const *), int count>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n)
{
    try {
        if (n != count) throw Bad{"wrong number of arguments"};
        return PyLong_FromLong(call(args));
    } catch (const Bad &b) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, b.what.c_str());
    } catch (const std::exception &e) {
        if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

PyMethodDef methods[] = {
    {"attend", (PyCFunction)(void (*)(void))entry<attend, 14>, METH_FASTCALL, "kv_attend on tensors; its status"},
    {"append", (PyCFunction)(void (*)(void))entry<append, 21>, METH_FASTCALL, "kv_append on tensors; its status"},
    {"read", (PyCFunction)(void (*)(void))entry<read, 9>, METH_FASTCALL, "kv_read on tensors; its status"},
    {"evict", (PyCFunction)(void (*)(void))entry<evict, 16>, METH_FASTCALL, "kv_evict on tensors; its status"},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_kvops", "argument marshalling of the operators on the device cache", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__kvops() { return PyModule_Create(&module); }
