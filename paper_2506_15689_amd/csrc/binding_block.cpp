// Python entry points of the operators around the linear layer and of a step's ends (include/basq.h): checks of shapes, types and places, then the C
// ABI.  A compiled module because of what a small call costs: marshalling thirty arguments of ten tensors in Python takes 7 .. 13 us,
// as long as the kernels of a decode step, here 1.  Every function takes its arguments by position (binding.py gives
// them names and defaults) and returns the C ABI's code; a tensor that does not fit is a ValueError.
#include <Python.h>

#include <c10/core/DeviceGuard.h>
#include <torch/csrc/autograd/python_variable.h>

#include <stdarg.h>

#include <string>

#include "../../include/basq.h"

namespace {

// thrown behind a Python exception that is set
struct Refused {};

[[noreturn]] void refuse(const char* format, ...) {
    char text[512];
    va_list ap;
    va_start(ap, format);
    vsnprintf(text, sizeof(text), format, ap);
    va_end(ap);
    PyErr_SetString(PyExc_ValueError, text);
    throw Refused{};
}

std::string shown(const at::Tensor& t) {
    std::string s = c10::toString(t.scalar_type());
    s += " [";
    for (int64_t d = 0; d < t.dim(); ++d) s += (d ? ", " : "") + std::to_string(t.size(d));
    return s + "]";
}

// The tensors of a call: all on one GPU.  (Arguments that a test of the checks gives on the CPU are refused last, so that their own
// fault is named.)
struct Call {
    const char* elsewhere = nullptr;
    int device = -2;

    const at::Tensor* tensor(PyObject* o, const char* name, bool needed = true) {
        if (o == Py_None) {
            if (needed) refuse("%s must be given", name);
            return nullptr;
        }
        if (!THPVariable_Check(o)) refuse("%s must be a tensor", name);
        const at::Tensor& t = THPVariable_Unpack(o);
        const int on = t.is_cuda() ? (int)t.get_device() : -1;
        if (device == -2) device = on;
        if (on < 0 || on != device) elsewhere = name;
        return &t;
    }
    void same_gpu() const {
        if (elsewhere) refuse("%s is not on the GPU of the other tensors", elsewhere);
    }
};

// Where a tensor's values are.  Asked for while the GIL is held: it throws for tensors without storage of their own (those that stand for
// others under torch.vmap, say).
template <class T = void>
T* data(const at::Tensor* t) { return t ? static_cast<T*>(t->data_ptr()) : nullptr; }

// a tensor [rows, ...] of this shape whose rows are contiguous: its row stride (one row has no stride of its own)
int64_t rows_of(const at::Tensor& t, const at::Tensor& like, const char* name, at::ScalarType type) {
    if (t.scalar_type() != type || t.sizes() != like.sizes())
        refuse("%s must be %s with the shape of %s, not %s", name, c10::toString(type), shown(like).c_str(), shown(t).c_str());
    int64_t width = 1;
    bool side_by_side = true;
    for (int64_t d = t.dim() - 1; d >= 1; --d) {
        if (t.size(d) > 1 && t.stride(d) != width) side_by_side = false;
        width *= t.size(d);
    }
    if (!side_by_side && t.numel() > 0) refuse("the values of one row of %s must lie side by side", name);
    return t.size(0) > 1 ? t.stride(0) : width;
}

void vector_of(const at::Tensor& t, int64_t n, const char* name, at::ScalarType type) {
    if (t.scalar_type() != type || t.numel() != n || !t.is_contiguous())
        refuse("%s must be contiguous %s of %lld values, not %s", name, c10::toString(type), (long long)n, shown(t).c_str());
}

// tokens of a page
int page_size_of(const at::Tensor& cache, int64_t D) {
    if (cache.scalar_type() != at::kByte || cache.dim() != 3 || !cache.is_contiguous() || cache.size(2) % (D + 16) != 0 || cache.size(2) > INT32_MAX)
        refuse("cache must be contiguous uint8 [pages, kv heads, page_size * %lld], not %s", (long long)(D + 16), shown(cache).c_str());
    return (int)(cache.size(2) / (D + 16));
}

int32_t narrow(int64_t v, const char* name) {
    if (v < INT32_MIN || v > INT32_MAX) refuse("%s does not fit 32 bits", name);
    return (int32_t)v;
}

int64_t whole(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Refused{};
    return v;
}
double real(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) throw Refused{};
    return v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refused{};
    return v != 0;
}
// The stream of a call, and its GPU made the current one while this lives (a launch goes to the current GPU, whatever the stream is).
// `handle_of(stream, device)` names the handle; it is asked behind the checks, which work without a GPU.
class Launch {
public:
    Launch(const Call& c, PyObject* handle_of, PyObject* of) {
        PyObject* index = PyLong_FromLong(c.device);
        PyObject* handle = index ? PyObject_CallFunctionObjArgs(handle_of, of, index, nullptr) : nullptr;
        Py_XDECREF(index);
        if (!handle) throw Refused{};
        const long long v = PyLong_AsLongLong(handle);
        Py_DECREF(handle);
        if (v == -1 && PyErr_Occurred()) throw Refused{};
        stream = reinterpret_cast<void*>((intptr_t)v);
        guard_.reset_device(c10::Device(c10::DeviceType::CUDA, (c10::DeviceIndex)c.device));
    }
    void* stream;

private:
    c10::OptionalDeviceGuard guard_;
};

// runs `body`; no C++ exception leaves a Python entry point
template <class Body>
PyObject* entry(Py_ssize_t given, Py_ssize_t wanted, Body body) {
    if (given != wanted) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, %zd are needed", given, wanted);
        return nullptr;
    }
    try {
        return PyLong_FromLong(body());
    } catch (const Refused&) {
        return nullptr;
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
        return nullptr;
    }
}

// (nothing in `run` may touch Python or throw)
template <class Run>
int without_gil(Run run) {
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = run();
    Py_END_ALLOW_THREADS
    return rc;
}

// (X, residual, weight, eps, Y, res_out, Y8, y8_scale, handle_of, stream)
PyObject* add_rms_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(n, 10, [&] {
        Call c;
        const at::Tensor& X = *c.tensor(args[0], "X");
        const at::Tensor* residual = c.tensor(args[1], "residual", false);
        const at::Tensor& weight = *c.tensor(args[2], "weight");
        const float eps = (float)real(args[3]);
        const at::Tensor *Y = c.tensor(args[4], "Y", false), *res_out = c.tensor(args[5], "res_out", false);
        const at::Tensor *Y8 = c.tensor(args[6], "Y8", false), *y8_scale = c.tensor(args[7], "y8_scale", false);
        if (X.dim() != 2) refuse("X must be [M, K], not %s", shown(X).c_str());
        const int64_t M = X.size(0), ldx = rows_of(X, X, "X", at::kBFloat16);
        const int32_t K = narrow(X.size(1), "K");
        vector_of(weight, K, "weight", at::kBFloat16);
        const int64_t ldr = residual ? rows_of(*residual, X, "residual", at::kBFloat16) : 0;
        const int64_t ldro = res_out ? rows_of(*res_out, X, "res_out", at::kBFloat16) : 0, ldy = Y ? rows_of(*Y, X, "Y", at::kBFloat16) : 0;
        const int64_t ldy8 = Y8 ? rows_of(*Y8, X, "Y8", at::kFloat8_e4m3fn) : 0;
        if (y8_scale) vector_of(*y8_scale, M, "y8_scale", at::kFloat);
        c.same_gpu();
        const void *x = data(&X), *r = data(residual), *w = data(&weight);
        void *h = data(res_out), *y = data(Y);
        uint8_t* y8 = data<uint8_t>(Y8);
        float* scale = data<float>(y8_scale);
        const Launch on(c, args[8], args[9]);
        return without_gil([&] { return basq_add_rms_norm(x, r, w, M, K, ldx, ldr, eps, h, ldro, y, ldy, y8, ldy8, scale, on.stream); });
    });
}

// (q, k, v, positions, cos_sin, slots, cache, clip_lo, clip_hi, q_out, k_hat, v_hat, interleaved, rotate, bits, handle_of, stream)
PyObject* rope_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(n, 17, [&] {
        Call c;
        const at::Tensor *q = c.tensor(args[0], "q", false), *k = c.tensor(args[1], "k", false), *v = c.tensor(args[2], "v", false);
        const at::Tensor *positions = c.tensor(args[3], "positions", false), *cos_sin = c.tensor(args[4], "cos_sin", false);
        const at::Tensor *slots = c.tensor(args[5], "slots", false), *cache = c.tensor(args[6], "cache", false);
        const float clip_lo = (float)real(args[7]), clip_hi = (float)real(args[8]);
        const at::Tensor *q_out = c.tensor(args[9], "q_out", false), *k_hat = c.tensor(args[10], "k_hat", false), *v_hat = c.tensor(args[11], "v_hat", false);
        const bool interleaved = truth(args[12]), rotate = truth(args[13]);
        const int32_t bits = narrow(whole(args[14]), "bits");
        if ((!q && !k) || !k != !v) refuse("q, or k and v, must be given");
        const at::Tensor& some = q ? *q : *k;
        if (some.dim() != 3 || (k && k->dim() != 3)) refuse("q, k and v must be [T, heads, head_dim]");
        const int64_t T = some.size(0), D = some.size(2);
        const int32_t head_dim = narrow(D, "head_dim");
        if (k && (k->size(0) != T || k->size(2) != D)) refuse("k must have the tokens and channels of q, %lld and %lld, not %s", (long long)T, (long long)D, shown(*k).c_str());
        int32_t heads = 0, kv_heads = 0, pages = 0, page_size = 0, rot = 0;
        int64_t ldq = 0, ldqo = 0, ldk = 0, ldv = 0, ldh = 0, table_rows = 0;
        if (q) {
            if (!q_out) refuse("q_out must be given with q");
            heads = narrow(q->size(1), "heads");
            ldq = rows_of(*q, *q, "q", at::kBFloat16);
            ldqo = rows_of(*q_out, *q, "q_out", at::kBFloat16);
        }
        if (k) {
            kv_heads = narrow(k->size(1), "kv_heads");
            ldk = rows_of(*k, *k, "k", at::kBFloat16);
            ldv = rows_of(*v, *k, "v", at::kBFloat16);
            if (cache) {
                page_size = page_size_of(*cache, D);
                pages = narrow(cache->size(0), "pages");
                if (cache->size(1) != kv_heads) refuse("the cache has %lld kv heads, k has %d", (long long)cache->size(1), kv_heads);
                if (!slots) refuse("slots must be given with cache");
                vector_of(*slots, T, "slots", at::kInt);
            }
            if (k_hat) ldh = rows_of(*k_hat, *k, "k_hat", at::kBFloat16);
            if (v_hat) {
                const int64_t ld = rows_of(*v_hat, *k, "v_hat", at::kBFloat16);
                if (k_hat && ld != ldh) refuse("k_hat and v_hat must have the same token stride");
                ldh = ld;
            }
        }
        if (cos_sin) {
            if (cos_sin->dim() != 2) refuse("cos_sin must be [rows, rot_dim], not %s", shown(*cos_sin).c_str());
            table_rows = cos_sin->size(0);
            rot = narrow(cos_sin->size(1), "rot_dim");
            vector_of(*cos_sin, table_rows * rot, "cos_sin", at::kFloat);
            if (!positions) refuse("positions must be given with cos_sin");
            vector_of(*positions, T, "positions", at::kInt);
        }
        c.same_gpu();
        const void *qs = data(q), *ks = data(k), *vs = data(v);
        const int32_t *at = data<int32_t>(positions), *to = data<int32_t>(slots);
        const float* table = data<float>(cos_sin);
        uint8_t* blocks = data<uint8_t>(cache);
        void *turned = data(q_out), *kh = data(k_hat), *vh = data(v_hat);
        const Launch on(c, args[15], args[16]);
        return without_gil([&] {
            return basq_rope_append(qs, ldq, ks, ldk, vs, ldv, T, heads, kv_heads, head_dim, at, table, table_rows, rot, interleaved, rotate, clip_lo,
                                    clip_hi, bits, to, blocks, pages, page_size, turned, ldqo, kh, vh, ldh, on.stream);
        });
    });
}

// (q, cache, page_table, lengths, max_len, scale, out, workspace, q_len, softcap, window, lse, bits, handle_of, stream)
PyObject* paged_attention(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(n, 15, [&] {
        Call c;
        const at::Tensor &q = *c.tensor(args[0], "q"), &cache = *c.tensor(args[1], "cache"), &table = *c.tensor(args[2], "page_table");
        const at::Tensor& lengths = *c.tensor(args[3], "lengths");
        const int32_t max_len = narrow(whole(args[4]), "max_len");
        const float scale = (float)real(args[5]);
        const at::Tensor& out = *c.tensor(args[6], "out");
        const at::Tensor* workspace = c.tensor(args[7], "workspace", false);
        const int32_t q_len = narrow(whole(args[8]), "q_len");
        const float softcap = (float)real(args[9]);
        const int32_t window = narrow(whole(args[10]), "window");
        const at::Tensor* lse = c.tensor(args[11], "lse", false);
        const int32_t bits = narrow(whole(args[12]), "bits");
        if (q.dim() != 3) refuse("q must be [B * q_len, heads, head_dim], not %s", shown(q).c_str());
        const int64_t rows = q.size(0), heads = q.size(1), D = q.size(2), B = lengths.numel();
        vector_of(lengths, B, "lengths", at::kInt);
        if (rows != B * q_len) refuse("q has %lld rows, %lld sequences of %d new tokens need %lld", (long long)rows, (long long)B, q_len, (long long)B * q_len);
        if (table.scalar_type() != at::kInt || table.dim() != 2 || table.size(0) != B || (table.size(1) > 1 && table.stride(1) != 1))
            refuse("page_table must be int32 [%lld, pages of a sequence], not %s", (long long)B, shown(table).c_str());
        const int64_t ldq = rows_of(q, q, "q", at::kBFloat16), ldo = rows_of(out, q, "out", at::kBFloat16);
        if (lse) vector_of(*lse, rows * heads, "lse", at::kFloat);
        const int page_size = page_size_of(cache, D);
        // (the row stride may be wider than the row)
        if (max_len > table.size(1) * (int64_t)page_size)
            refuse("max_len = %d is more than the %lld pages of %d tokens of a sequence hold", max_len, (long long)table.size(1), page_size);
        if (workspace && !workspace->is_contiguous()) refuse("workspace must be contiguous");
        const int32_t sequences = narrow(B, "B"), head_dim = narrow(D, "head_dim"), all_heads = narrow(heads, "heads");
        const int32_t kv_heads = narrow(cache.size(1), "kv_heads"), pages = narrow(cache.size(0), "pages");
        const int64_t table_stride = B > 1 ? table.stride(0) : table.size(1);
        const size_t room = workspace ? workspace->nbytes() : 0;
        c.same_gpu();
        const void* rows_q = data(&q);
        const uint8_t* blocks = data<uint8_t>(&cache);
        const int32_t *page_of = data<int32_t>(&table), *lens = data<int32_t>(&lengths);
        void *result = data(&out), *parts = data(workspace);
        float* sums = data<float>(lse);
        const Launch on(c, args[13], args[14]);
        return without_gil([&] {
            return basq_paged_attention(rows_q, ldq, sequences, q_len, all_heads, kv_heads, head_dim, bits, blocks, pages, page_size, page_of, table_stride,
                                        lens, max_len, scale, softcap, window, result, ldo, sums, parts, room, on.stream);
        });
    });
}

// codes, scales and zero points of [N, K] weights with groups: N and the channels of a group
struct Weights {
    int32_t N, group;
};
Weights weights_of(const at::Tensor& Wq, const at::Tensor& scale, const at::Tensor& zero, int64_t K, int32_t layout) {
    if (scale.scalar_type() != at::kBFloat16 || scale.dim() < 1 || scale.dim() > 2 || !scale.is_contiguous() || scale.numel() < 1)
        refuse("w_scale must be contiguous BFloat16 [N, groups], not %s", shown(scale).c_str());
    vector_of(zero, scale.numel(), "w_zero", at::kBFloat16);
    const int64_t N = scale.size(0), groups = scale.numel() / N;
    if (K < 1 || K % groups != 0) refuse("%lld channels are not %lld groups", (long long)K, (long long)groups);
    const int64_t rows = layout == BASQ_W_DECODE16 ? (N + 15) / 16 * 16 : N;
    vector_of(Wq, rows * (K / 2), "Wq", at::kByte);
    return Weights{narrow(N, "N"), narrow(K / groups, "K")};
}

// (x, Wq, w_scale, w_zero, y, bias, w_layout, handle_of, stream)
PyObject* w4a16_gemm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(n, 9, [&] {
        Call c;
        const at::Tensor &x = *c.tensor(args[0], "x"), &Wq = *c.tensor(args[1], "Wq"), &scale = *c.tensor(args[2], "w_scale"), &zero = *c.tensor(args[3], "w_zero");
        const at::Tensor& y = *c.tensor(args[4], "y");
        const at::Tensor* bias = c.tensor(args[5], "bias", false);
        const int32_t layout = narrow(whole(args[6]), "w_layout");
        if (x.dim() != 2) refuse("x must be [M, K], not %s", shown(x).c_str());
        const int64_t M = x.size(0), ldx = rows_of(x, x, "x", at::kBFloat16);
        const int32_t K = narrow(x.size(1), "K");
        const Weights w = weights_of(Wq, scale, zero, K, layout);
        const bool f32 = y.scalar_type() == at::kFloat;
        if (y.dim() != 2 || y.size(0) != M || y.size(1) != w.N || (!f32 && y.scalar_type() != at::kBFloat16))
            refuse("y must be Float or BFloat16 [%lld, %d], not %s", (long long)M, w.N, shown(y).c_str());
        const int64_t ldy = rows_of(y, y, "y", y.scalar_type());
        if (bias) vector_of(*bias, w.N, "bias", at::kFloat);
        c.same_gpu();
        const void *rows = data(&x), *s = data(&scale), *z = data(&zero);
        const uint8_t* codes = data<uint8_t>(&Wq);
        const float* add = data<float>(bias);
        void* out = data(&y);
        const Launch on(c, args[7], args[8]);
        return without_gil([&] { return basq_w4a16_gemm(rows, M, K, ldx, codes, w.N, layout, s, z, w.group, add, out, ldy, f32, on.stream); });
    });
}

// (ids, Wq, w_scale, w_zero, y, scale, w_layout, handle_of, stream)
PyObject* w4a16_lookup(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(n, 9, [&] {
        Call c;
        const at::Tensor &ids = *c.tensor(args[0], "ids"), &Wq = *c.tensor(args[1], "Wq"), &scale = *c.tensor(args[2], "w_scale"), &zero = *c.tensor(args[3], "w_zero");
        const at::Tensor& y = *c.tensor(args[4], "y");
        const float factor = (float)real(args[5]);
        const int32_t layout = narrow(whole(args[6]), "w_layout");
        if (y.dim() != 2) refuse("y must be [T, K], not %s", shown(y).c_str());
        const int64_t T = y.size(0), ldy = rows_of(y, y, "y", at::kBFloat16);
        const int32_t K = narrow(y.size(1), "K");
        vector_of(ids, T, "ids", at::kInt);
        const Weights w = weights_of(Wq, scale, zero, K, layout);
        c.same_gpu();
        const int32_t* which = data<int32_t>(&ids);
        const void *s = data(&scale), *z = data(&zero);
        const uint8_t* codes = data<uint8_t>(&Wq);
        void* out = data(&y);
        const Launch on(c, args[7], args[8]);
        return without_gil([&] { return basq_w4a16_lookup(which, T, codes, w.N, K, layout, s, z, w.group, factor, out, ldy, on.stream); });
    });
}

// (logits, u, token, workspace, temperature, top_k, top_p, min_p, logprob, kept, handle_of, stream)
PyObject* sample(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(n, 12, [&] {
        Call c;
        const at::Tensor &logits = *c.tensor(args[0], "logits"), &u = *c.tensor(args[1], "u"), &token = *c.tensor(args[2], "token");
        const at::Tensor* workspace = c.tensor(args[3], "workspace", false);
        const at::Tensor *temperature = c.tensor(args[4], "temperature", false), *top_k = c.tensor(args[5], "top_k", false);
        const at::Tensor *top_p = c.tensor(args[6], "top_p", false), *min_p = c.tensor(args[7], "min_p", false);
        const at::Tensor *logprob = c.tensor(args[8], "logprob", false), *kept = c.tensor(args[9], "kept", false);
        const bool f32 = logits.scalar_type() == at::kFloat;
        if (logits.dim() != 2 || (!f32 && logits.scalar_type() != at::kBFloat16)) refuse("logits must be Float or BFloat16 [B, V], not %s", shown(logits).c_str());
        const int32_t B = narrow(logits.size(0), "B"), V = narrow(logits.size(1), "V");
        const int64_t ldl = rows_of(logits, logits, "logits", logits.scalar_type());
        vector_of(u, B, "u", at::kDouble);
        vector_of(token, B, "token", at::kInt);
        if (temperature) vector_of(*temperature, B, "temperature", at::kFloat);
        if (top_k) vector_of(*top_k, B, "top_k", at::kInt);
        if (top_p) vector_of(*top_p, B, "top_p", at::kFloat);
        if (min_p) vector_of(*min_p, B, "min_p", at::kFloat);
        if (logprob) vector_of(*logprob, B, "logprob", at::kFloat);
        if (kept) vector_of(*kept, B, "kept", at::kInt);
        if (workspace && !workspace->is_contiguous()) refuse("workspace must be contiguous");
        const size_t room = workspace ? workspace->nbytes() : 0;
        c.same_gpu();
        const void* rows = data(&logits);
        const double* numbers = data<double>(&u);
        int32_t *drawn = data<int32_t>(&token), *many = data<int32_t>(kept);
        const float *heat = data<float>(temperature), *mass = data<float>(top_p), *least = data<float>(min_p);
        const int32_t* most = data<int32_t>(top_k);
        float* ln = data<float>(logprob);
        void* parts = data(workspace);
        const Launch on(c, args[10], args[11]);
        return without_gil([&] { return basq_sample(rows, ldl, B, V, f32, heat, most, mass, least, numbers, drawn, ln, many, parts, room, on.stream); });
    });
}

// (lengths, pool_table, free_pages, free_count, new_tokens, page_size, positions, slots, status, books, seqs, q_len, starts, batch_table,
//  batch_lengths, lengths_out, free_out, handle_of, stream)
PyObject* kv_extend(PyObject*, PyObject* const* args, Py_ssize_t n) {
    return entry(n, 19, [&] {
        Call c;
        const at::Tensor &lengths = *c.tensor(args[0], "lengths"), &pool = *c.tensor(args[1], "pool_table"), &pages = *c.tensor(args[2], "free_pages");
        const at::Tensor& count = *c.tensor(args[3], "free_count");
        const at::Tensor* fresh = c.tensor(args[4], "new_tokens", false);
        const int32_t page_size = narrow(whole(args[5]), "page_size");
        const at::Tensor &positions = *c.tensor(args[6], "positions"), &slots = *c.tensor(args[7], "slots"), &status = *c.tensor(args[8], "status");
        const at::Tensor &books = *c.tensor(args[9], "books"), *seqs = c.tensor(args[10], "seqs", false);
        const int32_t q_len = narrow(whole(args[11]), "q_len");
        const at::Tensor *starts = c.tensor(args[12], "starts", false), *table = c.tensor(args[13], "batch_table", false);
        const at::Tensor* batch_lengths = c.tensor(args[14], "batch_lengths", false);
        const at::Tensor *lengths_out = c.tensor(args[15], "lengths_out", false), *free_out = c.tensor(args[16], "free_out", false);
        if (pool.dim() != 2) refuse("pool_table must be [rows, columns], not %s", shown(pool).c_str());
        const int32_t rows = narrow(pool.size(0), "rows"), columns = narrow(pool.size(1), "columns");
        const int64_t pool_stride = rows_of(pool, pool, "pool_table", at::kInt);
        vector_of(lengths, rows, "lengths", at::kInt);
        if (lengths_out) vector_of(*lengths_out, rows, "lengths_out", at::kInt);
        const int32_t capacity = narrow(pages.numel(), "free_pages");
        vector_of(pages, capacity, "free_pages", at::kInt);
        vector_of(count, 1, "free_count", at::kInt);
        if (free_out) vector_of(*free_out, 1, "free_out", at::kInt);
        if (!seqs && !fresh) refuse("seqs or new_tokens must be given");
        const int32_t B = narrow((seqs ? *seqs : *fresh).numel(), "B");
        if (seqs) vector_of(*seqs, B, "seqs", at::kInt);
        if (fresh) vector_of(*fresh, B, "new_tokens", at::kInt);
        const int64_t T = positions.numel();
        vector_of(positions, T, "positions", at::kInt);
        vector_of(slots, T, "slots", at::kInt);
        vector_of(status, 2, "status", at::kInt);
        if (starts) vector_of(*starts, B + 1, "starts", at::kInt);
        if (batch_lengths) vector_of(*batch_lengths, B, "batch_lengths", at::kInt);
        int64_t batch_stride = 0;
        if (table) {
            if (table->dim() != 2 || table->size(0) != B || table->size(1) != columns) refuse("batch_table must be [%d, %d], not %s", B, columns, shown(*table).c_str());
            batch_stride = rows_of(*table, *table, "batch_table", at::kInt);
        }
        if (!books.is_contiguous()) refuse("books must be contiguous");
        const size_t room = books.nbytes();
        c.same_gpu();
        auto ints = [](const at::Tensor* t) { return data<int32_t>(t); };
        const int32_t *had = ints(&lengths), *free_n = ints(&count), *of = ints(seqs), *plus = ints(fresh);
        int32_t *pool_at = ints(&pool), *free_at = ints(&pages), *pos = ints(&positions), *to = ints(&slots), *why = ints(&status), *first = ints(starts);
        int32_t *rows_at = ints(table), *lens = ints(batch_lengths), *have = ints(lengths_out ? lengths_out : &lengths), *left = ints(free_out ? free_out : &count);
        void* plan = data(&books);
        const Launch on(c, args[17], args[18]);
        return without_gil([&] {
            return basq_kv_extend(had, pool_at, pool_stride, rows, columns, page_size, free_at, capacity, free_n, of, plus, B, q_len, pos, to, T, first,
                                  rows_at, batch_stride, lens, have, left, why, plan, room, on.stream);
        });
    });
}

PyMethodDef methods[] = {
    {"add_rms_norm", (PyCFunction)(void (*)(void))add_rms_norm, METH_FASTCALL, nullptr},
    {"rope_append", (PyCFunction)(void (*)(void))rope_append, METH_FASTCALL, nullptr},
    {"paged_attention", (PyCFunction)(void (*)(void))paged_attention, METH_FASTCALL, nullptr},
    {"w4a16_gemm", (PyCFunction)(void (*)(void))w4a16_gemm, METH_FASTCALL, nullptr},
    {"w4a16_lookup", (PyCFunction)(void (*)(void))w4a16_lookup, METH_FASTCALL, nullptr},
    {"sample", (PyCFunction)(void (*)(void))sample, METH_FASTCALL, nullptr},
    {"kv_extend", (PyCFunction)(void (*)(void))kv_extend, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_block", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__block(void) { return PyModule_Create(&module); }
