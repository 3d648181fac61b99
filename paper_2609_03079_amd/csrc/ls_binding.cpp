// ls_binding.cpp - Python module of the decoder-layer operators (include/ls_ops.h).
//
// Argument marshalling only: sizes, strides, types and addresses of torch tensors into the C
// calls.  It is compiled because these calls are short (one token's norm takes 3 us on the GPU)
// and filling the argument structures from Python took 10 to 15 us of host time a call.
#include <ATen/core/Tensor.h>
#include <torch/csrc/utils/pybind.h>

#include <optional>
#include <string>

#include "../../include/ls_ops.h"

namespace py = pybind11;

namespace {

using at::Tensor;
using Maybe = std::optional<Tensor>;

[[noreturn]] void bad(const std::string& text) { throw py::value_error(text); }

ls_dtype type_of(const Tensor& t, const char* what, bool int8 = false) {
    switch (t.scalar_type()) {
        case at::kFloat: return LS_F32;
        case at::kHalf: return LS_F16;
        case at::kBFloat16: return LS_BF16;
        case at::kChar:
            if (int8) return LS_I8;
            [[fallthrough]];
        default: bad(std::string(what) + " has an unsupported type");
    }
}

void expect(const Tensor& t, at::ScalarType type, const char* what) {
    if (t.scalar_type() != type) bad(std::string(what) + " has the wrong type");
}

// Stride of a dimension in elements, 0 where it has one entry.
int64_t step(const Tensor& t, int dim) { return t.size(dim) > 1 ? t.stride(dim) : 0; }

int32_t count(int64_t n, const char* what) {
    if (n < 0 || n > INT32_MAX) bad(std::string(what) + " does not fit 32 bits");
    return (int32_t)n;
}

const void* data(const Maybe& t) { return t ? t->const_data_ptr() : nullptr; }

class Ops {
public:
    // device: the current one, which the library makes the context on
    Ops(uint64_t workspace_bytes, uintptr_t stream, int device) : device_(device) {
        ls_ops_desc d{};
        d.workspace_bytes = workspace_bytes;
        d.stream = reinterpret_cast<void*>(stream);
        check(ls_ops_create(&d, &ctx_));
    }
    ~Ops() { close(); }
    Ops(const Ops&) = delete;

    void close() {
        if (ctx_) ls_ops_destroy(ctx_);
        ctx_ = nullptr;
    }
    uintptr_t ctx() const { return reinterpret_cast<uintptr_t>(ctx_); }
    void sync() { check(ls_ops_sync(ctx_)); }

    void norm(const Tensor& x, const Maybe& y, const Maybe& gate, bool post_norm, const Maybe& post_weight, bool pre_norm,
              const Maybe& pre_weight, float x_scale, float y_scale, float eps, const Maybe& x_out, const Maybe& h) {
        if (x.dim() != 2) bad("x has the wrong shape");
        ls_norm_args a{};
        const int64_t T = x.size(0), d = x.size(1);
        a.n_tokens = count(T, "x");
        a.d = count(d, "x");
        expect(x, at::kFloat, "x");
        shaped(x, {T, d}, "x");
        a.x = static_cast<const float*>(x.const_data_ptr());
        a.x_stride = step(x, 0);
        std::optional<at::ScalarType> type;
        auto take = [&](const Maybe& t, at::IntArrayRef sizes, const char* what) {
            if (!t) return;
            shaped(*t, sizes, what);
            if (!type) a.dtype = type_of(*t, what), type = t->scalar_type();
            expect(*t, *type, what);
        };
        take(y, {T, d}, "y");
        take(h, {T, d}, "h");
        if (gate && gate->dim() == 1) {
            take(gate, {d}, "gate");
        } else {
            take(gate, {T, d}, "gate");
            a.gate_stride = gate ? step(*gate, 0) : 0;
        }
        take(post_weight, {d}, "post_weight");
        take(pre_weight, {d}, "pre_weight");
        a.y_stride = y ? step(*y, 0) : 0;
        a.h_stride = h ? step(*h, 0) : 0;
        if (x_out) {
            expect(*x_out, at::kFloat, "x_out");
            shaped(*x_out, {T, d}, "x_out");
            a.x_out = static_cast<float*>(x_out->data_ptr());
            a.x_out_stride = step(*x_out, 0);
        }
        a.post_norm = post_norm, a.pre_norm = pre_norm;
        a.x_scale = x_scale, a.y_scale = y_scale, a.eps = eps;
        a.y = data(y), a.gate = data(gate), a.post_weight = data(post_weight), a.pre_weight = data(pre_weight);
        a.h = h ? h->data_ptr() : nullptr;
        check(ls_norm_residual(ctx_, &a));
    }

    void linear(const Tensor& x, const Tensor& w, const Tensor& w_scale, const Tensor& out, const Maybe& x_scale, const Maybe& bias) {
        if (x.dim() != 2 || w.dim() != 2) bad("x or w has the wrong shape");
        ls_linear_i8_args a{};
        const int64_t T = x.size(0), k = x.size(1), n = w.size(0);
        a.n_tokens = count(T, "x"), a.k = count(k, "x"), a.n = count(n, "w");
        shaped(x, {T, k}, "x");
        shaped(w, {n, k}, "w");
        shaped(out, {T, n}, "out");
        a.x_type = type_of(x, "x", true);
        a.out_type = type_of(out, "out");
        expect(w, at::kChar, "w");
        auto vector = [&](const Tensor& t, int64_t size, const char* what) {
            expect(t, at::kFloat, what);
            shaped(t, {size}, what);
            return static_cast<const float*>(t.const_data_ptr());
        };
        a.x = x.const_data_ptr(), a.x_stride = step(x, 0);
        a.w = static_cast<const int8_t*>(w.const_data_ptr()), a.w_stride = step(w, 0);
        a.w_scale = vector(w_scale, n, "w_scale");
        a.bias = bias ? vector(*bias, n, "bias") : nullptr;
        a.x_scale = x_scale ? vector(*x_scale, T, "x_scale") : nullptr;
        a.out = out.data_ptr(), a.out_stride = step(out, 0);
        check(ls_linear_i8(ctx_, &a));
    }

    void append(const Tensor& k_cache, const Tensor& v_cache, const Tensor& k, const Tensor& v, const Maybe& positions, const Tensor& slots,
                const Maybe& cos_sin, const Maybe& q, const Maybe& q_out, int style) {
        const ls_kv_cache c = cache(k_cache, v_cache);
        if (k.dim() != 3) bad("k has the wrong shape");
        ls_append_args a{};
        const int64_t T = k.size(0), d = c.head_dim;
        a.n_tokens = count(T, "k");
        a.style = static_cast<ls_rope>(style);
        auto heads = [&](const Tensor& t, int64_t n, const char* what, int64_t* token, int64_t* head) {
            expect(t, k_cache.scalar_type(), what);
            shaped(t, {T, n, d}, what);
            *token = step(t, 0), *head = step(t, 1);
        };
        heads(k, c.n_kv_heads, "k", &a.k_token_stride, &a.k_head_stride);
        heads(v, c.n_kv_heads, "v", &a.v_token_stride, &a.v_head_stride);
        a.k = k.const_data_ptr(), a.v = v.const_data_ptr();
        if (q) {
            if (q->dim() != 3) bad("q has the wrong shape");
            a.n_heads = count(q->size(1), "q");
            heads(*q, a.n_heads, "q", &a.q_token_stride, &a.q_head_stride);
            a.q = q->const_data_ptr();
        }
        if (q_out) {
            heads(*q_out, a.n_heads, "q_out", &a.q_out_token_stride, &a.q_out_head_stride);
            a.q_out = q_out->data_ptr();
        }
        if (positions) a.positions = indices(*positions, {T}, "positions");
        a.slots = indices(slots, {T}, "slots");
        if (cos_sin) {
            if (cos_sin->dim() != 2) bad("cos_sin has the wrong shape");
            expect(*cos_sin, at::kFloat, "cos_sin");
            on_device(*cos_sin, "cos_sin");
            if (!cos_sin->is_contiguous()) bad("cos_sin is not contiguous");
            a.n_pos = count(cos_sin->size(0), "cos_sin"), a.rot_dim = count(cos_sin->size(1), "cos_sin");
            a.cos_sin = static_cast<const float*>(cos_sin->const_data_ptr());
        }
        check(ls_kv_append(ctx_, &c, &a));
    }

    void attend(const Tensor& q, const Tensor& k_cache, const Tensor& v_cache, const Maybe& pages, const Tensor& lens, const Tensor& out,
                int64_t max_len, float scale, int64_t n_q, const Maybe& prefix_pages, int64_t prefix_len) {
        const ls_kv_cache c = cache(k_cache, v_cache);
        if (q.dim() != 3 || lens.dim() != 1) bad("q or lens has the wrong shape");
        ls_attend_args a{};
        const int64_t T = q.size(0), heads = q.size(1), S = lens.size(0);
        a.n_seqs = count(S, "lens"), a.n_q = count(n_q, "n_q"), a.n_heads = count(heads, "q");
        if (T != S * n_q) bad("q must have n_q tokens for every sequence");
        expect(q, k_cache.scalar_type(), "q");
        expect(out, k_cache.scalar_type(), "out");
        shaped(q, {T, heads, c.head_dim}, "q");
        shaped(out, {T, heads, c.head_dim}, "out");
        a.q = q.const_data_ptr(), a.q_token_stride = step(q, 0), a.q_head_stride = step(q, 1);
        a.out = out.data_ptr(), a.out_token_stride = step(out, 0), a.out_head_stride = step(out, 1);
        a.lens = indices(lens, {S}, "lens");
        a.max_len = max_len < 0 ? -1 : count(max_len, "max_len");
        a.prefix_len = prefix_len < 0 ? -1 : count(prefix_len, "prefix_len");
        a.scale = scale;
        if (prefix_pages) {
            if (prefix_pages->dim() != 1) bad("prefix_pages has the wrong shape");
            a.prefix_pages = indices(*prefix_pages, {prefix_pages->size(0)}, "prefix_pages");
        }
        if (prefix_len > 0 && (!prefix_pages || prefix_pages->size(0) * c.page_size < prefix_len))
            bad("prefix_pages hold fewer than prefix_len keys");
        if (pages) {
            if (pages->dim() != 2) bad("pages has the wrong shape");
            a.pages = indices(*pages, {S, pages->size(1)}, "pages");
            if (pages->size(1) * c.page_size < max_len) bad("pages hold fewer than max_len keys");
            a.pages_stride = S > 1 ? pages->stride(0) : pages->size(1);
        }
        check(ls_attend(ctx_, &c, &a));
    }

private:
    ls_ops* ctx_ = nullptr;
    int device_;

    void on_device(const Tensor& t, const char* what) const {
        if (!t.is_cuda()) bad(std::string(what) + " is not on the GPU");
        if (t.device().index() != device_) bad(std::string(what) + " is on another GPU than the context");
    }

    // A tensor of the context's GPU, of the given sizes, whose last dimension is contiguous.
    void shaped(const Tensor& t, at::IntArrayRef sizes, const char* what) const {
        on_device(t, what);
        if (t.sizes() != sizes) bad(std::string(what) + " has the wrong shape");
        if (t.size(-1) > 1 && t.stride(-1) != 1) bad(std::string(what) + " is not contiguous in its last dimension");
    }

    void check(ls_status st) const {
        if (st == LS_OK) return;
        const char* text = ls_ops_last_error(ctx_);
        const py::object error = py::module_::import("paper_2609_03079_amd").attr("LsError")((int)st, text ? text : "");
        PyErr_SetObject((PyObject*)Py_TYPE(error.ptr()), error.ptr());
        throw py::error_already_set();
    }

    const int32_t* indices(const Tensor& t, at::IntArrayRef sizes, const char* what) const {
        expect(t, at::kInt, what);
        shaped(t, sizes, what);
        return static_cast<const int32_t*>(t.const_data_ptr());
    }

    // [n_pages, n_kv_heads, page_size, head_dim], both of the same strides in any order
    ls_kv_cache cache(const Tensor& k, const Tensor& v) const {
        if (k.dim() != 4) bad("k_cache has the wrong shape");
        ls_kv_cache c{};
        c.dtype = type_of(k, "k_cache");
        expect(v, k.scalar_type(), "v_cache");
        shaped(k, k.sizes(), "k_cache");
        shaped(v, k.sizes(), "v_cache");
        for (int i = 0; i < 3; ++i)
            if (step(k, i) != step(v, i)) bad("k_cache and v_cache have different strides");
        c.k = k.data_ptr(), c.v = v.data_ptr();
        c.n_pages = count(k.size(0), "k_cache"), c.n_kv_heads = count(k.size(1), "k_cache");
        c.page_size = count(k.size(2), "k_cache"), c.head_dim = count(k.size(3), "k_cache");
        c.page_stride = step(k, 0), c.head_stride = step(k, 1), c.token_stride = step(k, 2);
        return c;
    }
};

}  // namespace

PYBIND11_MODULE(_lsops, m) {
    m.attr("digest") = LS_BUILD_DIGEST;
    py::class_<Ops>(m, "Ops", py::dynamic_attr())
        .def(py::init<uint64_t, uintptr_t, int>())
        .def("close", &Ops::close)
        .def_property_readonly("ctx", &Ops::ctx)
        .def("ls_ops_sync", &Ops::sync)
        .def("ls_norm_residual", &Ops::norm, py::arg("x"), py::kw_only(), py::arg("y") = py::none(), py::arg("gate") = py::none(),
             py::arg("post_norm") = false, py::arg("post_weight") = py::none(), py::arg("pre_norm") = false,
             py::arg("pre_weight") = py::none(), py::arg("x_scale") = 1.f, py::arg("y_scale") = 1.f, py::arg("eps") = 1e-6f,
             py::arg("x_out") = py::none(), py::arg("h") = py::none(),
             "x, x_out: fp32 [T, d]; y, h: [T, d]; gate: [d] or [T, d]; the weights: [d].")
        .def("ls_linear_i8", &Ops::linear, py::arg("x"), py::arg("w"), py::arg("w_scale"), py::arg("out"), py::kw_only(),
             py::arg("x_scale") = py::none(), py::arg("bias") = py::none(),
             "x: [T, k] int8 with x_scale fp32 [T], or floating; w: int8 [n, k]; w_scale, bias: fp32 [n]; out: [T, n].")
        .def("ls_kv_append", &Ops::append, py::arg("k_cache"), py::arg("v_cache"), py::arg("k"), py::arg("v"), py::arg("positions").none(true),
             py::arg("slots"), py::arg("cos_sin").none(true), py::kw_only(), py::arg("q") = py::none(), py::arg("q_out") = py::none(),
             py::arg("style") = (int)LS_ROPE_HALF,
             "Caches: [n_pages, n_kv_heads, page_size, head_dim], of the same strides in any order; k, v: [T, n_kv_heads, head_dim]; "
             "q, q_out: [T, n_heads, head_dim]; positions, slots: int32 [T]; cos_sin: fp32 [n_pos, rot_dim], or None (with positions "
             "None) for a plain append.")
        .def("ls_attend", &Ops::attend, py::arg("q"), py::arg("k_cache"), py::arg("v_cache"), py::arg("pages").none(true), py::arg("lens"),
             py::arg("out"), py::kw_only(), py::arg("max_len"), py::arg("scale"), py::arg("n_q") = 1, py::arg("prefix_pages") = py::none(),
             py::arg("prefix_len") = 0,
             "q, out: [n_seqs * n_q, n_heads, head_dim]; pages: int32 [n_seqs, pages of a sequence]; lens: int32 [n_seqs]; "
             "prefix_pages: int32 [pages of the prefix]; max_len: a bound of lens that the caller knows.");
}
