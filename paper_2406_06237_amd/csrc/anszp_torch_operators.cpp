// The binding's native calls of the operators that run decoded layers as a model (anszp_torch.cpp has the others).  They check their operands themselves (in Python the checks take longer than a
// small call's launch); whatever is not plainly as documented is declined, and the binding's own path names what is wrong.
//
// They return their tensors, the library's error code, or None where they decline.  The interpreter lock is held only while Python
// objects are read and made.
#include <ATen/ATen.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include <climits>
#include <cmath>
#include <optional>

#include "anszp.h"

namespace {

constexpr int kDeclined = INT_MIN;                          // (no code of the library's)
py::object none() { return py::none(); }
py::object failed(int rc) { return rc == kDeclined ? none() : py::object(py::int_(rc)); }
void* stream_of(uint64_t raw) { return reinterpret_cast<void*>(static_cast<uintptr_t>(raw)); }
template <class T>
T* data(const at::Tensor& t) { return static_cast<T*>(t.data_ptr()); }

using Maybe = std::optional<at::Tensor>;

bool is_float(const at::Tensor& t) { return t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16; }
uint32_t code_of(const at::Tensor& t) {
    return t.scalar_type() == at::kFloat ? ANSZP_OUT_F32 : t.scalar_type() == at::kBFloat16 ? ANSZP_OUT_BF16 : ANSZP_I8;
}
bool packed(const at::Tensor& t) { return t.stride(-1) == 1 || t.size(-1) <= 1; }
bool matrix(const at::Tensor& t, const at::Device& on, int64_t rows, int64_t cols) {
    return t.dim() == 2 && t.device() == on && t.size(0) == rows && t.size(1) == cols && packed(t);
}
bool vector(const at::Tensor& t, const at::Device& on, int64_t n) { return t.dim() == 1 && t.device() == on && t.size(0) == n && packed(t); }
template <class T = void>
T* address(const Maybe& t) { return t ? data<T>(*t) : nullptr; }
uint64_t rows_apart(const at::Tensor& t) { return static_cast<uint64_t>(t.stride(0)); }

// work() without the interpreter lock; a failed allocation is declined
template <class Work>
int unlocked(Work&& work) {
    py::gil_scoped_release released;
    try {
        return work();
    } catch (...) {
        return kDeclined;
    }
}

py::object rms_norm(const at::Tensor& x, const Maybe& weight, double eps, const Maybe& residual, Maybe total, int out_code, uint64_t stream) {
    if (x.dim() != 2 || !is_float(x) || !packed(x)) return none();
    const at::Device on = x.device();
    const int64_t rows = x.size(0), cols = x.size(1);
    if (weight && (!vector(*weight, on, cols) || !is_float(*weight))) return none();
    for (const Maybe* t : {&residual, const_cast<const Maybe*>(&total)})
        if (*t && (!matrix(**t, on, rows, cols) || (*t)->scalar_type() != x.scalar_type())) return none();
    at::Tensor out, scales;
    const int rc = unlocked([&] {
        out = at::empty({rows, cols}, x.options().dtype(out_code == ANSZP_OUT_F32 ? at::kFloat : out_code == ANSZP_OUT_BF16 ? at::kBFloat16 : at::kChar));
        if (out_code == ANSZP_I8) scales = at::empty({rows}, x.options().dtype(at::kFloat));
        if (residual && !total) total = at::empty({rows, cols}, x.options());
        anszp_norm_args_t a = {};
        a.x = x.data_ptr(); a.residual = address(residual); a.total = address(total); a.weight = address(weight); a.out = out.data_ptr();
        a.out_scales = scales.defined() ? data<float>(scales) : nullptr;
        a.rows = uint64_t(rows); a.cols = uint32_t(cols);
        if (cols >= 1ll << 31) return int(kDeclined);
        a.x_stride = rows_apart(x); a.residual_stride = residual ? rows_apart(*residual) : 0u; a.total_stride = total ? rows_apart(*total) : 0u;
        a.out_stride = uint64_t(cols); a.dtype = code_of(x); a.weight_dtype = weight ? code_of(*weight) : 0u; a.out_dtype = uint32_t(out_code);
        a.normalise = weight ? 1u : 0u; a.eps = float(eps);
        return anszp_rms_norm(&a, stream_of(stream));
    });
    if (rc) return failed(rc);
    return py::make_tuple(out, scales.defined() ? py::cast(scales) : none(), total ? py::cast(*total) : none());
}

py::object linear(const at::Tensor& x, const at::Tensor& weight, const Maybe& x_scales, int64_t zero_point, double scale, const Maybe& channel_scales, const Maybe& bias,
                  uint32_t activation, const Maybe& mul, const Maybe& residual, int out_code, Maybe out, uint64_t stream) {
    const bool bytes = x.scalar_type() == at::kChar;
    if (x.dim() != 2 || weight.dim() != 2 || !packed(x) || (!bytes && x.scalar_type() != at::kBFloat16) || zero_point < 0 || zero_point > (bytes ? 255 : 0)) return none();
    const at::Device on = x.device();
    const int64_t rows = x.size(0), k = x.size(1), cols = weight.size(0);
    if (!matrix(weight, on, cols, k) || weight.scalar_type() != (bytes ? at::kByte : at::kBFloat16) || k >= 1ll << 31) return none();
    if (out && (!matrix(*out, on, rows, cols) || !is_float(*out))) return none();
    const at::ScalarType type = out ? out->scalar_type() : out_code == ANSZP_OUT_F32 ? at::kFloat : at::kBFloat16;
    for (const Maybe* t : {&mul, &residual})
        if (*t && (!matrix(**t, on, rows, cols) || (*t)->scalar_type() != type)) return none();
    if (x_scales && (!vector(*x_scales, on, rows) || x_scales->scalar_type() != at::kFloat)) return none();
    for (const Maybe* t : {&channel_scales, &bias})
        if (*t && (!vector(**t, on, cols) || (*t)->scalar_type() != at::kFloat)) return none();
    const int rc = unlocked([&] {
        if (!out) out = at::empty({rows, cols}, x.options().dtype(type));
        anszp_linear_args_t a = {};
        a.x = x.data_ptr(); a.weight = weight.data_ptr(); a.x_scales = address<float>(x_scales); a.channel_scales = address<float>(channel_scales);
        a.bias = address<float>(bias); a.mul = address(mul); a.residual = address(residual); a.out = out->data_ptr();
        a.rows = uint64_t(rows); a.cols = uint64_t(cols); a.k = uint32_t(k);
        a.x_stride = rows_apart(x); a.weight_stride = rows_apart(weight); a.mul_stride = mul ? rows_apart(*mul) : 0u;
        a.residual_stride = residual ? rows_apart(*residual) : 0u; a.out_stride = rows_apart(*out);
        a.x_dtype = code_of(x); a.out_dtype = code_of(*out); a.zero_point = uint32_t(zero_point); a.activation = activation; a.scale = float(scale);
        at::Tensor workspace;
        a.workspace_bytes = anszp_linear_workspace_bytes(&a);
        if (a.workspace_bytes) {
            workspace = at::empty({int64_t(a.workspace_bytes)}, x.options().dtype(at::kByte));
            a.workspace = workspace.data_ptr();
        }
        return anszp_linear(&a, stream_of(stream));
    });
    return rc ? failed(rc) : py::cast(*out);
}

// A cache's tensors (k, k_params, v, v_params) and bits as the library takes them; false: not plainly one.
bool cache_of(const at::Tensor& k, const at::Tensor& kp, const at::Tensor& v, const at::Tensor& vp, int64_t bits, const Maybe& status, anszp_cache_t& c) {
    const at::Device on = k.device();
    if ((bits != 8 && bits != 4) || k.dim() != 4 || k.scalar_type() != at::kByte || v.scalar_type() != at::kByte || kp.scalar_type() != at::kFloat ||
        vp.scalar_type() != at::kFloat || v.device() != on || kp.device() != on || vp.device() != on || v.sizes() != k.sizes() || kp.sizes() != vp.sizes() ||
        kp.dim() != 4 || kp.size(0) != k.size(0) || kp.size(1) != k.size(1) || kp.size(2) != k.size(2) || kp.size(3) != 2 || !k.is_contiguous() ||
        !v.is_contiguous() || !kp.is_contiguous() || !vp.is_contiguous() || k.size(0) >= 1ll << 31 || k.size(1) >= 1 << 16 || k.size(2) > 65536 || k.size(3) > 256)
        return false;
    if (status && (!vector(*status, on, 2) || status->scalar_type() != at::kInt)) return false;
    c.k = data<uint8_t>(k); c.k_params = data<float>(kp); c.v = data<uint8_t>(v); c.v_params = data<float>(vp);
    c.n_pages = uint64_t(k.size(0)); c.heads = uint32_t(k.size(1)); c.page_size = uint32_t(k.size(2)); c.head_dim = uint32_t(k.size(3) * 8 / bits); c.bits = uint32_t(bits);
    return true;
}

py::object cache_write(const at::Tensor& ck, const at::Tensor& ckp, const at::Tensor& cv, const at::Tensor& cvp, int64_t bits, const Maybe& status, const at::Tensor& k,
                       const at::Tensor& v, const at::Tensor& slots, uint64_t stream) {
    anszp_cache_t c;
    if (!cache_of(ck, ckp, cv, cvp, bits, status, c) || k.dim() != 3 || !is_float(k) || v.scalar_type() != k.scalar_type() || v.sizes() != k.sizes() || !packed(k) ||
        !packed(v) || k.device() != ck.device() || v.device() != ck.device() || k.size(1) != c.heads || k.size(2) != c.head_dim ||
        !vector(slots, ck.device(), k.size(0)) || slots.scalar_type() != at::kLong)
        return none();
    const int rc = unlocked([&] {
        return anszp_cache_write(&c, k.data_ptr(), v.data_ptr(), code_of(k), uint64_t(k.stride(0)), uint64_t(k.stride(1)), uint64_t(v.stride(0)), uint64_t(v.stride(1)),
                                 data<int64_t>(slots), uint64_t(k.size(0)), address<uint32_t>(status), stream_of(stream));
    });
    return rc ? failed(rc) : py::object(py::bool_(true));
}

py::object cache_read(const at::Tensor& ck, const at::Tensor& ckp, const at::Tensor& cv, const at::Tensor& cvp, int64_t bits, const Maybe& status, const at::Tensor& slots,
                      int out_code, uint64_t stream) {
    anszp_cache_t c;
    if (!cache_of(ck, ckp, cv, cvp, bits, status, c) || slots.dim() != 1 || !vector(slots, ck.device(), slots.size(0)) || slots.scalar_type() != at::kLong) return none();
    at::Tensor k, v;
    const int rc = unlocked([&] {
        const at::TensorOptions like = ckp.options().dtype(out_code == ANSZP_OUT_F32 ? at::kFloat : at::kBFloat16);
        k = at::empty({slots.size(0), c.heads, c.head_dim}, like);
        v = at::empty({slots.size(0), c.heads, c.head_dim}, like);
        return anszp_cache_read(&c, k.data_ptr(), v.data_ptr(), uint32_t(out_code), data<int64_t>(slots), uint64_t(slots.size(0)), address<uint32_t>(status), stream_of(stream));
    });
    return rc ? failed(rc) : py::object(py::make_tuple(k, v));
}

py::object attend(const at::Tensor& q, const at::Tensor& ck, const at::Tensor& ckp, const at::Tensor& cv, const at::Tensor& cvp, int64_t bits, const Maybe& status,
                  const at::Tensor& pages, const at::Tensor& lengths, const at::Tensor& starts, std::optional<double> scale, int out_code, Maybe out, uint64_t stream) {
    anszp_attend_args_t a = {};
    const at::Device on = q.device();
    if (ck.device() != on || !cache_of(ck, ckp, cv, cvp, bits, status, a.cache) || q.dim() != 3 || q.scalar_type() != at::kBFloat16 || !packed(q) || a.cache.heads == 0 ||
        q.size(1) == 0 || q.size(1) % a.cache.heads || q.size(1) / a.cache.heads > 256 || q.size(2) != a.cache.head_dim || pages.dim() != 2 ||
        pages.scalar_type() != at::kInt || pages.device() != on || !pages.is_contiguous() || pages.size(1) > 1ll << 30 || !vector(lengths, on, pages.size(0)) ||
        lengths.scalar_type() != at::kInt || !vector(starts, on, pages.size(0) + 1) || starts.scalar_type() != at::kInt)
        return none();
    if (out && (out->device() != on || out->sizes() != q.sizes() || !is_float(*out) || !packed(*out))) return none();
    const int rc = unlocked([&] {
        if (!out) out = at::empty(q.sizes(), q.options().dtype(out_code == ANSZP_OUT_F32 ? at::kFloat : at::kBFloat16));
        a.q = q.data_ptr(); a.out = out->data_ptr(); a.pages = data<int32_t>(pages); a.lengths = data<int32_t>(lengths); a.starts = data<int32_t>(starts);
        a.status = address<uint32_t>(status); a.n_tokens = uint64_t(q.size(0)); a.n_seqs = uint64_t(pages.size(0)); a.table_width = uint32_t(pages.size(1));
        a.group = uint32_t(q.size(1) / a.cache.heads); a.q_token_stride = uint64_t(q.stride(0)); a.q_head_stride = uint64_t(q.stride(1));
        a.out_token_stride = uint64_t(out->stride(0)); a.out_head_stride = uint64_t(out->stride(1)); a.out_dtype = code_of(*out);
        a.scale = scale ? float(*scale) : 1.0f / std::sqrt(float(a.cache.head_dim));
        at::Tensor workspace;
        a.workspace_bytes = anszp_attend_workspace_bytes(&a);
        if (a.workspace_bytes) {
            workspace = at::empty({int64_t(a.workspace_bytes)}, ck.options());
            a.workspace = workspace.data_ptr();
        }
        return anszp_attend(&a, stream_of(stream));
    });
    return rc ? failed(rc) : py::cast(*out);
}

bool ints(const at::Tensor& t, const at::Device& on, int64_t n) { return vector(t, on, n) && t.scalar_type() == at::kInt; }
bool floats(const at::Tensor& t, const at::Device& on, int64_t n) { return vector(t, on, n) && t.scalar_type() == at::kFloat; }

py::object place_tokens(const at::Tensor& pages, int64_t page_size, const at::Tensor& lengths, const at::Tensor& fresh, const at::Tensor& free, const at::Tensor& n_free,
                        int64_t n_tokens, const Maybe& ends, Maybe lengths_out, Maybe n_free_out, const Maybe& status, const Maybe& last, uint64_t stream) {
    const at::Device on = pages.device();
    if (pages.dim() != 2 || pages.scalar_type() != at::kInt || !pages.is_contiguous() || pages.size(1) > 1ll << 30 || page_size < 0 || page_size > 65536 || n_tokens < 0 ||
        n_tokens >= 1ll << 31 || free.dim() != 1 || free.size(0) >= 1ll << 31)
        return none();
    const int64_t n = pages.size(0);
    if (!ints(lengths, on, n) || !ints(fresh, on, n) || !ints(free, on, free.size(0)) || !ints(n_free, on, 1) || (ends && !ints(*ends, on, n)) ||
        (lengths_out && !ints(*lengths_out, on, n)) || (n_free_out && !ints(*n_free_out, on, 1)) || (status && !ints(*status, on, 2)) || (last && !ints(*last, on, n)))
        return none();
    at::Tensor slots, owners, starts;
    const int rc = unlocked([&] {
        slots = at::empty({n_tokens}, pages.options().dtype(at::kLong));
        owners = at::empty({n_tokens}, pages.options());
        starts = at::empty({n + 1}, pages.options());
        if (!lengths_out) lengths_out = at::empty({n}, pages.options());
        if (!n_free_out) n_free_out = at::empty({1}, pages.options());
        anszp_place_args_t a = {};
        a.pages = data<int32_t>(pages); a.lengths = data<int32_t>(lengths); a.lengths_out = address<int32_t>(lengths_out); a.new_tokens = data<int32_t>(fresh);
        a.ends = address<int32_t>(ends); a.free_pages = data<int32_t>(free); a.n_free = data<int32_t>(n_free); a.n_free_out = address<int32_t>(n_free_out);
        a.slots = data<int64_t>(slots); a.owners = data<int32_t>(owners); a.starts = data<int32_t>(starts); a.status = address<uint32_t>(status);
        a.last = address<int32_t>(last);
        a.n_seqs = uint64_t(n); a.n_tokens = uint64_t(n_tokens); a.free_room = uint64_t(free.size(0)); a.table_width = uint32_t(pages.size(1)); a.page_size = uint32_t(page_size);
        at::Tensor workspace;
        a.workspace_bytes = anszp_place_workspace_bytes(&a);
        if (a.workspace_bytes) {
            workspace = at::empty({int64_t(a.workspace_bytes)}, pages.options().dtype(at::kByte));
            a.workspace = workspace.data_ptr();
        }
        return anszp_place(&a, stream_of(stream));
    });
    return rc ? failed(rc) : py::object(py::make_tuple(slots, starts, *lengths_out, owners, *n_free_out));
}

py::object embed(const at::Tensor& tokens, const at::Tensor& weight, int64_t zero_point, const Maybe& row_scales, double scale, int out_code, Maybe out, const Maybe& status,
                 uint64_t stream) {
    const at::Device on = tokens.device();
    const bool symbols = weight.scalar_type() == at::kByte;
    if (tokens.dim() != 1 || tokens.scalar_type() != at::kLong || !packed(tokens) || weight.dim() != 2 || weight.device() != on || !packed(weight) ||
        (!symbols && weight.scalar_type() != at::kBFloat16) || zero_point < 0 || zero_point > (symbols ? 255 : 0) || weight.size(1) >= 1ll << 31 ||
        (row_scales && (!symbols || !floats(*row_scales, on, weight.size(0)))) || (status && !ints(*status, on, 2)))
        return none();
    const int64_t n = tokens.size(0), cols = weight.size(1);
    if (out && (!matrix(*out, on, n, cols) || !is_float(*out))) return none();
    const int rc = unlocked([&] {
        if (!out) out = at::empty({n, cols}, weight.options().dtype(out_code == ANSZP_OUT_F32 ? at::kFloat : at::kBFloat16));
        anszp_embed_args_t a = {};
        a.tokens = data<int64_t>(tokens); a.weight = weight.data_ptr(); a.row_scales = address<float>(row_scales); a.out = out->data_ptr(); a.status = address<uint32_t>(status);
        a.n_tokens = uint64_t(n); a.vocabulary = uint64_t(weight.size(0)); a.weight_stride = rows_apart(weight); a.out_stride = rows_apart(*out); a.cols = uint32_t(cols);
        a.weight_dtype = symbols ? ANSZP_OUT_U8 : ANSZP_OUT_BF16; a.zero_point = uint32_t(zero_point); a.out_dtype = code_of(*out); a.scale = float(scale);
        return anszp_embed(&a, stream_of(stream));
    });
    return rc ? failed(rc) : py::cast(*out);
}

py::object adapt(const at::Tensor& base, const at::Tensor& x, const at::Tensor& wa, const at::Tensor& wb, const at::Tensor& ids, const Maybe& x_scales, const Maybe& scales,
                 uint32_t activation, const Maybe& mul, const Maybe& residual, int out_code, Maybe out, const Maybe& status, uint64_t stream) {
    const at::Device on = base.device();
    if (base.dim() != 2 || !is_float(base) || !packed(base) || x.dim() != 2 || wa.dim() != 3 || wb.dim() != 3) return none();
    const int64_t rows = base.size(0), cols = base.size(1), k = x.size(1), n = wa.size(0), rank = wa.size(1);
    if (!matrix(x, on, rows, k) || (x.scalar_type() != at::kChar && x.scalar_type() != at::kBFloat16) || wa.device() != on || wb.device() != on ||
        wa.scalar_type() != at::kBFloat16 || wb.scalar_type() != at::kBFloat16 || wa.size(2) != k || wb.size(0) != n || wb.size(1) != cols || wb.size(2) != rank ||
        !packed(wa) || !packed(wb) || !ints(ids, on, rows) || k >= 1ll << 31 || rank > 128 || n >= 1ll << 24)
        return none();
    if (out && (!matrix(*out, on, rows, cols) || !is_float(*out))) return none();
    const at::ScalarType type = out ? out->scalar_type() : out_code == ANSZP_OUT_F32 ? at::kFloat : at::kBFloat16;
    for (const Maybe* t : {&mul, &residual})
        if (*t && (!matrix(**t, on, rows, cols) || (*t)->scalar_type() != type)) return none();
    if ((x_scales && !floats(*x_scales, on, rows)) || (scales && !floats(*scales, on, n)) || (status && !ints(*status, on, 2))) return none();
    const int rc = unlocked([&] {
        if (!out) out = at::empty({rows, cols}, base.options().dtype(type));
        anszp_adapt_args_t a = {};
        a.x = x.data_ptr(); a.a = wa.data_ptr(); a.b = wb.data_ptr(); a.ids = data<int32_t>(ids); a.x_scales = address<float>(x_scales); a.scales = address<float>(scales);
        a.base = base.data_ptr(); a.mul = address(mul); a.residual = address(residual); a.out = out->data_ptr(); a.status = address<uint32_t>(status);
        a.rows = uint64_t(rows); a.cols = uint64_t(cols); a.x_stride = rows_apart(x); a.a_stride = rows_apart(wa); a.a_row_stride = uint64_t(wa.stride(1));
        a.b_stride = rows_apart(wb); a.b_row_stride = uint64_t(wb.stride(1)); a.base_stride = rows_apart(base); a.mul_stride = mul ? rows_apart(*mul) : 0u;
        a.residual_stride = residual ? rows_apart(*residual) : 0u; a.out_stride = rows_apart(*out); a.adapters = uint32_t(n); a.k = uint32_t(k); a.rank = uint32_t(rank);
        a.x_dtype = code_of(x); a.base_dtype = code_of(base); a.out_dtype = code_of(*out); a.activation = activation;
        at::Tensor workspace;
        a.workspace_bytes = anszp_adapt_workspace_bytes(&a);
        if (a.workspace_bytes) {
            workspace = at::empty({int64_t(a.workspace_bytes)}, base.options().dtype(at::kByte));
            a.workspace = workspace.data_ptr();
        }
        return anszp_adapt(&a, stream_of(stream));
    });
    return rc ? failed(rc) : py::cast(*out);
}

// A setting is a number for all rows, or a tensor with one for each; false: neither.
bool setting(const py::object& given, const at::Device& on, int64_t rows, at::ScalarType type, Maybe& each, double& all) {
    if (THPVariable_Check(given.ptr())) {
        each = THPVariable_Unpack(given.ptr());
        return vector(*each, on, rows) && each->scalar_type() == type;
    }
    if (!PyFloat_Check(given.ptr()) && !PyLong_Check(given.ptr())) return false;
    all = PyFloat_AsDouble(given.ptr());
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return type == at::kFloat || (all >= 0.0 && all < 2147483648.0 && PyLong_Check(given.ptr()));
}

py::object sample(const at::Tensor& logits, const at::Tensor& uniforms, const py::object& temperature, const py::object& top_k, const py::object& top_p, const py::object& min_p,
                  Maybe tokens, uint64_t stream) {
    const at::Device on = logits.device();
    if (logits.dim() != 2 || !is_float(logits) || !packed(logits) || logits.size(1) > 1ll << 24) return none();
    const int64_t rows = logits.size(0);
    Maybe temperatures, top_ks, top_ps, min_ps;
    double t = 1.0, k = 0.0, tp = 1.0, mp = 0.0;
    if (!floats(uniforms, on, rows) || !setting(temperature, on, rows, at::kFloat, temperatures, t) || !setting(top_k, on, rows, at::kInt, top_ks, k) ||
        !setting(top_p, on, rows, at::kFloat, top_ps, tp) || !setting(min_p, on, rows, at::kFloat, min_ps, mp) || !(t >= 0.0) || !(tp >= 0.0) || !(mp >= 0.0))
        return none();
    if (tokens && (!vector(*tokens, on, rows) || tokens->scalar_type() != at::kLong)) return none();
    at::Tensor chances;
    const int rc = unlocked([&] {
        if (!tokens) tokens = at::empty({rows}, logits.options().dtype(at::kLong));
        chances = at::empty({rows}, logits.options().dtype(at::kFloat));
        anszp_sample_args_t a = {};
        a.logits = logits.data_ptr(); a.uniforms = data<float>(uniforms); a.temperatures = address<float>(temperatures); a.top_ks = address<int32_t>(top_ks);
        a.top_ps = address<float>(top_ps); a.min_ps = address<float>(min_ps); a.tokens = address<int64_t>(tokens); a.chances = data<float>(chances);
        a.rows = uint64_t(rows); a.logits_stride = rows_apart(logits); a.vocabulary = uint32_t(logits.size(1)); a.dtype = code_of(logits);
        a.temperature = float(t); a.top_k = int32_t(k); a.top_p = float(tp); a.min_p = float(mp);
        return anszp_sample(&a, stream_of(stream));
    });
    return rc ? failed(rc) : py::object(py::make_tuple(*tokens, chances));
}

}  // namespace

PYBIND11_MODULE(_anszp_operators, m) {
    m.def("rms_norm", &rms_norm);
    m.def("linear", &linear);
    m.def("cache_write", &cache_write);
    m.def("cache_read", &cache_read);
    m.def("attend", &attend);
    m.def("place_tokens", &place_tokens);
    m.def("embed", &embed);
    m.def("adapt", &adapt);
    m.def("sample", &sample);
}
