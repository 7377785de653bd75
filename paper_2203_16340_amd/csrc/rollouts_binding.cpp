// Python's way into what makes rollouts: products with 4-bit weights, tokens drawn, drafts verified.  As in losses_binding.cpp, every function
// returns the C entry's code first.
#include "binding.h"

namespace {

Tensor workspace(size_t n, const at::Device& dev) {
    return n ? at::empty({(int64_t)n}, at::TensorOptions(dev).dtype(at::kByte)) : Tensor();
}
Tensor longs(at::IntArrayRef shape, const at::Device& dev) { return at::empty(shape, at::TensorOptions(dev).dtype(at::kLong)); }
Tensor floats(at::IntArrayRef shape, const at::Device& dev) { return at::empty(shape, at::TensorOptions(dev).dtype(at::kFloat)); }

// the address of a contiguous tensor of this shape
template <typename T>
T* grid(const Tensor& t, const char* name, at::IntArrayRef shape, const at::Device& dev, at::ScalarType type) {
    if (t.scalar_type() != type || t.device() != dev || !t.is_contiguous())
        throw py::type_error(std::string(name) + " must be a contiguous " + c10::toString(type) + " tensor on " + dev.str());
    if (t.sizes() != shape) {
        std::string want;
        for (const int64_t n : shape) want += (want.empty() ? "" : ", ") + std::to_string(n);
        throw py::value_error(std::string(name) + " must have the shape (" + want + ")");
    }
    return (T*)t.data_ptr();
}

lbfgsb_weights4 weights_of(int64_t rows, int64_t cols, int64_t group, int scale_type, bool zero) {
    // (matvec4 and the sizes look at whether there are zeros only)
    return {rows, cols, group, scale_type, nullptr, nullptr, zero ? (const void*)16 : nullptr};
}
int64_t groups_of(int64_t cols, int64_t group) { return group > 0 ? (cols + group - 1) / group : 0; }

auto quantize4(const Tensor& w, int64_t group, bool symmetric, py::object scale_dtype, int64_t stream) {
    const int type = logit_type(w, "weight");
    const auto dtype = scale_dtype.is_none() ? w.scalar_type() : torch::python::detail::py_object_to_dtype(scale_dtype);
    const int64_t rows = w.size(0), cols = w.size(1);
    lbfgsb_weights4 to = weights_of(rows, cols, group, type_code(dtype), !symmetric);
    if (lbfgsb_packed4_bytes(&to) == 0) return std::make_tuple((int)LBFGSB_E_INVALID_ARG, Tensor(), Tensor(), Maybe());
    Tensor codes = at::empty({rows, (cols + 1) / 2}, w.options().dtype(at::kByte));
    Tensor scale = at::empty({rows, groups_of(cols, group)}, w.options().dtype(dtype));
    Maybe zero;
    if (!symmetric) zero = at::empty_like(scale);
    to.codes = (const uint8_t*)codes.data_ptr();
    to.scale = scale.data_ptr();
    to.zero = zero ? zero->data_ptr() : nullptr;
    const int rc = lbfgsb_quantize4(type, row_stride(w), w.data_ptr(), &to, (void*)stream);
    return std::make_tuple(rc, codes, scale, zero);
}

auto pack4(const Tensor& codes, const Tensor& scale, const Maybe& zero, int64_t cols, int64_t group, int64_t stream) {
    const at::Device dev = codes.device();
    const int type = logit_type(scale, "scale");
    const int64_t rows = codes.dim() == 2 ? codes.size(0) : -1;
    lbfgsb_weights4 w = weights_of(rows, cols, group, type, zero.has_value());
    const size_t n = lbfgsb_packed4_bytes(&w);
    if (n == 0) return std::make_tuple((int)LBFGSB_E_INVALID_ARG, Tensor(), type);
    w.codes = grid<uint8_t>(codes, "codes", {rows, (cols + 1) / 2}, dev, at::kByte);
    w.scale = grid<void>(scale, "scale", {rows, groups_of(cols, group)}, dev, scale.scalar_type());
    w.zero = zero ? grid<void>(*zero, "zero", {rows, groups_of(cols, group)}, dev, scale.scalar_type()) : nullptr;
    Tensor packed = workspace(n, dev);
    const int rc = lbfgsb_pack4(&w, packed.data_ptr(), n, (void*)stream);
    return std::make_tuple(rc, packed, type);
}

// Whether the tensor holds what the products read of weights of these sizes (lbfgsb_matvec4 has only its address).  False: the sizes are of no weights.
bool holds(const Tensor& packed, const lbfgsb_weights4& w) {
    const size_t need = lbfgsb_packed4_bytes(&w);
    if (need == 0) return false;
    if (packed.scalar_type() != at::kByte || !packed.is_contiguous()) throw py::type_error("the packed weights must be a contiguous Byte tensor");
    if ((size_t)packed.numel() < need)
        throw py::value_error("the packed weights must have " + std::to_string(need) + " bytes for their rows, cols, group, scales and zeros, got " +
                              std::to_string(packed.numel()));
    return true;
}

auto matvec4(const Tensor& x, const Tensor& packed, int64_t rows, int64_t cols, int64_t group, int scale_type, bool zero, py::object dtype,
             const Maybe& out, int64_t stream) {
    const lbfgsb_weights4 w = weights_of(rows, cols, group, scale_type, zero);
    if (!holds(packed, w)) return std::make_tuple((int)LBFGSB_E_INVALID_ARG, Tensor());
    const int x_type = logit_type(x, "x");
    const at::Device dev = x.device();
    if (x.size(1) != cols) throw py::value_error("x must have " + std::to_string(cols) + " columns, got " + std::to_string(x.size(1)));
    if (packed.device() != dev) throw py::type_error("x and the weights must be on the same device");
    Tensor y;
    if (out) {
        logit_type(*out, "out");
        if (out->size(0) != x.size(0) || out->size(1) != rows || out->device() != dev)
            throw py::type_error("out must be (" + std::to_string(x.size(0)) + ", " + std::to_string(rows) + ") on " + dev.str());
        if (!dtype.is_none() && torch::python::detail::py_object_to_dtype(dtype) != out->scalar_type()) throw py::type_error("dtype is not that of out");
        y = *out;
    } else {
        const auto type = dtype.is_none() ? x.scalar_type() : torch::python::detail::py_object_to_dtype(dtype);
        if (type != x.scalar_type() && type != at::kFloat) throw py::type_error("dtype must be that of x or float32");
        y = at::empty({x.size(0), rows}, x.options().dtype(type));
    }
    Tensor ws = workspace(lbfgsb_matvec4_workspace_bytes(&w, x.size(0), x_type), dev);
    const int rc = lbfgsb_matvec4(&w, packed.data_ptr(), x.size(0), x_type, row_stride(x), x.data_ptr(), type_code(y.scalar_type()), row_stride(y), y.data_ptr(),
                                  address(ws), bytes(ws), (void*)stream);
    if (rc == LBFGSB_OK && out) written(y);
    return std::make_tuple(rc, y);
}

auto draw_tokens(const Tensor& z, const Tensor& uniform, double temperature, int64_t stream) {
    lbfgsb_logits lg;
    const at::Device dev = z.device();
    lg.dtype = logit_type(z, "logits");
    lg.rows = z.size(0);
    lg.vocab = z.size(1);
    lg.ld = row_stride(z);
    lg.z = z.data_ptr();
    lg.temperature = temperature;
    lg.grad = nullptr;
    lg.ld_grad = 0;
    const float* u = vec(uniform, "uniform", lg.rows, dev);
    Tensor tokens = longs({lg.rows}, dev), logp = floats({lg.rows}, dev), ws = workspace(lbfgsb_draw_workspace_bytes(&lg), dev);
    const int rc = lbfgsb_draw_tokens(&lg, u, (int64_t*)tokens.data_ptr(), (float*)logp.data_ptr(), address(ws), bytes(ws), (void*)stream);
    return std::make_tuple(rc, tokens, logp);
}

// a (requests, positions, vocab) tensor with unit stride of its last dimension
int check_positions(const Tensor& z, const char* name) {
    const int type = type_code(z.scalar_type());
    if (type < 0 || !z.is_cuda() || z.dim() != 3 || (z.stride(2) != 1 && z.size(2) != 1))
        throw py::type_error(std::string(name) + " must be a 3-d float32/bfloat16/float16 CUDA tensor with unit stride of its last dimension");
    return type;
}

auto verify_draft(const Tensor& z, const Tensor& drafted, const Tensor& uniform, const Tensor& last_uniform, const Maybe& draft_logits,
                  const Maybe& draft_logp, const Maybe& lengths, double temperature, double draft_temperature, int64_t stream) {
    lbfgsb_drafts d;
    const at::Device dev = z.device();
    d.dtype = check_positions(z, "logits");
    if (z.size(1) < 1) throw py::value_error("logits must have one position more than there are drafts");
    const int64_t n = d.requests = z.size(0), k = d.drafts = z.size(1) - 1;
    d.vocab = z.size(2);
    d.z = z.data_ptr();
    d.ld = z.stride(1);
    d.ld_request = z.stride(0);
    d.temperature = temperature;
    d.draft_z = nullptr;
    d.draft_ld = d.draft_ld_request = d.vocab;
    d.draft_temperature = draft_temperature;
    if (draft_logits) {
        if (check_positions(*draft_logits, "draft_logits") != d.dtype || draft_logits->device() != dev)
            throw py::type_error("draft_logits must have the type and device of the logits");
        if (draft_logits->size(0) != n || draft_logits->size(1) != k || draft_logits->size(2) != d.vocab)
            throw py::value_error("draft_logits must have the shape (" + std::to_string(n) + ", " + std::to_string(k) + ", " + std::to_string(d.vocab) + ")");
        d.draft_z = draft_logits->data_ptr();
        d.draft_ld = draft_logits->stride(1);
        d.draft_ld_request = draft_logits->stride(0);
    } else if (draft_logp) {
        throw py::value_error("draft_logp goes with draft_logits");
    }
    d.drafted = grid<int64_t>(drafted, "drafted", {n, k}, dev, at::kLong);
    d.uniform = grid<float>(uniform, "uniform", {n, k}, dev, at::kFloat);
    d.last_uniform = grid<float>(last_uniform, "last_uniform", {n}, dev, at::kFloat);
    d.draft_logp = draft_logp ? grid<float>(*draft_logp, "draft_logp", {n, k}, dev, at::kFloat) : nullptr;
    d.lengths = lengths ? grid<int64_t>(*lengths, "lengths", {n}, dev, at::kLong) : nullptr;
    Tensor tokens = longs({n, k + 1}, dev), count = longs({n}, dev), logp = floats({n, k + 1}, dev);
    Tensor ws = workspace(lbfgsb_verify_workspace_bytes(&d), dev);
    const int rc = lbfgsb_verify_draft(&d, (int64_t*)tokens.data_ptr(), (int64_t*)count.data_ptr(), (float*)logp.data_ptr(), address(ws), bytes(ws), (void*)stream);
    return std::make_tuple(rc, tokens, count, logp);
}

}  // namespace

void add_rollouts(py::module_& m) {
    m.def("quantize4", &quantize4);
    m.def("pack4", &pack4);
    m.def("matvec4", &matvec4);
    m.def("draw_tokens", &draw_tokens);
    m.def("verify_draft", &verify_draft);
}
