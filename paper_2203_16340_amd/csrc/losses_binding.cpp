// Python's way into the losses on logits: checks of the tensors, new tensors for the results and the C call, in one step.  (The calls
// take some 3 us each to enqueue what they do; made from Python, the rest of a call on a few rows took 8 to 13 us.)  Every function returns
// the C entry's code first; what the code says is the caller's to raise.
#include "binding.h"

namespace {

struct Call {
    lbfgsb_logits lg;
    Maybe grad;
    at::Device dev;
    int64_t rows;
    bool given = false;      // the gradient is the caller's tensor
    // want: a new gradient; out: one to write to
    Call(const Tensor& z, double temperature, bool want, const Maybe& out) : dev(z.device()), rows(0) {
        lg.dtype = logit_type(z, "logits");
        rows = lg.rows = z.size(0);
        lg.vocab = z.size(1);
        lg.ld = row_stride(z);
        lg.z = z.data_ptr();
        lg.temperature = temperature;
        if (out) {
            if (logit_type(*out, "grad") != lg.dtype || out->sizes() != z.sizes() || out->device() != dev)
                throw py::type_error("grad must have the type, shape and device of the logits");
            grad = out;
            given = true;
        } else if (want) {
            grad = at::empty(z.sizes(), z.options());
        }
        lg.grad = grad ? grad->data_ptr() : nullptr;
        lg.ld_grad = grad ? row_stride(*grad) : 0;
    }
    int done(int rc) const {
        if (rc == LBFGSB_OK && given) written(*grad);
        return rc;
    }
    Tensor rows_of_floats() const { return at::empty({rows}, at::TensorOptions(dev).dtype(at::kFloat)); }
    Tensor number() const { return at::empty({}, at::TensorOptions(dev).dtype(at::kFloat)); }
    // (torch's allocator keeps the memory until the stream is done with it)
    Tensor workspace(bool with_grad) const {
        lbfgsb_logits q = lg;
        if (!with_grad) q.grad = nullptr;
        const int64_t n = (int64_t)lbfgsb_logits_workspace_bytes(&q);
        return n ? at::empty({n}, at::TensorOptions(dev).dtype(at::kByte)) : Tensor();
    }
};
auto token_logprob(const Tensor& z, const Tensor& labels, double temperature, bool entropy, int64_t stream) {
    const Call c(z, temperature, false, std::nullopt);
    const int64_t* y = vec<int64_t>(labels, "labels", c.rows, c.dev, at::kLong);
    Tensor logp = c.rows_of_floats(), ws = c.workspace(false);
    // The other results in one piece of memory: every row's largest logit and its sum (what the way back reads), lse, lse_rest, the entropy.
    // (Each tensor of its own would cost a call 0.4 us more; 8 x 32768 takes 5.9.)
    Tensor all = at::empty({entropy ? 5 : 4, c.rows}, logp.options());
    std::vector<Tensor> part;
    {
        at::AutoDispatchBelowADInplaceOrView plain;
        part = all.unbind(0);
    }
    float* at_row = (float*)all.data_ptr();
    const int64_t n = c.rows;
    const int rc = lbfgsb_token_logprob_stats(&c.lg, y, (float*)logp.data_ptr(), at_row + 2 * n, at_row + 3 * n, entropy ? at_row + 4 * n : nullptr,
                                              at_row, at_row + n, address(ws), bytes(ws), (void*)stream);
    return std::make_tuple(rc, logp, part[2], part[3], entropy ? Maybe(part[4]) : Maybe(), all);
}

auto token_logprob_grad(const Tensor& z, const Tensor& labels, const Tensor& lse, const Maybe& lse_rest, const Maybe& entropy,
                        const Maybe& stats, const Tensor& d_logp, const Maybe& d_entropy, double temperature, const Maybe& out, int64_t stream) {
    const Call c(z, temperature, true, out);
    const int64_t* y = vec<int64_t>(labels, "labels", c.rows, c.dev, at::kLong);
    const float *l = vec(lse, "lse", c.rows, c.dev), *l_rest = maybe(lse_rest, "lse_rest", c.rows, c.dev);
    const float *h = maybe(entropy, "entropy", c.rows, c.dev), *d = vec(d_logp, "d_logp", c.rows, c.dev);
    const float* dh = maybe(d_entropy, "d_entropy", c.rows, c.dev);
    int rc;
    if (stats) {
        if (stats->scalar_type() != at::kFloat || stats->device() != c.dev || !stats->is_contiguous() || stats->dim() != 2 ||
            stats->size(0) < 2 || stats->size(1) != c.rows)
            throw py::type_error("stats must be what token_logprob returned for these logits");
        const float* top = (const float*)stats->data_ptr();
        rc = lbfgsb_token_logprob_stats_grad(&c.lg, y, top, top + c.rows, h, d, dh, (void*)stream);
    } else {
        rc = lbfgsb_token_logprob_grad(&c.lg, y, l, l_rest, h, d, dh, (void*)stream);
    }
    return std::make_tuple(c.done(rc), *c.grad);
}

auto distill_loss(const Tensor& z, const Tensor& index, const Tensor& logit, const Maybe& lse, const Maybe& weight, double temperature,
                  double scale, bool want, const Maybe& out, int64_t stream) {
    const Call c(z, temperature, want, out);
    lbfgsb_teacher t;
    t.logit_type = logit_type(logit, "teacher_logit");
    if ((index.scalar_type() != at::kInt && index.scalar_type() != at::kLong) || index.dim() != 2 || (index.stride(1) != 1 && index.size(1) != 1))
        throw py::type_error("teacher_index must be a 2-d int32/int64 tensor with unit column stride");
    if (index.sizes() != logit.sizes() || index.size(0) != c.rows)
        throw py::value_error("teacher_index and teacher_logit must both be (" + std::to_string(c.rows) + ", top)");
    if (index.device() != c.dev || logit.device() != c.dev) throw py::type_error("the teacher's tensors must be on " + c.dev.str());
    if (row_stride(index) != row_stride(logit)) throw py::value_error("teacher_index and teacher_logit must have the same row stride");
    t.index_type = index.scalar_type() == at::kInt ? LBFGSB_I32 : LBFGSB_I64;
    t.top = index.size(1);
    t.ld = row_stride(index);
    t.index = index.data_ptr();
    t.logit = logit.data_ptr();
    t.lse = maybe(lse, "teacher_lse", c.rows, c.dev);
    const float* w = maybe(weight, "weight", c.rows, c.dev);
    Tensor loss = c.number(), row = c.rows_of_floats(), ws = c.workspace(true);
    const int rc = lbfgsb_distill_loss(&c.lg, &t, w, scale, (float*)loss.data_ptr(), (float*)row.data_ptr(), address(ws), bytes(ws), (void*)stream);
    return std::make_tuple(c.done(rc), loss, row, c.grad);
}

auto policy_loss(const Tensor& z, const Tensor& labels, const Tensor& old_logp, const Tensor& advantage, const Maybe& ref_logp,
                 const Maybe& weight, double clip_low, double clip_high, double kl_coef, int kl_kind, double entropy_coef, bool entropy,
                 double temperature, double scale, bool want, const Maybe& out, int64_t stream) {
    const Call c(z, temperature, want, out);
    const lbfgsb_rollout p{vec<int64_t>(labels, "labels", c.rows, c.dev, at::kLong), vec(old_logp, "old_logp", c.rows, c.dev),
                           vec(advantage, "advantage", c.rows, c.dev), maybe(ref_logp, "ref_logp", c.rows, c.dev),
                           maybe(weight, "weight", c.rows, c.dev)};
    const lbfgsb_policy_options o{clip_low, clip_high, kl_coef, entropy_coef, kl_kind};
    Tensor loss = c.number(), row = c.rows_of_floats(), logp = c.rows_of_floats(), ws = c.workspace(true);
    Maybe h;
    if (entropy) h = c.rows_of_floats();
    const int rc = lbfgsb_policy_loss(&c.lg, &p, &o, scale, (float*)loss.data_ptr(), (float*)row.data_ptr(), (float*)logp.data_ptr(),
                                      h ? (float*)h->data_ptr() : nullptr, address(ws), bytes(ws), (void*)stream);
    return std::make_tuple(c.done(rc), loss, row, logp, h, c.grad);
}

auto preference_loss(const Tensor& logp, const Maybe& ref_logp, const Tensor& offsets, const Maybe& mask, const Maybe& weight, double beta, int kind,
                     double label_smoothing, double margin, bool length_normalised, double scale, bool want, int64_t stream) {
    if (!logp.is_cuda()) throw py::type_error("logp must be a CUDA tensor");
    if (offsets.dim() != 1 || offsets.size(0) % 2 != 1) throw py::value_error("offsets must have 2 * pairs + 1 entries");
    const at::Device dev = logp.device();
    const int64_t n = logp.numel(), pairs = offsets.size(0) / 2;
    const lbfgsb_preference_options o{kind, length_normalised ? 1 : 0, beta, label_smoothing, margin};
    const float* l = vec(logp, "logp", n, dev);
    const float* r = maybe(ref_logp, "ref_logp", n, dev);
    const int64_t* off = vec<int64_t>(offsets, "offsets", 2 * pairs + 1, dev, at::kLong);
    const uint8_t* m = mask ? vec<uint8_t>(*mask, "mask", n, dev, mask->scalar_type() == at::kBool ? at::kBool : at::kByte) : nullptr;
    const float* w = maybe(weight, "weight", pairs, dev);
    const auto floats = at::TensorOptions(dev).dtype(at::kFloat);
    Maybe grad;
    if (want) grad = at::empty({n}, floats);
    Tensor loss = at::empty({}, floats), pair = at::empty({pairs}, floats), rewards = at::empty({2 * pairs}, floats);
    const int rc = lbfgsb_preference_loss(n, pairs, l, r, off, m, w, &o, scale, (float*)loss.data_ptr(), (float*)pair.data_ptr(),
                                          (float*)rewards.data_ptr(), grad ? (float*)grad->data_ptr() : nullptr, (void*)stream);
    return std::make_tuple(rc, loss, pair, rewards, grad);
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
    m.def("token_logprob", &token_logprob);
    m.def("token_logprob_grad", &token_logprob_grad);
    m.def("distill_loss", &distill_loss);
    m.def("policy_loss", &policy_loss);
    m.def("preference_loss", &preference_loss);
    add_rollouts(m);
}
