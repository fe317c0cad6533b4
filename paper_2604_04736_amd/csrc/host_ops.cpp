// Host side of the calls that BayesianLinear and hot_stats_whole make: metadata checks, output and scratch allocation and
// the C call in one native function each, since a small layer's call is bound by the interpreter (a forecast of one row through
// three layers with 16 samples 69 -> 41 us, of which the GPU works 23; a training pass on 64 rows 456 -> 330).  Every function answers None where an argument is not what it takes without
// a copy or a conversion; the caller then goes through binding.py, whose checks name what is wrong.  No arithmetic here.
#include <torch/csrc/utils/pybind.h>

#include <ATen/ATen.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>

#include "hot.h"

namespace py = pybind11;
using at::Tensor;
typedef std::optional<Tensor> MaybeTensor;

namespace {

// A dense float32 tensor with memory of its own on the current device (no subclass, no transform's wrapper, no lazy negation).
bool plain(const Tensor &t, int64_t device)
{
    return t.is_cuda() && t.get_device() == device && t.scalar_type() == at::kFloat && t.layout() == at::kStrided && t.has_storage() &&
           !t.key_set().has(c10::DispatchKey::Python) && !t.is_neg() && t.is_contiguous();
}

bool is_vector(const MaybeTensor &t, int64_t n, int64_t device) { return t && plain(*t, device) && t->dim() == 1 && t->size(0) == n; }

const float *data(const Tensor &t) { return t.const_data_ptr<float>(); }
const float *data(const MaybeTensor &t) { return t ? t->const_data_ptr<float>() : nullptr; }

// the layer's description, if the arrays are as the C calls want them and have the layer's sizes (its draws and offsets are by these:
// with more outputs than that, the weights' eps would be those of its biases and of the next layer)
bool describe(const Tensor &x, const Tensor &mu_w, const Tensor &sigma_w, const MaybeTensor &mu_b, const MaybeTensor &sigma_b, int64_t in_features,
              int64_t out_features, int64_t s_local, int64_t weight_offset, int64_t bias_offset, int64_t device, hot_linear_desc &d)
{
    if (!plain(x, device) || !plain(mu_w, device) || !plain(sigma_w, device) || s_local < 1 || s_local > INT32_MAX) return false;
    if ((x.dim() != 2 && x.dim() != 3) || mu_w.dim() != 2 || mu_w.sizes() != sigma_w.sizes()) return false;
    const int64_t rows = x.size(-2), k = x.size(-1), o = mu_w.size(0);
    if (k != in_features || o != out_features || mu_w.size(1) != k || (x.dim() == 3 && x.size(0) != s_local)) return false;
    if (mu_b.has_value() != sigma_b.has_value() || (mu_b && !(is_vector(mu_b, o, device) && is_vector(sigma_b, o, device)))) return false;
    d.rows = rows;
    d.in_features = k;
    d.out_features = o;
    d.ldx = k;
    d.weight_offset = weight_offset;
    d.bias_offset = bias_offset;
    d.s_local = (int32_t)s_local;
    d.reserved = 0;
    d.x_sample_stride = x.dim() == 3 ? rows * k : 0;
    return true;
}

// Scratch memory: `bytes`, or the `least` where the device has no room for so much, which only buys time.
Tensor scratch(int64_t &bytes, int64_t least, const Tensor &like)
{
    const auto options = like.options().dtype(at::kByte);
    if (bytes > least) {
        try {
            return at::empty({bytes}, options);
        } catch (const c10::OutOfMemoryError &) {
            bytes = least;
        }
    }
    return bytes > 0 ? at::empty({bytes}, options) : Tensor();
}

// y, or the error code, or None
py::object linear_forward(const Tensor &x, const Tensor &mu_w, const Tensor &sigma_w, const MaybeTensor &mu_b, const MaybeTensor &sigma_b, uint64_t seed,
                          uint32_t step, uint32_t first_sample, int64_t in_features, int64_t out_features, int64_t s_local, int64_t weight_offset,
                          int64_t bias_offset, int64_t scratch_bytes, int64_t device, uintptr_t stream)
{
    hot_linear_desc d;
    if (!describe(x, mu_w, sigma_w, mu_b, sigma_b, in_features, out_features, s_local, weight_offset, bias_offset, device, d)) return py::none();
    Tensor y;
    int code;
    {
        py::gil_scoped_release others_run;
        y = at::empty({s_local, d.rows, d.out_features}, x.options());
        const Tensor ws = scratch(scratch_bytes, 0, x);
        const hot_rng rng = {seed, step, first_sample};
        code = hot_linear_forward_rng_ws(&d, &rng, data(x), data(mu_w), data(sigma_w), data(mu_b), data(sigma_b), y.mutable_data_ptr<float>(),
                                         scratch_bytes > 0 ? ws.mutable_data_ptr() : nullptr, scratch_bytes, reinterpret_cast<void *>(stream));
    }
    if (code != HOT_OK) return py::int_(code);
    return py::cast(y);
}

// (dx or None, grad mu_w, grad sigma_w, grad mu_b or None, grad sigma_b or None), or the error code, or None
py::object linear_backward(const Tensor &x, const Tensor &grad_y, const Tensor &mu_w, const Tensor &sigma_w, const MaybeTensor &mu_b, const MaybeTensor &sigma_b,
                           bool want_dx, uint64_t seed, uint32_t step, uint32_t first_sample, int64_t in_features, int64_t out_features, int64_t s_local,
                           double dataset_size, int64_t weight_offset, int64_t bias_offset, int64_t scratch_bytes, int64_t least_scratch, int64_t device,
                           uintptr_t stream)
{
    hot_linear_desc d;
    if (!describe(x, mu_w, sigma_w, mu_b, sigma_b, in_features, out_features, s_local, weight_offset, bias_offset, device, d)) return py::none();
    if (!plain(grad_y, device) || grad_y.dim() != 3 || grad_y.size(0) != s_local || grad_y.size(1) != d.rows || grad_y.size(2) != d.out_features)
        return py::none();
    Tensor dx, gmw, gsw, gmb, gsb;
    int code;
    {
        py::gil_scoped_release others_run;
        gmw = at::empty(mu_w.sizes(), x.options());
        gsw = at::empty(mu_w.sizes(), x.options());
        if (mu_b) {
            gmb = at::empty({d.out_features}, x.options());
            gsb = at::empty({d.out_features}, x.options());
        }
        if (want_dx) dx = at::empty({s_local, d.rows, d.in_features}, x.options());
        const Tensor ws = scratch(scratch_bytes, least_scratch, x);
        const hot_rng rng = {seed, step, first_sample};
        code = hot_linear_backward_rng_ws(&d, (int32_t)s_local, dataset_size, HOT_REDUCE_NONE, &rng, data(x), data(grad_y), data(mu_w), data(sigma_w),
                                          data(mu_b), data(sigma_b), gmw.mutable_data_ptr<float>(), gsw.mutable_data_ptr<float>(),
                                          mu_b ? gmb.mutable_data_ptr<float>() : nullptr, mu_b ? gsb.mutable_data_ptr<float>() : nullptr,
                                          want_dx ? dx.mutable_data_ptr<float>() : nullptr, scratch_bytes > 0 ? ws.mutable_data_ptr() : nullptr,
                                          scratch_bytes > 0 ? scratch_bytes : 0, reinterpret_cast<void *>(stream));
    }
    if (code != HOT_OK) return py::int_(code);
    auto maybe = [](const Tensor &t) -> py::object { return t.defined() ? py::cast(t) : py::none(); };
    return py::make_tuple(maybe(dx), gmw, gsw, maybe(gmb), maybe(gsb));
}

// the KL term (a float64 of no dimensions), or the error code, or None
py::object kl_layer(const Tensor &mu_w, const Tensor &sigma_w, const MaybeTensor &mu_b, const MaybeTensor &sigma_b, int64_t n_w, int64_t n_b,
                    int64_t device, uintptr_t stream)
{
    if (!plain(mu_w, device) || !plain(sigma_w, device) || mu_w.numel() != n_w || sigma_w.numel() != n_w) return py::none();
    if (n_b > 0 && !(is_vector(mu_b, n_b, device) && is_vector(sigma_b, n_b, device))) return py::none();
    Tensor out;
    int code;
    {
        py::gil_scoped_release others_run;
        out = at::empty({}, mu_w.options().dtype(at::kDouble));
        code = hot_kl_layer(n_w, data(mu_w), data(sigma_w), n_b, n_b > 0 ? data(mu_b) : nullptr, n_b > 0 ? data(sigma_b) : nullptr,
                            out.mutable_data_ptr<double>(), reinterpret_cast<void *>(stream));
    }
    if (code != HOT_OK) return py::int_(code);
    return py::cast(out);
}

// the error code, or None
py::object stats_whole(const Tensor &yhat, int32_t ddof, const Tensor &mean, const Tensor &std, int64_t device, uintptr_t stream)
{
    if (!plain(yhat, device) || yhat.dim() != 2 || yhat.size(0) < 1 || yhat.size(0) > INT32_MAX) return py::none();
    const int64_t m = yhat.size(1);
    if (!is_vector(mean, m, device) || !is_vector(std, m, device)) return py::none();
    int code;
    {
        py::gil_scoped_release others_run;
        code = hot_stats_whole(data(yhat), m, m, (int32_t)yhat.size(0), ddof, mean.mutable_data_ptr<float>(), std.mutable_data_ptr<float>(),
                               reinterpret_cast<void *>(stream));
    }
    return py::int_(code);
}

// ---------------------------------------------------------------------------------
// Layer norm and a head's loss as differentiable functions: the whole call, forward and backward, without the interpreter (a norm of 5003 x
// 777, forward and backward, 164 us through torch.autograd.Function).  What is not dense or not on the current device goes the other way.

using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

int type_of(const Tensor &t)
{
    return t.scalar_type() == at::kFloat ? HOT_F32 : (t.scalar_type() == at::kBFloat16 ? HOT_BF16 : (t.scalar_type() == at::kHalf ? HOT_F16 : -1));
}

bool dense(const Tensor &t, int64_t device)
{
    return t.is_cuda() && t.get_device() == device && t.layout() == at::kStrided && t.has_storage() && !t.key_set().has(c10::DispatchKey::Python) && !t.is_neg() &&
           t.is_contiguous();
}

const void *raw(const Tensor &t) { return t.defined() ? t.const_data_ptr() : nullptr; }
void *raw_mut(const Tensor &t) { return t.defined() ? t.mutable_data_ptr() : nullptr; }
void *stream_of(const Tensor &t) { return c10::hip::getCurrentHIPStream(t.get_device()).stream(); }

void check(int code, const char *where)
{
    TORCH_CHECK(code == HOT_OK, where, ": ", hot_strerror(code), " (code ", code, code == HOT_EHIP ? ", hipError " + std::to_string(hot_last_hip_error(nullptr)) : std::string(), ")");
}

// gradients that are asked for with a graph of their own carry a node that says there is none
variable_list once(variable_list grads, const char *name)
{
    if (!at::GradMode::is_enabled()) return grads;
    variable_list out;
    for (Tensor &g : grads) {
        if (g.defined()) {
            const auto error = std::make_shared<torch::autograd::DelayedError>(std::string(name) + " is differentiable once", 1);
            g = (*error)({g.detach().requires_grad_()})[0];
        }
        out.push_back(g);
    }
    return out;
}

Tensor given(const MaybeTensor &t) { return t ? *t : Tensor(); }

// room for the gradient of the next input, where it is wanted
Tensor gradient_of(AutogradContext *ctx, const Tensor &t, size_t &input)
{
    return t.defined() && ctx->needs_input_grad(input++) ? at::empty(t.sizes(), t.options()) : Tensor();
}

hot_norm_desc norm_desc(const Tensor &x, const Tensor &shaped, double eps)
{
    const int64_t width = x.size(-1), samples = shaped.defined() && shaped.dim() == 2 ? x.size(0) : 1, rows = x.numel() / width / std::max<int64_t>(samples, 1);
    hot_norm_desc d = {};
    d.rows = rows;
    d.width = width;
    d.ldx = d.ldy = width;
    d.x_sample = d.y_sample = rows * width;
    d.w_sample = shaped.defined() && shaped.dim() == 2 ? width : 0;
    d.eps = eps;
    d.samples = (int32_t)samples;
    d.dtype = type_of(x);
    d.weight_dtype = shaped.defined() ? type_of(shaped) : type_of(x);
    return d;
}

struct Norm : torch::autograd::Function<Norm> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, const MaybeTensor &maybe_weight, const MaybeTensor &maybe_bias, double eps)
    {
        const Tensor weight = given(maybe_weight), bias = given(maybe_bias);
        const hot_norm_desc d = norm_desc(x, weight.defined() ? weight : bias, eps);
        const Tensor y = at::empty(x.sizes(), x.options());
        // (autograd leaves no graph here; what is kept is of no use where nothing asked for gradients)
        const bool keep = x.requires_grad() || (weight.defined() && weight.requires_grad()) || (bias.defined() && bias.requires_grad());
        const Tensor stats = keep ? at::empty({2, d.samples * d.rows}, x.options().dtype(at::kFloat)) : Tensor();
        float *const mean = keep ? stats.mutable_data_ptr<float>() : nullptr;
        check(hot_norm_forward(&d, raw(x), raw(weight), raw(bias), raw_mut(y), mean, keep ? mean + d.samples * d.rows : nullptr, stream_of(x)), "hot_norm_forward");
        if (keep) ctx->save_for_backward({x, weight, bias, stats});
        return y;
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        const Tensor &x = saved[0], &weight = saved[1], &bias = saved[2], &stats = saved[3];
        const Tensor dy = grads[0].contiguous();
        const hot_norm_desc d = norm_desc(x, weight.defined() ? weight : bias, 0.0);
        size_t input = 0;        // (inputs that are not there are not counted)
        const Tensor dx = gradient_of(ctx, x, input), dw = gradient_of(ctx, weight, input), db = gradient_of(ctx, bias, input);
        const int64_t bytes = dw.defined() || db.defined() ? hot_norm_backward_workspace_bytes(&d) : 0;
        const Tensor ws = bytes > 0 ? at::empty({bytes}, x.options().dtype(at::kByte)) : Tensor();
        const float *const mean = stats.const_data_ptr<float>();
        check(hot_norm_backward(&d, raw(x), raw(weight), mean, mean + d.samples * d.rows, raw(dy), raw_mut(dx), raw_mut(dw), raw_mut(db), raw_mut(ws), bytes, stream_of(x)),
              "hot_norm_backward");
        return once({dx, dw, db, Tensor()}, "layer_norm");
    }
};

// y, or None
py::object layer_norm(const Tensor &x, const MaybeTensor &maybe_weight, const MaybeTensor &maybe_bias, double eps, int64_t device)
{
    const Tensor weight = given(maybe_weight), bias = given(maybe_bias), &shaped = weight.defined() ? weight : bias;
    if (!dense(x, device) || type_of(x) < 0 || x.dim() < 1 || x.numel() < 1 || !(eps >= 0.0)) return py::none();
    for (const Tensor &t : {weight, bias}) {
        if (!t.defined()) continue;
        if (!dense(t, device) || (t.scalar_type() != x.scalar_type() && t.scalar_type() != at::kFloat) || t.scalar_type() != shaped.scalar_type() || t.sizes() != shaped.sizes())
            return py::none();
        if (t.size(-1) != x.size(-1) || t.dim() > 2 || (t.dim() == 2 && (x.dim() < 2 || t.size(0) != x.size(0)))) return py::none();
    }
    const hot_norm_desc d = norm_desc(x, shaped, eps);
    if (hot_norm_backward_workspace_bytes(&d) < 0) return py::none();
    Tensor y;
    {
        py::gil_scoped_release others_run;
        y = Norm::apply(x, maybe_weight, maybe_bias, eps);
    }
    return py::cast(y);
}

// The shapes of a head's call (see autograd.py), for dense arrays.
struct HeadShape {
    hot_head_desc d;
    c10::SmallVector<int64_t, 5> loss;
};

bool head_shape(const Tensor &x, const Tensor &weight, const Tensor &bias, const Tensor &index, const Tensor &logit, int64_t ignore_index, double temperature, HeadShape &h)
{
    const int64_t entries = logit.defined() ? 1 : 0;
    if ((weight.dim() != 2 && weight.dim() != 3) || x.dim() < 1 || index.dim() < entries || x.size(-1) != weight.size(-1)) return false;
    if (bias.defined() && bias.sizes() != weight.sizes().slice(0, weight.dim() - 1)) return false;
    if (logit.defined() && logit.sizes() != index.sizes()) return false;
    const bool sampled = weight.dim() == 3, own = sampled && x.dim() > 2;
    const int64_t samples = sampled ? weight.size(0) : 1, top = entries ? index.size(-1) : 0;
    if (own && x.size(0) != samples) return false;
    const at::IntArrayRef rows = own ? x.sizes().slice(1, x.dim() - 2) : x.sizes().slice(0, x.dim() - 1), lead = index.sizes().slice(0, index.dim() - entries);
    if (sampled) h.loss.push_back(samples);
    h.loss.append(rows.begin(), rows.end());
    const bool all = lead == at::IntArrayRef(h.loss);
    if (!all && lead != rows) return false;
    if (entries && (top < 1 || top > INT32_MAX)) return false;
    int64_t count = 1;
    for (const int64_t n : rows) count *= n;
    hot_head_desc &d = h.d;
    d = {};
    d.rows = count;
    d.width = weight.size(-1);
    d.vocab = weight.size(-2);
    d.ldx = d.ldw = d.width;
    d.x_sample = own && samples > 1 ? count * d.width : 0;
    d.w_sample = samples > 1 ? d.vocab * d.width : 0;
    d.bias_sample = samples > 1 && bias.defined() ? d.vocab : 0;
    d.index_row = d.logit_row = entries ? top : 1;
    d.index_sample = d.logit_sample = samples > 1 && all ? count * d.index_row : 0;
    d.ignore_index = ignore_index;
    d.temperature = temperature;
    d.top = (int32_t)top;
    d.samples = (int32_t)samples;
    d.dtype = type_of(x);
    d.logit_dtype = logit.defined() ? type_of(logit) : 0;
    d.w_aligned = reinterpret_cast<uintptr_t>(weight.const_data_ptr()) % 16 == 0;
    return true;
}

struct Head : torch::autograd::Function<Head> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, const Tensor &weight, const MaybeTensor &maybe_bias, const Tensor &index, const MaybeTensor &maybe_logit,
                          int64_t ignore_index, double temperature)
    {
        const Tensor bias = given(maybe_bias), logit = given(maybe_logit);
        HeadShape h;
        TORCH_CHECK(head_shape(x, weight, bias, index, logit, ignore_index, temperature, h));
        const Tensor loss = at::empty(h.loss, x.options().dtype(at::kFloat));
        const bool keep = x.requires_grad() || weight.requires_grad() || (bias.defined() && bias.requires_grad());
        const Tensor lse = keep ? at::empty(h.loss, x.options().dtype(at::kDouble)) : Tensor();
        const int64_t bytes = hot_head_workspace_bytes(&h.d, 0);
        const Tensor ws = at::empty({bytes}, x.options().dtype(at::kByte));
        check(hot_head_forward(&h.d, raw(x), raw(weight), raw(bias), index.const_data_ptr<int64_t>(), raw(logit), loss.mutable_data_ptr<float>(),
                               keep ? lse.mutable_data_ptr<double>() : nullptr, raw_mut(ws), bytes, stream_of(x)),
              "hot_head_forward");
        if (keep) {
            ctx->save_for_backward({x, weight, bias, index, logit, lse});
            ctx->saved_data["ignore_index"] = ignore_index;
            ctx->saved_data["temperature"] = temperature;
        }
        return loss;
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        const Tensor &x = saved[0], &weight = saved[1], &bias = saved[2], &index = saved[3], &logit = saved[4], &lse = saved[5];
        HeadShape h;
        TORCH_CHECK(head_shape(x, weight, bias, index, logit, ctx->saved_data["ignore_index"].toInt(), ctx->saved_data["temperature"].toDouble(), h));
        const Tensor g = grads[0].reshape({h.d.samples, h.d.rows});
        size_t input = 0;
        const Tensor dx = gradient_of(ctx, x, input), dw = gradient_of(ctx, weight, input), db = gradient_of(ctx, bias, input);
        const int64_t bytes = hot_head_workspace_bytes(&h.d, dx.defined() ? 1 : 2);
        const Tensor ws = at::empty({bytes}, x.options().dtype(at::kByte));
        check(hot_head_backward(&h.d, raw(x), raw(weight), raw(bias), index.const_data_ptr<int64_t>(), raw(logit), lse.const_data_ptr<double>(), g.const_data_ptr<float>(),
                                g.size(0) > 1 ? g.stride(0) : 0, g.size(1) > 1 ? g.stride(1) : 0, raw_mut(dx), raw_mut(dw), raw_mut(db), raw_mut(ws), bytes, stream_of(x)),
              "hot_head_backward");
        return once({dx, dw, db, Tensor(), Tensor(), Tensor(), Tensor()}, "the head's loss");
    }
};

// the rows' losses, or None
py::object head_loss(const Tensor &x, const Tensor &weight, const MaybeTensor &maybe_bias, const Tensor &index, const MaybeTensor &maybe_logit, int64_t ignore_index,
                     double temperature, int64_t device)
{
    const Tensor bias = given(maybe_bias), logit = given(maybe_logit);
    if (!dense(x, device) || !dense(weight, device) || !dense(index, device) || type_of(x) < 0 || weight.scalar_type() != x.scalar_type() || index.scalar_type() != at::kLong)
        return py::none();
    if (bias.defined() && (!dense(bias, device) || bias.scalar_type() != x.scalar_type())) return py::none();
    if (logit.defined() && (!dense(logit, device) || type_of(logit) < 0)) return py::none();
    HeadShape h;
    if (!head_shape(x, weight, bias, index, logit, ignore_index, temperature, h) || hot_head_workspace_bytes(&h.d, 0) < 0) return py::none();
    Tensor loss;
    {
        py::gil_scoped_release others_run;
        loss = Head::apply(x, weight, maybe_bias, index, maybe_logit, ignore_index, temperature);
    }
    return py::cast(loss);
}

}  // namespace

PYBIND11_MODULE(_hot_host, m)
{
    m.def("layer_norm", &layer_norm);
    m.def("head_loss", &head_loss);
    m.def("linear_forward", &linear_forward);
    m.def("linear_backward", &linear_backward);
    m.def("kl_layer", &kl_layer);
    m.def("stats_whole", &stats_whole);
}
