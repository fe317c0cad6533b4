// Host side of the calls that BayesianLinear and hot_stats_whole make: metadata checks, output and scratch allocation and
// the C call in one native function each, since a small layer's call is bound by the interpreter (a forecast of one row through
// three layers with 16 samples 69 -> 41 us, of which the GPU works 23; a training pass on 64 rows 456 -> 330).  Every function answers None where an argument is not what it takes without
// a copy or a conversion; the caller then goes through binding.py, whose checks name what is wrong.  No arithmetic here.
#include <unordered_set>

#include <torch/csrc/utils/pybind.h>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
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

// In a backward pass that is being captured: the gradient of a leaf is handed over on the stream that was current when the leaf's first living graph was made.  Where that is
// the default stream (an eager graph of the leaf lives), the capture becomes invalid and its end ends the process: an error here instead, before that.
void captured_alone(const Tensor &like, const char *name)
{
    const auto stream = c10::hip::getCurrentHIPStream(like.device().index());
    const c10::StreamId eager = c10::hip::getDefaultHIPStream(like.device().index()).id();
    // (the default stream is never captured, and to ask it while another one is would be an error, left for a later call to find)
    if (stream.id() == eager) return;
    hipStreamCaptureStatus status = hipStreamCaptureStatusNone;
    const hipError_t asked = hipStreamIsCapturing(stream, &status);
    TORCH_CHECK(asked == hipSuccess, name, ": ", hipGetErrorString(asked));
    if (status == hipStreamCaptureStatusNone) return;
    const auto self = torch::autograd::get_current_node();
    std::vector<torch::autograd::Node *> left;
    std::unordered_set<torch::autograd::Node *> seen;
    if (self) left.push_back(self.get());
    while (!left.empty()) {
        torch::autograd::Node *const node = left.back();
        left.pop_back();
        for (uint32_t i = 0; i < node->num_outputs(); ++i) {
            torch::autograd::Node *const to = node->next_edge(i).function.get();
            if (!to || !node->task_should_compute_output(i) || !seen.insert(to).second) continue;
            const auto of = to->stream();
            TORCH_CHECK(to->num_outputs() != 0 || !of || of->id() != eager, name,
                        ": this backward pass is being captured while a graph of the same leaves, made on the default stream, lives; drop that graph first");
            left.push_back(to);
        }
    }
}

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

// ---------------------------------------------------------------------------------
// Dropout, a block's end and attention: every call goes this way, dense or not, with the checks that name what is wrong.

#define HOT_NEED(condition, ...) TORCH_CHECK_VALUE(condition, __VA_ARGS__)

void on_gpu(const Tensor &t, const char *name, const Tensor &like)
{
    TORCH_CHECK_TYPE(t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && !t.key_set().has(c10::DispatchKey::Python), name,
                     ": need a float32, bfloat16 or float16 tensor on a GPU");
    TORCH_CHECK_TYPE(t.device() == like.device(), name, ": need a tensor on ", like.device());
}

void elements(const Tensor &t, const char *name, const Tensor &like)
{
    TORCH_CHECK_TYPE(type_of(t) >= 0, name, ": need a float32, bfloat16 or float16 tensor on a GPU");
    on_gpu(t, name, like);
}

struct Counter {
    hot_rng rng;
    int64_t samples, offset;
    double keep;
};

// samples = 0: all rows are of one sample
int64_t samples_of(const Tensor &x, const char *name, int64_t samples)
{
    HOT_NEED(samples >= 0 && samples <= 65535, "samples: need 0 to 65535, got ", samples);
    HOT_NEED(x.dim() >= (samples ? 2 : 1) && x.size(-1) >= 1, name, ": need [", samples ? "samples, " : "", "..., width] with a width, got ", x.sizes());
    HOT_NEED(!samples || x.size(0) == samples, name, ": need ", samples, " samples in front, got ", x.sizes());
    return samples ? samples : 1;
}

hot_rng counter_rng(uint64_t seed, int64_t step, int64_t first_sample, int64_t samples)
{
    HOT_NEED(step >= 0 && step <= UINT32_MAX, "rng: need a step below 2^32, got ", step);
    HOT_NEED(first_sample >= 0 && first_sample + samples <= (int64_t(1) << 32), "rng: need samples below 2^32, got ", first_sample, " and ", samples, " from there on");
    hot_rng r = {};
    r.seed = seed;
    r.step = (uint32_t)step;
    r.first_sample = (uint32_t)first_sample;
    return r;
}

void check_keep(double keep, int64_t offset)
{
    HOT_NEED(keep > 0.0 && keep <= 1.0, "keep: need 0 < keep <= 1, got ", keep);
    HOT_NEED(offset >= 0, "offset: need at least 0, got ", offset);
}

struct Dropout : torch::autograd::Function<Dropout> {
    static Tensor forward(AutogradContext *ctx, const Tensor &x, double keep, int64_t seed, int64_t step, int64_t first_sample, int64_t samples, int64_t offset)
    {
        const c10::DeviceGuard guard(x.device());
        const int64_t sets = samples ? samples : 1, width = x.size(-1);
        const Tensor from = x.resolve_neg().contiguous(), y = at::empty(x.sizes(), from.options());
        hot_dropout_desc d = {};
        d.width = width;
        d.rows = x.numel() / width / sets;
        d.offset = offset;
        d.keep = keep;
        d.samples = (int32_t)sets;
        d.dtype = type_of(x);
        const hot_rng rng = counter_rng((uint64_t)seed, step, first_sample, sets);
        check(hot_dropout(&d, &rng, raw(from), raw_mut(y), stream_of(x)), "hot_dropout");
        ctx->saved_data["keep"] = keep;
        ctx->saved_data["counter"] = std::vector<int64_t>{seed, step, first_sample, samples, offset};
        return y;
    }

    // (its own gradient, as often as it is asked for)
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const auto c = ctx->saved_data["counter"].toIntVector();
        if (grads[0].defined()) captured_alone(grads[0], "dropout");
        return {grads[0].defined() ? apply(grads[0], ctx->saved_data["keep"].toDouble(), c[0], c[1], c[2], c[3], c[4]) : Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor(), Tensor()};
    }
};

Tensor dropout(const Tensor &x, double keep, uint64_t seed, int64_t step, int64_t first_sample, int64_t samples, int64_t offset)
{
    elements(x, "x", x);
    const int64_t sets = samples_of(x, "x", samples);
    check_keep(keep, offset);
    counter_rng(seed, step, first_sample, sets);
    py::gil_scoped_release others_run;
    return Dropout::apply(x, keep, (int64_t)seed, step, first_sample, samples, offset);
}

// What a block's call is described by, beside its tensors
struct BlockRule {
    std::vector<int64_t> whole;      // norm, branch_norm, seed, step, first_sample, samples, offset
    double scale, keep, eps;
};

int64_t own_pitch(const Tensor &v) { return v.defined() && v.dim() == 2 ? v.size(1) : 0; }

hot_block_desc block_desc(const Tensor &x, const Tensor (&v)[5], const BlockRule &r, hot_rng &rng)
{
    hot_block_desc d = {};
    const int64_t sets = r.whole[5] ? r.whole[5] : 1;
    d.width = x.size(-1);
    d.rows = x.numel() / d.width / sets;
    d.weight_sample = own_pitch(v[0]);
    d.bias_sample = own_pitch(v[1]);
    d.gate_sample = own_pitch(v[2]);
    d.branch_weight_sample = own_pitch(v[3]);
    d.branch_bias_sample = own_pitch(v[4]);
    d.offset = r.whole[6];
    d.scale = r.scale;
    d.keep = r.keep;
    d.eps = r.eps;
    d.samples = (int32_t)sets;
    d.dtype = type_of(x);
    d.vector_dtype = d.dtype;
    for (const Tensor &t : v)
        if (t.defined()) d.vector_dtype = type_of(t);
    d.norm = (int32_t)r.whole[0];
    d.branch_norm = (int32_t)r.whole[1];
    rng = counter_rng((uint64_t)r.whole[2], r.whole[3], r.whole[4], sets);
    return d;
}

struct BlockEnd : torch::autograd::Function<BlockEnd> {
    static variable_list forward(AutogradContext *ctx, const Tensor &x, const Tensor &branch, const MaybeTensor &weight, const MaybeTensor &bias, const MaybeTensor &gate,
                                 const MaybeTensor &branch_weight, const MaybeTensor &branch_bias, std::vector<int64_t> whole, double scale, double keep, double eps, bool graph)
    {
        const c10::DeviceGuard guard(x.device());
        const BlockRule rule = {whole, scale, keep, eps};
        const Tensor xs = x.resolve_neg().contiguous(), bs = branch.resolve_neg().contiguous();
        Tensor v[5] = {given(weight), given(bias), given(gate), given(branch_weight), given(branch_bias)};
        bool wanted = x.requires_grad() || branch.requires_grad();
        for (Tensor &t : v)
            if (t.defined()) {
                wanted = wanted || t.requires_grad();
                t = t.resolve_neg().contiguous();
            }
        hot_rng rng;
        wanted = wanted && graph;
        const hot_block_desc d = block_desc(xs, v, rule, rng);
        const Tensor h = at::empty(x.sizes(), xs.options()), y = d.norm != HOT_NORM_NONE ? at::empty(x.sizes(), xs.options()) : Tensor();
        const Tensor stats = wanted ? at::empty({d.samples, d.rows, 4}, xs.options().dtype(at::kFloat)) : Tensor();
        check(hot_block_forward(&d, &rng, raw(xs), raw(bs), raw(v[0]), raw(v[1]), raw(v[2]), raw(v[3]), raw(v[4]), raw_mut(h), raw_mut(y),
                                stats.defined() ? stats.mutable_data_ptr<float>() : nullptr, stream_of(x)),
              "hot_block_forward");
        if (wanted) {
            ctx->set_materialize_grads(false);
            ctx->save_for_backward({xs, bs, v[0], v[1], v[2], v[3], v[4], stats});
            ctx->saved_data["whole"] = whole;
            ctx->saved_data["real"] = std::vector<double>{scale, keep, eps};
        }
        if (y.defined()) return {h, y};
        return {h};
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        const variable_list saved = ctx->get_saved_variables();
        const Tensor &x = saved[0], &branch = saved[1], &stats = saved[7];
        const c10::DeviceGuard guard(x.device());
        const Tensor v[5] = {saved[2], saved[3], saved[4], saved[5], saved[6]};
        const auto real = ctx->saved_data["real"].toDoubleVector();
        const BlockRule rule = {ctx->saved_data["whole"].toIntVector(), real[0], real[1], real[2]};
        hot_rng rng;
        const hot_block_desc d = block_desc(x, v, rule, rng);
        const Tensor dh = grads[0].defined() ? grads[0].resolve_neg().contiguous() : Tensor();
        const Tensor dy = grads.size() > 1 && grads[1].defined() ? grads[1].resolve_neg().contiguous() : Tensor();
        if (!dh.defined() && !dy.defined()) return variable_list(12);
        captured_alone(x, "residual_norm");
        size_t input = 0;        // (inputs that are not there are not counted)
        const Tensor dx = gradient_of(ctx, x, input), dbranch = gradient_of(ctx, branch, input);
        Tensor dv[5];
        bool sums = false;
        for (int k = 0; k < 5; ++k) {
            dv[k] = gradient_of(ctx, v[k], input);
            sums = sums || dv[k].defined();
        }
        const int64_t bytes = sums ? hot_block_backward_workspace_bytes(&d) : 0;
        const Tensor ws = bytes > 0 ? at::empty({bytes}, x.options().dtype(at::kByte)) : Tensor();
        check(hot_block_backward(&d, &rng, raw(x), raw(branch), raw(v[0]), raw(v[2]), raw(v[3]), raw(v[4]), stats.const_data_ptr<float>(), raw(dh), raw(dy), raw_mut(dx),
                                 raw_mut(dbranch), raw_mut(dv[0]), raw_mut(dv[1]), raw_mut(dv[2]), raw_mut(dv[3]), raw_mut(dv[4]), raw_mut(ws), bytes, stream_of(x)),
              "hot_block_backward");
        return once({dx, dbranch, dv[0], dv[1], dv[2], dv[3], dv[4], Tensor(), Tensor(), Tensor(), Tensor(), Tensor()}, "residual_norm");
    }
};

// (h, y), or (h,) without a norm
std::vector<Tensor> block_end(const Tensor &x, const Tensor &branch, const MaybeTensor &weight, const MaybeTensor &bias, const MaybeTensor &gate, const MaybeTensor &branch_weight,
                              const MaybeTensor &branch_bias, int64_t norm, int64_t branch_norm, double scale, double keep, double eps, uint64_t seed, int64_t step,
                              int64_t first_sample, int64_t samples, int64_t offset)
{
    elements(x, "x", x);
    elements(branch, "branch", x);
    const int64_t sets = samples_of(x, "x", samples), width = x.size(-1);
    HOT_NEED(width <= HOT_BLOCK_MOST_WIDTH, "x: need a width of at most ", HOT_BLOCK_MOST_WIDTH, ", got ", width);
    TORCH_CHECK_TYPE(branch.scalar_type() == x.scalar_type(), "branch: need x's type");
    HOT_NEED(branch.sizes() == x.sizes(), "branch: need x's shape ", x.sizes(), ", got ", branch.sizes());
    check_keep(keep, offset);
    HOT_NEED(eps >= 0.0 && eps <= 3.0e38, "eps: need at least 0, got ", eps);
    HOT_NEED(scale >= -3.0e38 && scale <= 3.0e38, "scale: need a finite number, got ", scale);
    const char *const names[5] = {"weight", "bias", "gate", "branch_weight", "branch_bias"};
    const Tensor v[5] = {given(weight), given(bias), given(gate), given(branch_weight), given(branch_bias)};
    at::ScalarType type = at::ScalarType::Undefined;
    for (int k = 0; k < 5; ++k) {
        if (!v[k].defined()) continue;
        elements(v[k], names[k], x);
        HOT_NEED(k == 2 || (k < 2 ? norm : branch_norm) != HOT_NORM_NONE, names[k], ": there is no norm that it belongs to");
        TORCH_CHECK_TYPE((v[k].scalar_type() == x.scalar_type() || v[k].scalar_type() == at::kFloat) && (type == at::ScalarType::Undefined || v[k].scalar_type() == type), names[k],
                         ": the vectors need one type, x's or float32");
        type = v[k].scalar_type();
        HOT_NEED((v[k].dim() == 1 || (v[k].dim() == 2 && samples && v[k].size(0) == samples)) && v[k].size(-1) == width, names[k], ": need [", width, "] or [samples, ", width,
                 "], got ", v[k].sizes());
    }
    counter_rng(seed, step, first_sample, sets);
    py::gil_scoped_release others_run;
    return BlockEnd::apply(x, branch, weight, bias, gate, branch_weight, branch_bias, std::vector<int64_t>{norm, branch_norm, (int64_t)seed, step, first_sample, samples, offset},
                           scale, keep, eps, at::GradMode::is_enabled());
}

// [..., heads, tokens, width] as [batch, heads, tokens, width] with adjacent elements: a view, or a copy where the leading axes are no single one
Tensor four_axes(const Tensor &t)
{
    Tensor u = t.resolve_neg();
    if (u.size(-1) > 1 && u.stride(-1) != 1) u = u.contiguous();
    return u.dim() == 4 ? u : (u.dim() == 3 ? u.unsqueeze(0) : u.flatten(0, -4));
}

hot_pitch pitch_of(const Tensor &t)
{
    const auto of = [&](int64_t i) { return t.size(i) > 1 ? t.stride(i) : 0; };
    return {of(0), of(1), of(2)};
}

// Heads side by side in a token's row, as the products around attention have them
Tensor token_major(const Tensor &like) { return at::empty({like.size(0), like.size(2), like.size(1), like.size(3)}, like.options()).transpose(1, 2); }

Tensor room_like(const Tensor &t) { return t.is_non_overlapping_and_dense() && (t.size(-1) < 2 || t.stride(-1) == 1) ? at::empty_like(t) : token_major(t); }

hot_attention_desc attention_desc(const Tensor &q, const Tensor &k, const Tensor &v, const Tensor &table, const Tensor &bucket, const Tensor &query_groups, int64_t first_query,
                                  double scale, bool causal)
{
    hot_attention_desc d = {};
    d.queries = q.size(2);
    d.keys = k.size(2);
    d.q = pitch_of(q);
    d.k = pitch_of(k);
    d.v = pitch_of(v);
    d.scale = scale;
    d.batch = (int32_t)q.size(0);
    d.heads = (int32_t)q.size(1);
    d.kv_heads = (int32_t)k.size(1);
    d.width = (int32_t)q.size(3);
    if (table.defined()) {
        d.tables = (int32_t)(table.dim() == 3 ? table.size(0) : 1);
        d.buckets = (int32_t)table.size(-2);
        d.codes = (int32_t)bucket.size(0);
        d.first_query = (int32_t)first_query;
        d.table_dtype = type_of(table);
    }
    d.groups = query_groups.defined() ? (int32_t)query_groups.size(0) : 0;
    d.causal = causal;
    d.dtype = type_of(q);
    for (const Tensor *t : {&q, &k, &v}) d.loose |= reinterpret_cast<uintptr_t>(t->const_data_ptr()) % 4 != 0;
    return d;
}

const int32_t *codes(const Tensor &t) { return t.defined() ? t.const_data_ptr<int32_t>() : nullptr; }

Tensor attention_room(const hot_attention_desc &d, int which, const Tensor &like)
{
    const int64_t bytes = hot_attention_workspace_bytes(&d, which);
    TORCH_CHECK(bytes >= 0, "hot_attention_workspace_bytes: ", hot_strerror((int)bytes), " (code ", bytes, ")");
    return at::empty({bytes}, like.options().dtype(at::kByte));
}

struct Attention : torch::autograd::Function<Attention> {
    static Tensor forward(AutogradContext *ctx, const Tensor &q_, const Tensor &k_, const Tensor &v_, const MaybeTensor &maybe_table, const MaybeTensor &query_code,
                          const MaybeTensor &key_code, const MaybeTensor &query_range, const MaybeTensor &key_range, const MaybeTensor &bucket, const MaybeTensor &query_groups, const MaybeTensor &key_groups,
                          int64_t first_query, double scale, bool causal, bool graph)
    {
        const c10::DeviceGuard guard(q_.device());
        const Tensor q = four_axes(q_), k = four_axes(k_), v = four_axes(v_);
        const Tensor table = maybe_table ? maybe_table->resolve_neg().contiguous() : Tensor(), qg = given(query_groups), kg = given(key_groups);
        hot_attention_desc d = attention_desc(q, k, v, table, given(bucket), qg, first_query, scale, causal);
        const Tensor o = token_major(q);
        d.o = pitch_of(o);
        const bool keep = graph && (q_.requires_grad() || k_.requires_grad() || v_.requires_grad() || (maybe_table && maybe_table->requires_grad()));
        const Tensor stats = keep ? at::empty({q.size(0), q.size(1), q.size(2), 2}, q.options().dtype(at::kFloat)) : Tensor();
        const Tensor rest = keep && d.dtype != HOT_F32 ? token_major(q) : Tensor();
        const Tensor ws = attention_room(d, 0, q);
        check(hot_attention_forward(&d, raw(q), raw(k), raw(v), raw(table), codes(given(query_code)), codes(given(key_code)), codes(given(query_range)), codes(given(key_range)),
                                    codes(given(bucket)), codes(qg), codes(kg), raw_mut(o), raw_mut(rest), stats.defined() ? stats.mutable_data_ptr<float>() : nullptr, raw_mut(ws), ws.numel(), stream_of(q)),
              "hot_attention_forward");
        if (keep) {
            ctx->save_for_backward({q, k, v, table, given(query_code), given(key_code), given(query_range), given(key_range), given(bucket), qg, kg, o, rest, stats});
            ctx->saved_data["whole"] = std::vector<int64_t>{first_query, causal};
            ctx->saved_data["scale"] = scale;
            ctx->saved_data["q"] = q_.sizes().vec();
            ctx->saved_data["k"] = k_.sizes().vec();
        }
        return o.reshape(q_.sizes());
    }

    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        variable_list none(15);
        if (!grads[0].defined()) return none;
        captured_alone(grads[0], "attention");
        const variable_list s = ctx->get_saved_variables();
        const Tensor &q = s[0], &k = s[1], &v = s[2], &table = s[3], &o = s[11], &rest = s[12], &stats = s[13];
        const c10::DeviceGuard guard(q.device());
        const auto whole = ctx->saved_data["whole"].toIntVector();
        const Tensor up = four_axes(grads[0]);
        hot_attention_desc d = attention_desc(q, k, v, table, s[8], s[9], whole[0], ctx->saved_data["scale"].toDouble(), whole[1]);
        const Tensor dq = ctx->needs_input_grad(0) ? room_like(q) : Tensor(), dk = ctx->needs_input_grad(1) ? room_like(k) : Tensor(), dv = ctx->needs_input_grad(2) ? room_like(v) : Tensor();
        const Tensor dtable = table.defined() && ctx->needs_input_grad(3) ? at::empty_like(table) : Tensor();
        d.o = pitch_of(o);
        d.grad_o = pitch_of(up);
        d.loose |= reinterpret_cast<uintptr_t>(up.const_data_ptr()) % 4 != 0;
        if (dq.defined()) d.grad_q = pitch_of(dq);
        if (dk.defined()) d.grad_k = pitch_of(dk);
        if (dv.defined()) d.grad_v = pitch_of(dv);
        const Tensor ws = attention_room(d, 1, q);
        check(hot_attention_backward(&d, raw(q), raw(k), raw(v), raw(table), codes(s[4]), codes(s[5]), codes(s[6]), codes(s[7]), codes(s[8]), codes(s[9]), codes(s[10]), raw(o), raw(rest),
                                     stats.const_data_ptr<float>(), raw(up), raw_mut(dq), raw_mut(dk), raw_mut(dv), raw_mut(dtable), raw_mut(ws), ws.numel(), stream_of(q)),
              "hot_attention_backward");
        const auto as = [&](const Tensor &t, const char *name) { return t.defined() ? t.reshape(ctx->saved_data[name].toIntVector()) : t; };
        none[0] = as(dq, "q");
        none[1] = as(dk, "k");
        none[2] = as(dv, "k");
        none[3] = dtable;
        return once(none, "attention");
    }
};

// Rows of group numbers as int32 [groups, n], or an error
Tensor group_rows(const MaybeTensor &maybe, const char *name, int64_t n, const Tensor &like)
{
    if (!maybe) return Tensor();
    const Tensor &t = *maybe;
    TORCH_CHECK_TYPE(t.is_cuda() && t.device() == like.device() && t.scalar_type() == at::kInt && !t.key_set().has(c10::DispatchKey::Python), name, ": need an int32 tensor on ", like.device());
    HOT_NEED((t.dim() == 1 || t.dim() == 2) && t.size(-1) == n && t.size(0) >= (t.dim() == 2), name, ": need [", n, "] or [entries, ", n, "], got ", t.sizes());
    return (t.dim() == 1 ? t.unsqueeze(0) : t).contiguous();
}

Tensor attention(const Tensor &q, const Tensor &k, const Tensor &v, const MaybeTensor &table, const MaybeTensor &query_code, const MaybeTensor &key_code, const MaybeTensor &query_range,
                 const MaybeTensor &key_range, const MaybeTensor &bucket, int64_t buckets, const MaybeTensor &query_groups, const MaybeTensor &key_groups, int64_t first_query, double scale, bool causal)
{
    elements(q, "q", q);
    elements(k, "k", q);
    elements(v, "v", q);
    TORCH_CHECK_TYPE(k.scalar_type() == q.scalar_type() && v.scalar_type() == q.scalar_type(), "k and v: need q's type");
    const int64_t n = q.dim();
    HOT_NEED(n >= 3 && q.size(-1) >= HOT_ATTENTION_LEAST_WIDTH && q.size(-1) <= HOT_ATTENTION_MOST_WIDTH && q.size(-3) >= 1, "q: need [..., heads, queries, width] with a width of 8 to ",
             HOT_ATTENTION_MOST_WIDTH, ", got ", q.sizes());
    HOT_NEED(k.dim() == n && k.sizes() == v.sizes() && k.size(-1) == q.size(-1) && k.sizes().slice(0, n - 3) == q.sizes().slice(0, n - 3), "k and v: need one shape, q's leading axes and width ",
             q.sizes(), ", got ", k.sizes(), " and ", v.sizes());
    HOT_NEED(k.size(-3) >= 1 && q.size(-3) % k.size(-3) == 0, "k and v: need a number of heads that divides ", q.size(-3), ", got ", k.size(-3));
    HOT_NEED(scale >= -1.0e30 && scale <= 1.0e30, "scale: need a number up to 1e30, got ", scale);
    int64_t batch = 1;
    for (const int64_t m : q.sizes().slice(0, n - 3)) batch *= m;
    HOT_NEED((double)batch * (double)q.size(-3) * (double)std::max<int64_t>(1, std::max(q.size(-2), k.size(-2))) < 2147483647.0 && q.size(-3) <= 65535,
             "q: need fewer than 2^31 rows and 65536 heads, got ", q.sizes());
    HOT_NEED(std::max(q.size(-2), k.size(-2)) <= HOT_ATTENTION_MOST_TOKENS, "q and k: need at most ", HOT_ATTENTION_MOST_TOKENS, " tokens, got ", q.sizes(), " and ", k.sizes());
    if (table) {
        elements(*table, "table", q);
        TORCH_CHECK_TYPE(table->scalar_type() == q.scalar_type() || table->scalar_type() == at::kFloat, "table: need q's type or float32");
        HOT_NEED(bucket && query_code && key_code && query_range && key_range, "table: need positions");
        HOT_NEED((table->dim() == 2 || (table->dim() == 3 && n >= 4 && table->size(0) == q.size(0) && table->size(0) >= 1 && table->size(0) <= 65535)) && table->size(-1) == q.size(-3) &&
                     table->size(-2) == buckets,
                 "table: need [", buckets, ", ", q.size(-3), "], or one for each of q's first axis, got ", table->sizes());
        for (const MaybeTensor *t : {&query_code, &key_code, &query_range, &key_range, &bucket})
            TORCH_CHECK_TYPE((*t)->is_cuda() && (*t)->device() == q.device() && (*t)->scalar_type() == at::kInt && (*t)->is_contiguous(), "positions: need those of ", q.device());
        HOT_NEED(first_query >= 0 && first_query + q.size(-2) <= query_code->size(0), "first_query: the positions know ", query_code->size(0), " queries, got ", q.size(-2), " from ",
                 first_query, " on");
        HOT_NEED(k.size(-2) <= key_code->size(0), "k: the positions know ", key_code->size(0), " keys, got ", k.size(-2));
    }
    Tensor qg = group_rows(query_groups, "query_groups", q.size(-2), q), kg = group_rows(key_groups, "key_groups", k.size(-2), q);
    HOT_NEED(!qg.defined() || kg.defined(), "query_groups: need key_groups too");
    if (kg.defined()) {
        if (!qg.defined()) qg = at::zeros({1, q.size(-2)}, kg.options());
        const int64_t rows = std::max(qg.size(0), kg.size(0));
        HOT_NEED((qg.size(0) == rows || qg.size(0) == 1) && (kg.size(0) == rows || kg.size(0) == 1) && batch % rows == 0, "query_groups and key_groups: need as many rows, dividing ", batch,
                 " entries, got ", qg.sizes(), " and ", kg.sizes());
        qg = qg.expand({rows, qg.size(1)}).contiguous();
        kg = kg.expand({rows, kg.size(1)}).contiguous();
    }
    const auto there = [](const Tensor &t) { return t.defined() ? MaybeTensor(t) : MaybeTensor(); };
    const bool graph = at::GradMode::is_enabled();
    py::gil_scoped_release others_run;
    if (!table) return Attention::apply(q, k, v, MaybeTensor(), MaybeTensor(), MaybeTensor(), MaybeTensor(), MaybeTensor(), MaybeTensor(), there(qg), there(kg), 0, scale, causal, graph);
    return Attention::apply(q, k, v, table, query_code, key_code, query_range, key_range, bucket, there(qg), there(kg), first_query, scale, causal, graph);
}

}  // namespace

PYBIND11_MODULE(_hot_host, m)
{
    m.def("dropout", &dropout);
    m.def("block_end", &block_end);
    m.def("attention", &attention);
    m.def("layer_norm", &layer_norm);
    m.def("head_loss", &head_loss);
    m.def("linear_forward", &linear_forward);
    m.def("linear_backward", &linear_backward);
    m.def("kl_layer", &kl_layer);
    m.def("stats_whole", &stats_whole);
}
