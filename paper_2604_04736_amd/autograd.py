"""torch.autograd plumbing around the C ABI: the Gaussian sample layer as a differentiable
function of (mu, sigma), so that a PyTorch training loop can use the HIP path unchanged, and the
sampled linear layer (BayesianLinear, at the end), whose per-sample weight gradients never exist in
memory, nor its drawn weights up to 128 rows.  With more rows the drawn weights of a call may lie in
scratch memory, as bf16 pieces (six bytes per weight and sample, at most 1 GiB, from torch's allocator
and given back when the call returns); where there is no room for them the call runs without.

    layer = GaussianSampleLayer(n_weights, s_local, dataset_size)
    w, kl = layer.sample(mu, sigma, step)          # w[s] = mu + sigma * eps_s,  eps drawn in the kernel
    loss = sum(net_loss(w[s]) for s in range(s_local)) / s_local
    loss.backward()                                 # mu.grad, sigma.grad = d(loss + KL/|D|)/d(mu, sigma)

The KL term of the negative scaled ELBO (Algorithm 1 / 2 of arxiv 2604.04736: L = L_data + KL/|D|)
is added to the gradients inside the backward kernel, as a fused regulariser; `kl` is returned
detached for logging.  No arithmetic of the method happens here: the forward is hot_forward_rng,
the backward hot_backward_rng with HOT_REDUCE_NONE (the incoming gradient already carries the
caller's scaling).
"""
from __future__ import annotations

import functools
import math
import operator

import torch

from . import binding as hot


class _Sample(torch.autograd.Function):
    @staticmethod
    def forward(ctx, mu, sigma, layer, step):
        w = torch.empty(layer.s_local, layer.n_weights, dtype=torch.float32, device=mu.device)
        kl = torch.empty(1, dtype=torch.float64, device=mu.device)
        rng = hot.hot_rng(seed=layer.seed, step=step, first_sample=layer.first_sample)
        hot.hot_forward_rng(layer.plan, rng, mu.detach(), sigma.detach(), w, kl)
        ctx.layer, ctx.rng = layer, rng
        ctx.save_for_backward(mu.detach(), sigma.detach())
        ctx.mark_non_differentiable(kl)
        return w, kl

    @staticmethod
    def backward(ctx, grad_w, _grad_kl):
        mu, sigma = ctx.saved_tensors
        grad_w = grad_w.contiguous()
        gmu, gsig = torch.empty_like(mu), torch.empty_like(sigma)
        hot.hot_backward_rng(ctx.layer.plan, ctx.rng, mu, sigma, grad_w, gmu, gsig)
        return gmu, gsig, None, None


class GaussianSampleLayer:
    """Holds the plan of one flat parameter vector; `first_sample` is the global index of this GPU's
    first sample (rank * s_local under sampling parallelism), so that GPUs sharing a seed draw
    disjoint samples."""

    def __init__(self, n_weights: int, s_local: int, dataset_size: float, device: int = 0, seed: int = 0,
                 first_sample: int = 0):
        self.n_weights, self.s_local, self.seed, self.first_sample = n_weights, s_local, seed, first_sample
        self.plan = hot.hot_create(n_weights, n_weights, s_local, s_local, dataset_size, device, hot.HOT_REDUCE_NONE)

    def sample(self, mu: torch.Tensor, sigma: torch.Tensor, step: int):
        """w[S_loc, N] (differentiable with respect to mu and sigma) and the KL term (detached, fp64)."""
        return _Sample.apply(mu, sigma, self, int(step))


# What the library asks for by a layer's sizes (pure functions of them; kept, since a query costs a small layer's call some microseconds).
@functools.lru_cache(maxsize=4096)
def _forward_scratch(rows: int, k: int, o: int, s_local: int, per_sample_x: bool) -> int:
    return hot.hot_linear_planes_workspace_bytes(rows, k, o, s_local, 0, per_sample_x)


@functools.lru_cache(maxsize=4096)
def _backward_scratch(rows: int, k: int, o: int, s_local: int, with_dx: bool) -> tuple[int, int]:
    """What is asked for, and what is left of it where there is no room for the planes."""
    split = hot.hot_linear_backward_workspace_bytes(rows, k, o, s_local)
    return max(split, hot.hot_linear_planes_workspace_bytes(rows, k, o, s_local, 1)) if with_dx else split, split


def _scratch(wanted: int, least: int, device):
    """A tensor of `wanted` bytes, or of the `least` where the device has no room for so much, which only buys time."""
    if wanted > least:
        try:
            return torch.empty(wanted // 4, dtype=torch.float32, device=device)
        except torch.OutOfMemoryError:
            pass
    return torch.empty(least // 4, dtype=torch.float32, device=device) if least > 0 else None


_M32, _M64 = 0xFFFFFFFF, (1 << 64) - 1


def _device_and_stream():
    dev = torch.cuda.current_device()
    return dev, hot._stream(dev)


def _answer(result, where: str):
    """The answer of a function of hot.host(): a result, None, or an error code, which is raised."""
    if type(result) is int:
        hot._check_planless(result, where)
    return result


class _Linear(torch.autograd.Function):
    """The native functions take what is dense and on the current device (hot.host(); all of a call in one); whatever else the
    layer is given goes through binding.py."""

    @staticmethod
    def forward(ctx, x, mu_w, sigma_w, mu_b, sigma_b, layer, step):
        # (as Python's integers: NumPy's have no room for the mask)
        draw = (operator.index(layer.seed) & _M64, step & _M32, operator.index(layer.first_sample) & _M32)
        x = x.contiguous()
        ctx.layer, ctx.draw = layer, draw
        ctx.save_for_backward(x, mu_w, sigma_w, mu_b, sigma_b)
        # many rows: the library leaves the drawn weights in scratch memory of ours instead of drawing them for every tile of rows
        # (never up to 128, where the look itself would cost a small layer's call)
        rows = x.shape[-2]
        ws_bytes = _forward_scratch(rows, layer.in_features, layer.out_features, layer.s_local, x.dim() == 3) if rows > 128 else 0
        if x.is_cuda:
            y = _answer(hot.host().linear_forward(x, mu_w, sigma_w, mu_b, sigma_b, *draw, layer.in_features, layer.out_features, layer.s_local,
                                                 layer.weight_offset, layer.bias_offset, ws_bytes, *_device_and_stream()), "hot_linear_forward_rng")
            if y is not None:
                return y
        y = torch.empty(layer.s_local, rows, layer.out_features, dtype=torch.float32, device=x.device)
        det = [t.detach() if t is not None else None for t in (mu_w, sigma_w, mu_b, sigma_b)]
        ws = _scratch(ws_bytes, 0, x.device)
        hot.hot_linear_forward_rng(hot.hot_rng(*draw), x.detach(), det[0], det[1], det[2], det[3], y, layer.weight_offset, layer.bias_offset,
                                   workspace=ws)
        return y

    @staticmethod
    def backward(ctx, grad_y):
        layer, draw = ctx.layer, ctx.draw
        xd, mu_w, sigma_w, mu_b, sigma_b = (t.detach() if t is not None else None for t in ctx.saved_tensors)
        want_dx, grad_y = ctx.needs_input_grad[0], grad_y.contiguous()
        # few weights and many rows: the library spreads the rows over the chip through scratch memory of ours
        ws_bytes, least = _backward_scratch(xd.shape[-2], layer.in_features, layer.out_features, layer.s_local, want_dx)
        grads = None
        if xd.is_cuda:
            grads = _answer(hot.host().linear_backward(xd, grad_y, mu_w, sigma_w, mu_b, sigma_b, want_dx, *draw, layer.in_features, layer.out_features,
                                                      layer.s_local, layer.dataset_size, layer.weight_offset, layer.bias_offset, ws_bytes, least,
                                                      *_device_and_stream()), "hot_linear_backward_rng_ws" if ws_bytes > 0 else "hot_linear_backward_rng")
        if grads is None:
            grads = [torch.empty(layer.s_local, xd.shape[-2], layer.in_features, dtype=torch.float32, device=xd.device) if want_dx else None]
            grads += [torch.empty_like(t) if t is not None else None for t in (mu_w, sigma_w, mu_b, sigma_b)]
            ws = _scratch(ws_bytes, least, xd.device)
            hot.hot_linear_backward_rng(hot.hot_rng(*draw), xd, grad_y, mu_w, sigma_w, mu_b, sigma_b, *grads[1:], grads[0],
                                        layer.s_local, layer.dataset_size, hot.HOT_REDUCE_NONE, layer.weight_offset,
                                        layer.bias_offset, workspace=ws)
        dx = grads[0]
        if dx is not None and xd.dim() == 2:
            dx = dx.sum(0)          # a shared input collects every sample's share
        return (dx, *grads[1:], None, None)


class BayesianLinear:
    """One mean-field Gaussian linear layer on the fused kernels.  `weight_offset` places the layer in
    the flat parameter vector of the network (it selects the generator's counters, so two layers must
    not overlap); `next_offset` is where the following layer may start.  forward(x, ...) takes the
    minibatch [R, K] (first layer) or one input per sample [S_loc, R, K] and returns y [S_loc, R, O];
    the gradients it hands to autograd include the KL part divided by dataset_size."""

    def __init__(self, in_features: int, out_features: int, s_local: int, dataset_size: float, bias: bool = True,
                 seed: int = 0, first_sample: int = 0, weight_offset: int = 0):
        if in_features % 4 or weight_offset % 4:
            raise ValueError("in_features and weight_offset must be multiples of 4")
        self.in_features, self.out_features, self.s_local = in_features, out_features, s_local
        self.dataset_size, self.seed, self.first_sample, self.bias = float(dataset_size), seed, first_sample, bias
        self.weight_offset = weight_offset
        self.bias_offset = weight_offset + in_features * out_features        # a multiple of 4 as well
        self.next_offset = (self.bias_offset + (out_features if bias else 0) + 3) // 4 * 4

    def kl(self, mu_w, sigma_w, mu_b=None, sigma_b=None) -> torch.Tensor:
        """The layer's KL term (one float64 on the device, detached; its gradient is added by backward)."""
        sizes = [self.in_features * self.out_features] + ([self.out_features] if self.bias else [])
        if sum(sizes) <= hot.HOT_KL_LAYER_MAX and mu_w.is_cuda:           # (small layers: one launch)
            parts = (mu_w, sigma_w, mu_b, sigma_b) if self.bias else (mu_w, sigma_w, None, None)
            out = _answer(hot.host().kl_layer(*parts, sizes[0], sizes[1] if self.bias else 0, *_device_and_stream()), "hot_kl_layer")
            if out is not None:
                return out
        if not hasattr(self, "_kl_plans"):
            dev = mu_w.device.index or 0
            self._kl_plans = [hot.hot_create(n, n, 1, 1, self.dataset_size, dev) for n in sizes]
        out = torch.empty(len(self._kl_plans), dtype=torch.float64, device=mu_w.device)       # (each call below writes its element)
        hot.hot_kl(self._kl_plans[0], mu_w.detach().reshape(-1), sigma_w.detach().reshape(-1), out[0:1])
        if self.bias:
            hot.hot_kl(self._kl_plans[1], mu_b.detach(), sigma_b.detach(), out[1:2])
        return out.sum()

    def forward(self, x, mu_w, sigma_w, mu_b, sigma_b, step: int):
        if self.bias == (mu_b is None):
            raise ValueError("bias arrays do not match the layer's bias setting")
        return _Linear.apply(x, mu_w, sigma_w, mu_b, sigma_b, self, int(step))


class BayesianModule(torch.nn.Module):
    """Any torch.nn.Module with all of its parameters made mean-field Gaussian: the module's
    parameters are flattened into one vector, `mu` starts at their current values, `sigma` at
    sqrt(kappa / fan_in) per parameter tensor (a constant that shrinks with the layer width, as the
    paper's experiments initialise it), and every forward call draws S_loc weight samples with the
    library, runs the module once per sample on views of the sampled vector, and returns the stacked
    outputs [S_loc, ...] with the KL term (detached; its gradient, divided by dataset_size, reaches
    mu.grad and sigma.grad through the backward kernel)."""

    def __init__(self, module: torch.nn.Module, s_local: int, dataset_size: float, kappa: float = 0.01, seed: int = 0,
                 first_sample: int = 0):
        super().__init__()
        self.module = module
        params = list(module.named_parameters())
        if not params:
            raise ValueError("the module has no parameters")
        device = params[0][1].device
        self._slices, at = [], 0
        for name, p in params:
            self._slices.append((name, at, at + p.numel(), tuple(p.shape)))
            at += p.numel()
        flat = torch.cat([p.detach().reshape(-1).float() for _, p in params])
        spread = torch.cat([torch.full((p.numel(),), (kappa / (p[0].numel() if p.dim() > 1 else p.numel())) ** 0.5)
                            for _, p in params]).to(device)
        self.mu = torch.nn.Parameter(flat.clone())
        self.sigma = torch.nn.Parameter(spread)
        for _, p in params:
            p.requires_grad_(False)             # the module's own tensors are only shape templates from here on
        self.layer = GaussianSampleLayer(at, s_local, dataset_size, device.index or 0, seed, first_sample)

    def forward(self, *inputs, step: int):
        w, kl = self.layer.sample(self.mu, self.sigma, step)
        outs = []
        for s in range(self.layer.s_local):
            sampled = {name: w[s, a:b].view(shape) for name, a, b, shape in self._slices}
            outs.append(torch.func.functional_call(self.module, sampled, inputs))
        return torch.stack(outs), kl


# ------------------------------------------------------------------ layer norm, and a head's loss over a vocabulary

def _adjacent(t):
    """t, or a copy whose last axis is adjacent in memory."""
    return t if t.shape[-1] < 2 or t.stride(-1) == 1 else t.contiguous()


def _apart(weight):
    """weight [..., vocab, width], or a copy where its rows or samples lie between each other (one set for all samples is left as it is)."""
    weight = _adjacent(weight)
    vocab, width = weight.shape[-2:]
    rows = weight.stride(-2) if vocab > 1 else width
    between = rows < width or (weight.dim() == 3 and weight.shape[0] > 1 and 0 < weight.stride(0) < (vocab - 1) * rows + width)
    return weight.contiguous() if between else weight


class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, per_sample):
        samples = x.shape[0] if per_sample else 1
        x3 = _adjacent(x).reshape(samples, -1, x.shape[-1])
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        keep = any(ctx.needs_input_grad[:3])
        mean, rstd = torch.empty(2, *x3.shape[:2], dtype=torch.float32, device=x.device) if keep else (None, None)
        hot.hot_norm_forward(x3, weight, bias, eps, y.view(x3.shape), mean, rstd)
        if keep:
            ctx.save_for_backward(x3, weight, bias, mean, rstd)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x3, weight, bias, mean, rstd = ctx.saved_tensors
        want_x, want_w, want_b = ctx.needs_input_grad[:3]
        dx = torch.empty(dy.shape, dtype=x3.dtype, device=dy.device) if want_x else None
        dw = torch.empty_like(weight) if want_w else None
        db = torch.empty_like(bias) if want_b else None
        ws = None
        if want_w or want_b:
            ws = torch.empty(hot.hot_norm_backward_workspace_bytes(x3, weight if weight is not None else bias) // 4, dtype=torch.float32, device=dy.device)
        hot.hot_norm_backward(x3, weight, mean, rstd, _adjacent(dy).reshape(x3.shape), dx.view(x3.shape) if want_x else None, dw, db, ws)
        return dx, dw, db, None, None


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5) -> torch.Tensor:
    """Layer norm of x [..., width] over the last axis, differentiable in x, weight and bias.  weight and bias: [width], or
    [S, width] with x [S, ..., width], where weight sample s (a row of what GaussianSampleLayer draws) belongs to x[s]; either may be
    None.  x: float32, bfloat16 or float16, which y has too; weight and bias: of x's type or float32.  Statistics and sums are float32."""
    if x.is_cuda:
        y = hot.host().layer_norm(x, weight, bias, eps, torch.cuda.current_device())
        if y is not None:           # (dense and on the current device: the call, its checks and its backward pass in native code)
            return y
    if x.dim() < 1 or x.shape[-1] < 1:
        raise ValueError(f"x: need [..., width] with a width, got {tuple(x.shape)}")
    shaped = weight if weight is not None else bias
    per_sample = shaped is not None and shaped.dim() == 2
    if per_sample and (x.dim() < 2 or shaped.shape[0] != x.shape[0]):
        raise ValueError(f"weights of {shaped.shape[0]} samples need x [{shaped.shape[0]}, ..., width], got {tuple(x.shape)}")
    weight, bias = (t.contiguous() if t is not None else None for t in (weight, bias))
    return _Norm.apply(x, weight, bias, float(eps), per_sample)


class _Head(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, index, logit, ignore_index, temperature):
        loss = torch.empty(weight.shape[0], x.shape[1], dtype=torch.float32, device=x.device)
        keep = any(ctx.needs_input_grad[:3])
        lse = torch.empty(loss.shape, dtype=torch.float64, device=x.device) if keep else None
        hot.hot_head_forward(x, weight, bias, index, logit, loss, lse, ignore_index, temperature)
        if keep:
            ctx.save_for_backward(x, weight, bias, index, logit, lse)
            ctx.rule = (ignore_index, temperature)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        x, weight, bias, index, logit, lse = ctx.saved_tensors
        if ctx.needs_input_grad[0] and x.shape[0] > 1 and x.stride(0) == 0:
            x = x.contiguous()          # (features expanded over the samples: on one memory the call forms one gradient for all of them)
        dx, dw, db = (torch.empty(t.shape, dtype=t.dtype, device=t.device) if want else None for t, want in zip((x, weight, bias), ctx.needs_input_grad[:3]))
        hot.hot_head_backward(x, weight, bias, index, logit, lse, grad_loss, dx, dw, db, *ctx.rule)
        return dx, dw, db, None, None, None, None


def _head(x, weight, bias, index, logit, ignore_index, temperature, entries: int):
    """Shapes of a user's call to those of the binding; `entries`: axes of index behind the rows'."""
    if x.is_cuda:
        loss = hot.host().head_loss(x, weight, bias, index, logit, ignore_index, temperature, torch.cuda.current_device())
        if loss is not None:
            return loss
    if not isinstance(weight, torch.Tensor) or weight.dim() not in (2, 3):
        raise ValueError("weight: need [vocab, width] or [S, vocab, width]")
    if x.dim() < 1 or x.shape[-1] != weight.shape[-1]:
        raise ValueError(f"x: need [..., {weight.shape[-1]}], got {tuple(x.shape)}")
    if bias is not None and bias.shape != weight.shape[:-1]:
        raise ValueError(f"bias: need {tuple(weight.shape[:-1])}, got {tuple(bias.shape)}")
    width, tail = x.shape[-1], index.shape[index.dim() - entries:]
    x, weight = _adjacent(x), _apart(weight)
    if weight.dim() == 2:
        shape = x.shape[:-1]
        if index.shape[:index.dim() - entries] != shape:
            raise ValueError(f"targets: need {tuple(shape)} rows, got {tuple(index.shape)}")
        x3, weight = x.reshape(1, -1, width), weight.unsqueeze(0)
        bias = bias.unsqueeze(0) if bias is not None else None
        index = index.reshape(1, -1, *tail)
        logit = logit.reshape(index.shape) if logit is not None else None
    else:
        # [rows, width]: the same rows for every sample; [S, ..., width]: its own; targets for all samples or for each
        samples = weight.shape[0]
        own = x.dim() > 2
        if own and x.shape[0] != samples:
            raise ValueError(f"x: need [{samples}, ..., width] or [rows, width], got {tuple(x.shape)}")
        rows = x.shape[1:-1] if own else x.shape[:-1]
        x3 = x.reshape(samples if own else 1, -1, width)
        shape = (samples, *rows)
        lead = index.shape[:index.dim() - entries]
        if lead not in (torch.Size(rows), torch.Size(shape)):
            raise ValueError(f"targets: need {tuple(rows)} or {tuple(shape)} rows, got {tuple(index.shape)}")
        sets = samples if len(lead) == len(shape) else 1
        index = index.reshape(sets, -1, *tail)
        logit = logit.reshape(index.shape) if logit is not None else None
    if logit is not None:
        index, logit = _adjacent(index), _adjacent(logit)
    bias = _adjacent(bias) if bias is not None else None
    return _Head.apply(x3, weight, bias, index, logit, int(ignore_index), float(temperature)).reshape(shape)


def head_cross_entropy(x, weight, target, bias=None, ignore_index: int = -100) -> torch.Tensor:
    """Cross entropy of the rows of a linear head, float32, from the features in front of it: ln sum_v exp(z_v) - z_target with
    z = x weight^T + bias, without logits in memory; differentiable in x, weight and bias.  x [..., width], weight [vocab, width],
    bias [vocab] or None, target int64 [...]; or one head per weight sample: weight [S, vocab, width], bias [S, vocab], x
    [S, ..., width] or [rows, width] (which every sample then sees, and whose gradient is formed once), target with or without the samples' axis.  Rows whose target is
    ignore_index have loss 0 and take no part; a loss over the others is loss.sum() / their number.  x, weight and bias have one type:
    float32, bfloat16 or float16."""
    return _head(x, weight, bias, target, None, ignore_index, 1.0, 0)


def head_distillation(x, weight, top_index, top_logit, bias=None, temperature: float = 1.0) -> torch.Tensor:
    """T^2 KL(p || softmax(z / T)) of the rows of a linear head (see head_cross_entropy for x, weight, bias and samples), float32, where
    p = softmax(top_logit / T) over a teacher's likeliest words top_index (int64 [..., top], negative: not there); differentiable in
    x, weight and bias, not in the teacher.  Words that are not listed have p = 0 but count in the student's softmax.  A row that lists
    nothing has loss 0 and takes no part."""
    if top_index.dim() < 1 or top_index.shape != top_logit.shape:
        raise ValueError(f"top_index and top_logit: need one shape, got {tuple(top_index.shape)} and {tuple(top_logit.shape)}")
    if not 1 <= top_index.shape[-1] <= hot.HOT_HEAD_MOST_TOP:
        raise ValueError(f"top_index: need 1 to {hot.HOT_HEAD_MOST_TOP} words a row, got {top_index.shape[-1]}")
    return _head(x, weight, bias, top_index, top_logit.detach(), -100, temperature, 1)


# ------------------------------------------------------------------ dropout, the end of a block, attention

def _counter(rng, keep: float):
    if rng is None:
        if keep != 1.0:
            raise ValueError("rng: dropout needs a hot_rng")
        return 0, 0, 0
    return rng.seed, rng.step, rng.first_sample


def dropout(x, keep: float, rng, samples: int = 0, offset: int = 0) -> torch.Tensor:
    """Dropout of activations x [..., width] (with samples = S: [S, ..., width], one mask per Monte-Carlo sample): an element stays with probability keep, in
    steps of 2^-16, and is divided by it; the others are zeros.  Which ones stay follows from rng (binding.hot_rng: seed, step, first_sample, the
    global number of sample 0) and the element's place alone, so no mask is stored, the backward pass draws it again, and GPUs that share a seed draw
    different samples.  Layers of one network take disjoint ranges of offset: dropout_calls(x, samples) calls of the generator each.
    float32, bfloat16 or float16; differentiable any number of times."""
    if not isinstance(rng, hot.hot_rng):
        raise TypeError("rng: need a hot_rng")
    return hot.host().dropout(x, float(keep), rng.seed, rng.step, rng.first_sample, int(samples), int(offset))


def dropout_calls(x, samples: int = 0) -> int:
    """Calls of the generator that a sample of x [..., width] takes: the next layer's offset lies that much further."""
    width = x.shape[-1]
    return x.numel() // width // (samples or 1) * ((width + 7) // 8)


def residual_norm(x, branch, weight=None, bias=None, *, norm: str | None = "layer", gate=None, scale: float = 1.0, branch_norm: str | None = None, branch_weight=None,
                  branch_bias=None, keep: float = 1.0, rng=None, samples: int = 0, offset: int = 0, eps: float = 1e-5):
    """The end of a block and the norm that begins the next: (h, y) with h = x + scale gate dropout(norm'(branch)) and y = norm(h), in one pass, differentiable
    in all tensors.  norm, branch_norm (norm'): "layer", "rms" or None (norm None: y is None).  x, branch: [..., width] of one type, float32, bfloat16 or float16,
    width up to 16384; weight, bias, gate, branch_weight, branch_bias: [width], or with samples = S and x [S, ..., width] also [S, width], x's type or float32
    (all of them one), None for ones and zeros.  keep, rng, samples, offset: as in dropout; keep = 1 leaves it out.  y is the norm of h before h is rounded
    to x's type."""
    for kind, name in ((norm, "norm"), (branch_norm, "branch_norm")):
        if kind not in hot.HOT_NORMS:
            raise ValueError(f"{name}: need 'layer', 'rms' or None, got {kind!r}")
    if rng is not None and not isinstance(rng, hot.hot_rng):
        raise TypeError("rng: need a hot_rng")
    out = hot.host().block_end(x, branch, weight, bias, gate, branch_weight, branch_bias, hot.HOT_NORMS[norm], hot.HOT_NORMS[branch_norm], float(scale), float(keep),
                               float(eps), *_counter(rng, keep), int(samples), int(offset))
    return out[0], (out[1] if len(out) > 1 else None)


class RelativePositions:
    """Where queries and keys stand, for attention's bias: whole-number codes of both, and for every difference query code - key code, from the smallest on,
    which of `buckets` rows of the table it takes.  Made once and kept; distances() and windows() make the usual ones."""

    def __init__(self, query_codes, key_codes, bucket_of, buckets: int, device):
        query, key, bucket = (torch.as_tensor(t).detach().cpu() for t in (query_codes, key_codes, bucket_of))
        for t, name in ((query, "query_codes"), (key, "key_codes"), (bucket, "bucket_of")):
            if t.dim() != 1 or t.numel() < 1 or t.is_floating_point() or t.is_complex() or t.dtype == torch.bool:
                raise ValueError(f"{name}: need a vector of whole numbers, got {tuple(t.shape)} of {t.dtype}")
        query, key, bucket = query.long(), key.long(), bucket.long()
        codes = int(query.max()) - int(key.min()) - (int(query.min()) - int(key.max())) + 1
        if not 1 <= codes <= hot.HOT_ATTENTION_MOST_CODES:
            raise ValueError(f"codes: need at most {hot.HOT_ATTENTION_MOST_CODES} differences, got {codes}")
        if bucket.numel() != codes:
            raise ValueError(f"bucket_of: need a bucket for each of {codes} differences, got {bucket.numel()}")
        if not 1 <= buckets <= hot.HOT_ATTENTION_MOST_BUCKETS:
            raise ValueError(f"buckets: need 1 to {hot.HOT_ATTENTION_MOST_BUCKETS}, got {buckets}")
        if int(bucket.min()) < 0 or int(bucket.max()) >= buckets:
            raise ValueError(f"bucket_of: need 0 to {buckets - 1}, got {int(bucket.min())} to {int(bucket.max())}")
        self.queries, self.keys, self.buckets = query.numel(), key.numel(), int(buckets)
        query, key = query - query.min(), key - key.max()

        def ranges(code):
            tiles = torch.nn.functional.pad(code, (0, -len(code) % 64), value=int(code[-1])).view(-1, 64)
            steps = torch.ones_like(tiles).view(-1)             # (whether the code behind a token's is one more; the last token has none behind)
            steps[:len(code) - 1] = code[1:] - code[:-1] == 1
            return torch.stack([tiles.amin(1), tiles.amax(1), steps.view(-1, 64).amin(1), torch.zeros(len(tiles), dtype=code.dtype)], 1)

        # the last difference of the run of equal buckets that each lies in
        ends = torch.cat([bucket[1:] != bucket[:-1], torch.tensor([True])]).nonzero()[:, 0]
        runs = torch.stack([bucket, ends[torch.searchsorted(ends, torch.arange(codes))]], 1)
        self.query_code, self.key_code, self.query_range, self.key_range, self.bucket = (
            t.to(torch.int32).contiguous().to(device) for t in (query, key, ranges(query), ranges(key), runs))

    @classmethod
    def distances(cls, queries: int, keys: int, buckets: int, furthest: int, device, both_sides: bool = True, first_query: int = 0):
        """Tokens on a line, query i at first_query + i, key j at j: half of the buckets (of a side, where both_sides) for one distance each, the others for ranges that
        grow with the logarithm up to `furthest` and hold what is further.  One-sided, keys behind the query share the bucket of distance 0."""
        side = buckets // 2 if both_sides else buckets
        near = side // 2
        if near < 1 or furthest <= near or (both_sides and buckets % 2):
            raise ValueError(f"buckets and furthest: need an even number of buckets of at least {4 if both_sides else 2} and a distance beyond {max(near, 1)}, got {buckets} and {furthest}")
        if queries < 1 or keys < 1:
            raise ValueError(f"queries and keys: need at least one, got {queries} and {keys}")
        query, key = torch.arange(queries) + first_query, torch.arange(keys)
        distance = torch.arange(int(query[0]) - int(key[-1]), int(query[-1]) + 1)
        away = distance.abs() if both_sides else distance.clamp(min=0)
        far = near + (torch.log(away.clamp(min=1).double() / near) / math.log(furthest / near) * (side - near)).long()
        bucket = torch.where(away < near, away, far.clamp(max=side - 1))
        return cls(query, key, bucket + side * (distance < 0) if both_sides else bucket, buckets, device)

    @classmethod
    def windows(cls, *extent: int, device):
        """The tokens of a window of extent[0] x extent[1] x ... in order of memory, a row of the table for every difference of places: prod(2 extent - 1) buckets, in
        order of the differences from the smallest on, the last axis fastest."""
        if not extent or min(extent) < 1:
            raise ValueError(f"extent: need at least one axis of at least one token, got {extent}")
        place, code = torch.meshgrid(*(torch.arange(n) for n in extent), indexing="ij"), 0
        for axis, n in zip(place, extent):
            code = code * (2 * n - 1) + axis
        code = code.reshape(-1)
        span = 2 * int(code[-1]) + 1
        return cls(code, code, torch.arange(span), span, device)


def attention(q, k, v, table=None, positions: RelativePositions | None = None, *, scale: float | None = None, causal: bool = False, query_groups=None, key_groups=None,
              first_query: int = 0) -> torch.Tensor:
    """softmax over the keys of scale q k^T + bias, times v, without scores in memory; differentiable in q, k, v and table.
    q [..., heads, queries, width], k and v [..., kv heads, keys, width], kv heads dividing heads, width 8 to 128; float32, bfloat16 or float16, any strides with adjacent
    elements of a row (the result's and the gradients' tokens lie as [..., tokens, heads, width] where q, k and v are no dense arrays of their own).  scale: 1 / sqrt(width) where None.
    The bias of head h is table[bucket, h] with the bucket of positions for the two tokens' codes: table [buckets, heads], or [S, buckets, heads] with one table per
    weight sample and q [S, ..., heads, queries, width]; q's type or float32.  Query i is query first_query + i of positions, so one object serves single tokens of a
    growing text.
    Causal: query i sees keys up to i + keys - queries.  query_groups, key_groups: int32 [queries] and [keys], or [entries, ...], row b mod entries for entry b of q's
    flattened leading axes; a query sees the keys of its own group (texts packed into a row, pieces of a shifted window), negative groups are padding
    and whatever lies there reaches nothing (keys and values that order or another group hides have to be finite: their weight is a zero that is multiplied).
    key_groups alone: all queries are of group 0.  A query that sees nothing gives zeros and has no gradients.
    A backward pass that is captured into a graph while an eager graph of the same leaves lives raises RuntimeError (dropout's and residual_norm's too)."""
    if table is not None and not isinstance(positions, RelativePositions):
        raise TypeError("positions: a table needs RelativePositions")
    if not isinstance(q, torch.Tensor):
        raise TypeError("q: need a tensor")
    p = (positions.query_code, positions.key_code, positions.query_range, positions.key_range, positions.bucket, positions.buckets) if table is not None else (None,) * 5 + (0,)
    return hot.host().attention(q, k, v, table, *p, query_groups, key_groups, int(first_query), float(scale if scale is not None else max(q.shape[-1:] or (1,)) ** -0.5), bool(causal))
