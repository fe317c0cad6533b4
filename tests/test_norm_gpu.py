"""Layer norm (autograd.layer_norm, hot_norm_*) against the plain form in 64 bits: types, widths around every kernel's limits, weight samples,
strides, rows that are no numbers, gradients against differences, refusals."""
import pytest
import torch

import head_norm_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ops():
    from paper_2604_04736_amd import autograd
    return autograd


def _inputs(kind, samples, rows, width, weights="both", weight_kind=None, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + rows * 7 + width)
    dt, wt = U.TYPES[kind], U.TYPES[weight_kind or kind]
    sets = (samples,) if samples else ()
    x = (torch.randn(*sets, rows, width, device=DEV, generator=g) * 2 + torch.randn(*sets, rows, 1, device=DEV, generator=g)).to(dt)
    w = (1 + 0.3 * torch.randn(*sets, width, device=DEV, generator=g)).to(wt) if weights in ("both", "weight") else None
    b = (0.5 * torch.randn(*sets, width, device=DEV, generator=g)).to(wt) if weights in ("both", "bias") else None
    dy = torch.randn(*sets, rows, width, device=DEV, generator=g).to(dt)
    return x, w, b, dy


def _pass(x, w, b, dy, eps=1e-5):
    leaves = [t.detach().requires_grad_() if t is not None else None for t in (x, w, b)]
    y = _ops().layer_norm(*leaves, eps=eps)
    there = [(n, t) for n, t in zip(("dx", "dw", "db"), leaves) if t is not None]
    return {"y": y.detach(), **dict(zip([n for n, _ in there], torch.autograd.grad(y, [t for _, t in there], dy)))}


def _check(x, w, b, dy, eps=1e-5):
    got = _pass(x, w, b, dy, eps)
    three = x.dim() == 3
    x3, dy3 = (x, dy) if three else (x.reshape(1, -1, x.shape[-1]), dy.reshape(1, -1, x.shape[-1]))
    want = U.norm_plain(x3, w, b, eps, dy3)
    shaped = {"y": x.shape, "dx": x.shape, "dw": w.shape if w is not None else None, "db": b.shape if b is not None else None}
    if w is None and b is not None:                      # (the plain form types the sums by the weight)
        db, off = want["db"]
        want["db"] = (db, off - U.rounded(db, x.dtype) + U.rounded(db, b.dtype))
    for name, v in got.items():
        assert v.dtype == {"y": x, "dx": x, "dw": w, "db": b}[name].dtype
        ref, bound = want[name]
        U.within(v, ref.reshape(shaped[name]), bound.reshape(shaped[name]), f"{name} {tuple(x.shape)} {x.dtype}")
    again = _pass(x, w, b, dy, eps)
    assert all(torch.equal(got[n], again[n]) for n in got)
    return got


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width", [1, 2, 7, 8, 9, 63, 64, 128, 129, 192, 257, 511, 777, 1025, 2048, 2049, 4097, 8192, 8193, 16385, 40001])
def test_widths(kind, width):
    for rows in (1, 37):
        _check(*_inputs(kind, 0, rows, width))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("samples,rows,width", [(1, 5, 40), (2, 300, 192), (3, 65, 777), (5, 1, 4100), (2, 3, 20000), (7, 33, 16)])
def test_weight_samples(kind, samples, rows, width):
    _check(*_inputs(kind, samples, rows, width))


@pytest.mark.parametrize("rows,width", [(2000, 64), (5003, 100), (40000, 16), (3000, 1000)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_many_rows(kind, rows, width):
    _check(*_inputs(kind, 0, rows, width))


@pytest.mark.parametrize("kind,weight_kind", [("bf16", "f32"), ("f16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("weights", ["both", "weight", "bias", "none"])
def test_weights_given_or_not_and_their_type(kind, weight_kind, weights):
    for samples in (0, 2):
        _check(*_inputs(kind, samples, 21, 200, weights, weight_kind))


def test_shared_weights_of_a_batch_of_sequences():
    x, w, b, dy = _inputs("bf16", 0, 60, 96)
    flat = _check(x, w, b, dy)
    batch = _pass(x.view(3, 4, 5, 96), w, b, dy.view(3, 4, 5, 96))
    assert all(torch.equal(batch[n].reshape(flat[n].shape), flat[n]) for n in flat)
    own = _pass(x.view(2, 5, 6, 96), torch.stack([w, w]), torch.stack([b, b]), dy.view(2, 5, 6, 96))
    assert torch.equal(own["y"].reshape(60, 96), flat["y"]) and torch.equal(own["dx"].reshape(60, 96), flat["dx"])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_layouts_in_memory(kind):
    x, w, b, dy = _inputs(kind, 0, 30, 100)
    want = _pass(x, w, b, dy)
    wide = torch.zeros(30, 133, device=DEV, dtype=x.dtype)
    wide[:, 5:105] = x                                           # rows that lie apart and on odd elements
    rows_apart = wide[:, 5:105]
    across = x.t().contiguous().t()
    every_other = torch.stack([x, x], 1).reshape(60, 100)[::2]
    for v in (rows_apart, across, every_other):
        got = _pass(v, w, b, dy)
        assert all(torch.equal(got[n], want[n]) for n in want)
    got = _pass(x, w, b, dy.t().contiguous().t())
    assert all(torch.equal(got[n], want[n]) for n in want)
    odd = torch.zeros(101, device=DEV, dtype=w.dtype)[1:]
    odd.copy_(w)
    got = _pass(x, odd, b, dy)
    assert all(torch.equal(got[n], want[n]) for n in want)
    # a gradient that is the same everywhere: no strides at all
    leaf = x.detach().requires_grad_()
    _ops().layer_norm(leaf, w, b).sum().backward()
    ones = _pass(x, w, b, torch.ones_like(x))
    assert torch.equal(leaf.grad, ones["dx"])
    # the same row everywhere
    got = _pass(x[:1].expand(30, 100), w, b, dy)
    dense = _pass(x[:1].repeat(30, 1), w, b, dy)
    assert all(torch.equal(got[n], dense[n]) for n in got)


def test_weights_that_are_views_of_a_sampled_vector():
    """[S, N] as the sample layer draws it: the norm's weights lie anywhere in a sample's row, and gradients reach the vector."""
    drawn = torch.randn(3, 1001, device=DEV).requires_grad_()
    x = torch.randn(3, 20, 70, device=DEV)
    y = _ops().layer_norm(x, drawn[:, 5:75], drawn[:, 75:145])
    dy = torch.randn_like(y)
    y.backward(dy)
    want = U.norm_plain(x, drawn[:, 5:75].detach(), drawn[:, 75:145].detach(), 1e-5, dy)
    U.within(y, *want["y"], "y")
    U.within(drawn.grad[:, 5:75], *want["dw"], "dw")
    U.within(drawn.grad[:, 75:145], *want["db"], "db")
    assert not drawn.grad[:, 145:].any() and not drawn.grad[:, :5].any()


@pytest.mark.parametrize("width", [48, 777, 9000, 40001])
def test_rows_that_are_no_numbers_stay_alone(width):
    x, w, b, dy = _inputs("f32", 0, 9, width)
    clean = _pass(x, w, b, dy)
    x[2, width // 2], x[5, 0], x[7, width - 1] = float("nan"), float("inf"), -float("inf")
    got = _pass(x, w, b, dy)
    bad = torch.tensor([2, 5, 7], device=DEV)
    fine = torch.tensor([0, 1, 3, 4, 6, 8], device=DEV)
    for n in ("y", "dx"):
        assert torch.equal(got[n][fine], clean[n][fine]) and torch.isnan(got[n][bad]).any(1).all()
    assert torch.equal(got["db"], clean["db"])


def test_rows_without_spread_and_large_values():
    x = torch.full((4, 96), 3.0, device=DEV)
    x[1] = 0
    got = _pass(x, None, torch.full((96,), 0.25, device=DEV), torch.ones_like(x))
    assert torch.equal(got["y"], torch.full_like(x, 0.25)) and not got["dx"].any()
    x = torch.randn(5, 300, device=DEV) + 3e4                    # a mean far above the spread
    want = U.norm_plain(x[None], None, None, 1e-5, x[None])["y"]
    U.within(_ops().layer_norm(x), want[0][0], want[1][0], "y")


def test_gradients_against_differences():
    x, w, b, dy = (t.double() for t in _inputs("f32", 2, 6, 50))
    got = _pass(x.float(), w.float(), b.float(), dy.float())
    gen = torch.Generator(device=DEV).manual_seed(3)
    for name, t in (("dx", x), ("dw", w), ("db", b)):
        way = torch.randn(t.shape, device=DEV, generator=gen, dtype=torch.float64)
        step = 2.0 ** -8

        def loss(v):
            args = {"dx": (v, w, b), "dw": (x, v, b), "db": (x, w, v)}[name]
            return float((_ops().layer_norm(*(a.float() for a in args)).double() * dy).sum())
        # third differences are below 1 and the forward pass is good for 2^-21 of the sum's terms
        slope = (loss(t + step * way) - loss(t - step * way)) / (2 * step)
        size = float(dy.abs().sum()) * 4
        assert abs(slope - float((got[name].double() * way).sum())) <= size * (2.0 ** -21 / step + step * step), name


def test_no_rows():
    for samples in (0, 2):
        x, w, b, dy = _inputs("bf16", samples, 0, 24)
        got = _pass(x, w, b, dy)
        assert got["y"].shape == x.shape and got["dx"].shape == x.shape and not got["dw"].any() and not got["db"].any()


def test_only_what_is_asked_for():
    x, w, b, dy = _inputs("f32", 0, 40, 130)
    full = _pass(x, w, b, dy)
    for wanted in (("dx",), ("dw",), ("db",), ("dx", "db"), ("dw", "db")):
        leaves = {n: t.detach().requires_grad_(n in wanted) for n, t in zip(("dx", "dw", "db"), (x, w, b))}
        y = _ops().layer_norm(leaves["dx"], leaves["dw"], leaves["db"])
        grads = torch.autograd.grad(y, [leaves[n] for n in wanted], dy)
        assert all(torch.equal(a, full[n]) for a, n in zip(grads, wanted))
    assert not _ops().layer_norm(x, w, b).requires_grad


def test_differentiable_once():
    x = torch.randn(4, 16, device=DEV, requires_grad=True)
    for v in (x, x.t().contiguous().t()):
        (dx,) = torch.autograd.grad(_ops().layer_norm(v).square().sum(), v, create_graph=True)
        with pytest.raises(RuntimeError):
            dx.sum().backward()


def test_another_stream_and_replays_of_a_graph():
    x, w, b, dy = _inputs("bf16", 0, 500, 640)
    want = _pass(x, w, b, dy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _pass(x, w, b, dy)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(got[n], want[n]) for n in want)

    from paper_2604_04736_amd import binding as hot
    x3, dy3 = x[None].clone(), dy[None].clone()
    y, dx, dw, db = torch.empty_like(x3), torch.empty_like(x3), torch.empty_like(w), torch.empty_like(b)
    mean, rstd = torch.empty(2, 1, 500, device=DEV)
    ws = torch.empty(hot.hot_norm_backward_workspace_bytes(x3, w), dtype=torch.uint8, device=DEV)

    def step():
        hot.hot_norm_forward(x3, w, b, 1e-5, y, mean, rstd)
        hot.hot_norm_backward(x3, w, mean, rstd, dy3, dx, dw, db, ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(3):
        xs, _, _, ds = _inputs("bf16", 0, 500, 640, seed=seed + 1)
        x3.copy_(xs[None])
        dy3.copy_(ds[None])
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        want = _pass(xs, w, b, ds)
        for n, v in (("y", y[0]), ("dx", dx[0]), ("dw", dw), ("db", db)):
            assert torch.equal(v, want[n]), (n, seed)


def test_offsets_beyond_32_bits():
    rows, width = 70000, 32768                                    # 4.6 GB
    x = torch.empty(rows, width, dtype=torch.bfloat16, device=DEV)
    x[:, :] = torch.randn(1, width, device=DEV).to(x.dtype)
    x[-3:] = torch.randn(3, width, device=DEV).to(x.dtype)
    y = _ops().layer_norm(x)
    want = U.norm_plain(x[None, -3:], None, None, 1e-5, x[None, -3:])["y"]
    U.within(y[-3:], want[0][0], want[1][0], "y")
    assert torch.equal(y[5], y[65000])


def test_refusals():
    ln = _ops().layer_norm
    x = torch.randn(4, 6, device=DEV)
    for bad in (lambda: ln(x.double()), lambda: ln(x.cpu()), lambda: ln(x, torch.ones(6, device=DEV).double()), lambda: ln(x, torch.ones(6, device=DEV, dtype=torch.bfloat16)),
                lambda: ln(x, torch.ones(6))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: ln(x, torch.ones(5, device=DEV)), lambda: ln(x, torch.ones(3, 6, device=DEV)), lambda: ln(x, torch.ones(6, device=DEV), torch.ones(4, 6, device=DEV)),
                lambda: ln(torch.zeros((), device=DEV)), lambda: ln(torch.zeros(4, 0, device=DEV)), lambda: ln(x, torch.ones(1, 4, 6, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(RuntimeError):
        ln(x, eps=-1.0)
