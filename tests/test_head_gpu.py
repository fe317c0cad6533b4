"""A linear head's losses over a vocabulary without logits (autograd.head_cross_entropy, head_distillation, hot_head_*) against the plain form in
64 bits: types, sizes around the tiles' edges, ragged and empty targets, masked words, weight samples, strides, pieces of the vocabulary,
gradients against differences, refusals."""
import math

import pytest
import torch

import head_norm_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"
NAN = float("nan")


def _ops():
    from paper_2604_04736_amd import autograd
    return autograd


def _inputs(kind, rows, width, vocab, samples=0, bias=False, shared_x=False, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + 31 * rows + 7 * width + vocab)
    dt, sets = U.TYPES[kind], (samples,) if samples else ()
    x = torch.randn(*(() if shared_x else sets), rows, width, device=DEV, generator=g).to(dt)
    w = (torch.randn(*sets, vocab, width, device=DEV, generator=g) * (2 / math.sqrt(width))).to(dt)
    b = torch.randn(*sets, vocab, device=DEV, generator=g).to(dt) if bias else None
    up = (torch.rand(*sets, rows, device=DEV, generator=g) + 0.5) * (64.0 if kind == "f16" else 1.0) / max(rows, 1)
    return x, w, b, up, g


def _pass(x, w, b, up, targets, **more):
    """targets: labels, or (index, logit)."""
    leaves = [t.detach().requires_grad_() if t is not None else None for t in (x, w, b)]
    if isinstance(targets, tuple):
        loss = _ops().head_distillation(leaves[0], leaves[1], *targets, bias=leaves[2], **more)
    else:
        loss = _ops().head_cross_entropy(leaves[0], leaves[1], targets, bias=leaves[2], **more)
    there = [(n, t) for n, t in zip(("dx", "dw", "db"), leaves) if t is not None]
    return {"loss": loss.detach(), **dict(zip([n for n, _ in there], torch.autograd.grad(loss, [t for _, t in there], up)))}


def _check(x, w, b, up, targets, temperature=1.0, name=""):
    more = {"temperature": temperature} if isinstance(targets, tuple) else {}
    got = _pass(x, w, b, up, targets, **more)
    w3 = w if w.dim() == 3 else w[None]
    x3 = x if x.dim() == 3 else x[None]
    b2 = b if b is None or b.dim() == 2 else b[None]
    up2 = up if up.dim() == 2 else up[None]
    vocab = w3.shape[1]
    if isinstance(targets, tuple):
        index, logit = (t if t.dim() == 3 else t[None] for t in targets)
        teach = U.teacher(index, logit, temperature, vocab)
    else:
        teach = U.labels(targets if targets.dim() == 2 else targets[None], vocab)
    want = U.head_plain(x3, w3, b2, teach, up2, temperature)
    assert got["loss"].dtype == torch.float32
    for n, v in got.items():
        ref, bound = want[n]
        like = {"loss": up, "dx": x, "dw": w, "db": b}[n]
        assert n == "loss" or v.dtype == like.dtype
        U.within(v, ref.reshape(like.shape), bound.reshape(like.shape), f"{n} {name} {tuple(x.shape)} {tuple(w.shape)} {x.dtype}")
    again = _pass(x, w, b, up, targets, **more)
    assert all(torch.equal(torch.nan_to_num(got[n]), torch.nan_to_num(again[n])) for n in got)
    return got


def _lists(g, rows, vocab, top, lead=(), ragged=True):
    index = torch.stack([torch.randperm(vocab, device=DEV, generator=g)[:top] for _ in range(rows * math.prod(lead))]).reshape(*lead, rows, top)
    logit = torch.randn(*lead, rows, top, device=DEV, generator=g) * 3
    if ragged:
        gone = torch.rand(*lead, rows, top, device=DEV, generator=g) < 0.3
        index[gone] = -1
        index[..., rows // 2, :] = -1                              # a row that lists nothing
        if top > 1:
            logit[..., 0, 0] = -math.inf
    return index, logit


# (rows, width, vocabulary): every size of tile, its edges, odd sizes, one of each
SIZES = [(1, 1, 1), (1, 8, 2), (2, 16, 31), (5, 24, 300), (31, 40, 257), (32, 64, 256), (33, 64, 64), (40, 7, 65), (64, 33, 130), (65, 192, 10), (129, 72, 1000), (128, 128, 4000),
         (257, 65, 3000), (300, 520, 5000), (513, 96, 16400), (1030, 48, 20000), (700, 200, 33000), (20, 36, 40000), (70, 44, 33001), (128, 33, 40000)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("rows,width,vocab", SIZES)
def test_labels(kind, bias, rows, width, vocab):
    x, w, b, up, g = _inputs(kind, rows, width, vocab, bias=bias)
    target = torch.randint(vocab, (rows,), device=DEV, generator=g)
    if bias:
        target[torch.rand(rows, device=DEV, generator=g) < 0.4] = -100
    _check(x, w, b, up, target)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width,vocab,top,temperature", [(1, 8, 2, 1, 1.0), (3, 40, 33, 33, 2.0), (32, 64, 500, 7, 0.7), (33, 33, 65, 65, 4.0), (64, 192, 1000, 8, 2.0), (200, 96, 2500, 130, 1.5),
                                                              (300, 64, 20000, 64, 2.0), (40, 16, 3000, 1024, 1.0), (520, 128, 33000, 20, 1.0)])
def test_a_teachers_words(kind, rows, width, vocab, top, temperature):
    x, w, b, up, g = _inputs(kind, rows, width, vocab, bias=top % 2 == 0)
    _check(x, w, b, up, _lists(g, rows, vocab, top), temperature)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("samples,rows,width,vocab", [(1, 10, 16, 20), (2, 40, 64, 257), (16, 64, 192, 10), (3, 5, 33, 700), (4, 300, 40, 3000)])
@pytest.mark.parametrize("shared_x", [False, True])
def test_weight_samples(kind, samples, rows, width, vocab, shared_x):
    x, w, b, up, g = _inputs(kind, rows, width, vocab, samples, bias=True, shared_x=shared_x)
    target = torch.randint(vocab, (rows,), device=DEV, generator=g)
    target[0] = -100
    _check(x, w, b, up, target, name="labels of all samples")
    own = torch.randint(vocab, (samples, rows), device=DEV, generator=g)
    own[torch.rand(samples, rows, device=DEV, generator=g) < 0.3] = -100
    _check(x, w, b, up, own, name="labels of each sample")
    top = min(vocab, 9)
    _check(x, w, b, up, _lists(g, rows, vocab, top), 2.0, "lists of all samples")
    _check(x, w, b, up, _lists(g, rows, vocab, top, (samples,)), 2.0, "lists of each sample")


@pytest.mark.parametrize("kind,rows,width,vocab", [("f32", 1500, 40, 60001), ("bf16", 4100, 24, 70001), ("f16", 9000, 16, 33333)])
def test_more_than_one_piece_of_the_vocabulary(kind, rows, width, vocab):
    x, w, b, up, g = _inputs(kind, rows, width, vocab, bias=True)
    target = torch.randint(vocab, (rows,), device=DEV, generator=g)
    target[::3] = vocab - 1 - target[::3] // 7
    target[1::5] = -100
    rows_seen = torch.cat([torch.arange(40, device=DEV), torch.arange(rows - 40, rows, device=DEV)])
    got = _pass(x, w, b, up, target)
    # in 64 bits a few rows, and as many words: those need all rows of a few words' columns, with every row's log sum of exponentials
    want = U.head_plain(x[rows_seen][None], w[None], b[None], U.labels(target[rows_seen][None], vocab), up[rows_seen][None])
    if kind != "f32":                   # (the bound of 80 rows is that of many)
        assert rows_seen.numel() > 32
    for n in ("loss", "dx"):
        U.within(got[n][rows_seen], want[n][0][0], want[n][1][0] + 2 ** -36 * float(up.max()) * (n == "dx"), n)
    words = torch.cat([torch.arange(30, device=DEV), torch.arange(vocab - 30, vocab, device=DEV), target[target >= 0][:20]])
    keep = target != -100
    z = x.double() @ w.double().T + b.double()
    lse = torch.logsumexp(z, 1)
    dz = (torch.exp(z[:, words] - lse[:, None]) - (target[:, None] == words).double()) * (up.double() * keep)[:, None]
    u = U.HALF_UNIT[x.dtype] * (4 if kind == "f32" else 1.01)
    z_off = (width / 16 + 24) * U.U32 * (x.double().abs() @ w.double().abs()[words].T + b.double().abs()[words])
    dz_off = u * dz.abs() + (up.double() * keep)[:, None] * torch.exp(z[:, words] - lse[:, None]) * (5 * z_off + 2 ** -18) + 2 ** -36 * float(up.max())
    for n, other, size in (("dw", x.double(), x.double().abs()), ("db", torch.ones(rows, 1, device=DEV, dtype=torch.float64), torch.ones(rows, 1, device=DEV, dtype=torch.float64))):
        ref = dz.T @ other
        bound = 1.01 * (dz_off.T @ size + (rows / 16 + 64) * U.U32 * (dz.abs().T @ size)) + U.rounded(ref, x.dtype)
        U.within(got[n][words].reshape(ref.shape), ref, bound, n)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [20, 90, 1200])
def test_rows_left_out_take_no_part(kind, rows):
    """Whatever rows without a label or a list hold, results are those of the other rows alone, bit for bit."""
    x, w, b, up, g = _inputs(kind, rows, 48, 700, bias=True)
    target = torch.randint(700, (rows,), device=DEV, generator=g)
    out = torch.rand(rows, device=DEV, generator=g) < 0.5
    target[out] = -100
    clean = _check(x, w, b, up, target)
    x[out] = torch.tensor([NAN, math.inf, -math.inf, 6e4] * 12, device=DEV).to(x.dtype)
    up[out] = NAN
    got = _pass(x, w, b, up, target)
    assert all(torch.equal(got[n], clean[n]) for n in got)
    assert not got["loss"][out].any() and not got["dx"][out].any()
    index, logit = _lists(g, rows, 700, 5, ragged=False)
    index[out] = -1
    logit[out] = NAN
    x[out] = 0
    up[out] = 1
    clean = _check(x, w, b, up, (index, logit), 2.0)
    x[out], up[out] = NAN, math.inf
    got = _pass(x, w, b, up, (index, logit), temperature=2.0)
    assert all(torch.equal(got[n], clean[n]) for n in got)
    # words with a teacher's logit of -inf are not there either
    index[out], logit[out] = 3, -math.inf
    got = _pass(x, w, b, up, (index, logit), temperature=2.0)
    assert all(torch.equal(got[n], clean[n]) for n in got)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shared_x", [False, True])
@pytest.mark.parametrize("rows,width,vocab", [(30, 40, 9000), (300, 72, 5000), (1500, 40, 20001)])
def test_as_many_rows_as_count_choose_the_runs_of_words(kind, shared_x, rows, width, vocab):
    """Samples of which all, a third, one, and none of the rows are labelled: each has runs of its own for its features' gradients."""
    x, w, b, up, g = _inputs(kind, rows, width, vocab, 4, False, shared_x)
    labels = torch.randint(0, vocab, (4, rows), device=DEV, generator=g)
    place = torch.rand(4, rows, device=DEV, generator=g).argsort(1)
    for s, kept in enumerate((rows, rows // 3, 1, 0)):
        labels[s, place[s, kept:]] = -100
    _check(x, w, b, up, labels)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_no_row_counts_and_no_rows(kind):
    for rows in (0, 1, 33, 1100):
        x, w, b, up, g = _inputs(kind, rows, 24, 90, bias=True)
        for targets in (torch.full((rows,), -100, device=DEV), (torch.full((rows, 3), -1, device=DEV), torch.zeros(rows, 3, device=DEV))):
            got = _pass(x, w, b, up, targets)
            assert got["loss"].shape == (rows,) and got["dx"].shape == x.shape
            assert not any(v.any() for v in got.values())
        x, w, b, up, g = _inputs(kind, rows, 24, 90, 3, bias=True, shared_x=True)
        got = _pass(x, w, b, up, torch.full((rows,), -100, device=DEV))
        assert got["loss"].shape == (3, rows) and not any(v.any() for v in got.values())


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("low", ["-inf", "lowest"])
def test_words_masked_by_the_bias(kind, low):
    for rows, vocab in ((9, 300), (70, 1000), (400, 20000)):
        x, w, b, up, g = _inputs(kind, rows, 40, vocab, bias=True)
        masked = torch.rand(vocab, device=DEV, generator=g) < 0.5
        masked[:vocab // 3] = True                                  # whole tiles of them
        target = torch.nonzero(~masked).flatten()[torch.randint(int((~masked).sum()), (rows,), device=DEV, generator=g)]
        b[masked] = -math.inf if low == "-inf" else torch.finfo(b.dtype).min
        got = _check(x, w, b, up, target)
        assert not got["dw"][masked].any() and not got["db"][masked].any() and torch.isfinite(got["dw"]).all()
        # the label itself masked: an infinite loss, q = 0 there
        if low == "-inf":
            target[0] = int(torch.nonzero(masked)[0])
            loss = _ops().head_cross_entropy(x, w, target, bias=b)
            assert loss[0] == math.inf and torch.equal(loss[1:], got["loss"][1:])


def test_every_word_masked_is_no_number():
    x, w, b, up, g = _inputs("f32", 50, 16, 200, bias=True)
    got = _pass(x, w, torch.full_like(b, -math.inf), up, torch.zeros(50, dtype=torch.long, device=DEV))
    assert torch.isnan(got["loss"]).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows", [12, 80, 1300])
def test_what_is_no_number_stays_in_its_row(kind, rows):
    x, w, b, up, g = _inputs(kind, rows, 40, 500)
    target = torch.randint(500, (rows,), device=DEV, generator=g)
    clean = _pass(x, w, b, up, target)
    others = torch.ones(rows, dtype=torch.bool, device=DEV)
    others[[2, 5, 7, 11]] = False
    x[2, 3], x[5, 0] = NAN, math.inf
    target[7], target[11] = 500, -3                                 # outside the vocabulary
    got = _pass(x, w, b, up, target)
    for n in ("loss", "dx"):
        assert torch.isnan(got[n][~others]).reshape(4, -1).any(1).all() and torch.equal(got[n][others], clean[n][others])
    index, logit = _lists(g, rows, 500, 6, ragged=False)
    x[2, 3] = x[5, 0] = 0
    clean = _pass(x, w, b, up, (index, logit))
    index[2, 1], logit[5, 2], logit[7, 0], index[11, 5] = 500, NAN, math.inf, 1 << 40
    got = _pass(x, w, b, up, (index, logit))
    for n in ("loss", "dx"):
        assert torch.isnan(got[n][~others]).reshape(4, -1).any(1).all() and torch.equal(got[n][others], clean[n][others])


def test_a_word_that_stands_twice_and_order_do_not_matter():
    x, w, b, up, g = _inputs("f32", 30, 24, 100)
    index = torch.tensor([[7, 3, 7, 99, 0, 3]], device=DEV).repeat(30, 1)
    logit = torch.randn(30, 6, device=DEV, generator=g)
    _check(x, w, b, up, (index, logit), 2.0)
    index, logit = _lists(g, 30, 100, 50, ragged=False)
    first = _check(x, w, b, up, (index, logit))
    order = torch.randperm(50, device=DEV, generator=g)
    again = _pass(x, w, b, up, (index[:, order].contiguous(), logit[:, order].contiguous()))
    assert torch.equal(first["dw"], again["dw"]) and torch.equal(first["dx"], again["dx"])
    for dt in (torch.bfloat16, torch.float16):                      # a teacher in another type than the student
        soft = logit.to(dt)
        a, c = _pass(x, w, b, up, (index, soft)), _pass(x, w, b, up, (index, soft.float()))
        assert all(torch.equal(a[n], c[n]) for n in a)


def test_one_word_a_row_is_the_cross_entropy():
    for kind in ("f32", "bf16"):
        x, w, b, up, g = _inputs(kind, 70, 64, 900, bias=True)
        target = torch.randint(900, (70,), device=DEV, generator=g)
        a = _pass(x, w, b, up, target)
        c = _pass(x, w, b, up, (target[:, None], torch.full((70, 1), 2.5, device=DEV)))
        assert all(torch.equal(a[n], c[n]) for n in a)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_layouts_in_memory(kind):
    x, w, b, up, g = _inputs(kind, 70, 64, 300, bias=True)
    target = torch.randint(300, (70,), device=DEV, generator=g)
    want = _pass(x, w, b, up, target)

    def same(*args, **more):
        got = _pass(*args, **more)
        assert all(torch.equal(got[n], want[n]) for n in want)
    wide = torch.full((300, 100), NAN, device=DEV, dtype=w.dtype)
    wide[:, 3:67] = w
    same(x, wide[:, 3:67], b, up, target)                           # off the 16-byte grid
    wide[:, 8:72] = w
    same(x, wide[:, 8:72], b, up, target)
    wide = torch.full((300, 104), NAN, device=DEV, dtype=w.dtype)   # on it, rows apart: read as they lie
    wide[:, 8:72] = w
    same(x, wide[:, 8:72], b, up, target)
    off = torch.empty(300 * 64 + 1, device=DEV, dtype=w.dtype)[1:].view(300, 64)
    off.copy_(w)
    same(x, off, b, up, target)
    same(x, w.t().contiguous().t(), b, up, target)
    xs = torch.full((70, 90), NAN, device=DEV, dtype=x.dtype)
    xs[:, 1:65] = x
    same(xs[:, 1:65], w, b, up, target)
    same(x.t().contiguous().t(), w, b, up, target)
    same(x, w, torch.stack([b, b], 1)[:, 0], up, target)
    same(x, w, b, torch.stack([up, up], 1)[:, 0], torch.stack([target, target], 1)[:, 1])
    batch = _pass(x.view(2, 5, 7, 64), w, b, up.view(2, 5, 7), target.view(2, 5, 7))
    assert all(torch.equal(batch[n].reshape(want[n].shape), want[n]) for n in want)
    # one gradient for all rows
    leaf = x.detach().requires_grad_()
    _ops().head_cross_entropy(leaf, w, target, bias=b).sum().backward()
    assert torch.equal(leaf.grad, _pass(x, w, b, torch.ones_like(up), target)["dx"])
    index, logit = _lists(g, 70, 300, 6)
    want = _pass(x, w, b, up, (index, logit))
    more = torch.full((70, 20), 5, device=DEV)
    more[:, 4:10] = index
    other = torch.full((70, 20), NAN, device=DEV)
    other[:, 2:8] = logit
    same(x, w, b, up, (more[:, 4:10], other[:, 2:8]))
    same(x, w, b, up, (index.t().contiguous().t(), logit.t().contiguous().t()))


def test_weights_that_are_views_of_a_sampled_vector():
    drawn = torch.randn(3, 5001, device=DEV).mul_(0.2).requires_grad_()
    x = torch.randn(3, 37, 40, device=DEV)
    w, b = drawn[:, 7:4007].view(3, 100, 40), drawn[:, 4007:4107]
    target = torch.randint(100, (37,), device=DEV)
    loss = _ops().head_cross_entropy(x, w, target, bias=b)
    up = torch.rand(3, 37, device=DEV)
    loss.backward(up)
    want = U.head_plain(x, w.detach(), b.detach(), U.labels(target[None], 100), up)
    U.within(loss, *want["loss"], "loss")
    U.within(drawn.grad[:, 7:4007].reshape(3, 100, 40), *want["dw"], "dw")
    U.within(drawn.grad[:, 4007:4107], *want["db"], "db")


def test_only_what_is_asked_for():
    x, w, b, up, g = _inputs("bf16", 50, 32, 200, bias=True)
    target = torch.randint(200, (50,), device=DEV, generator=g)
    full = _pass(x, w, b, up, target)
    for wanted in (("dx",), ("dw",), ("db",), ("dx", "db"), ("dw", "db")):
        leaves = {n: t.detach().requires_grad_(n in wanted) for n, t in zip(("dx", "dw", "db"), (x, w, b))}
        loss = _ops().head_cross_entropy(leaves["dx"], leaves["dw"], target, bias=leaves["db"])
        grads = torch.autograd.grad(loss, [leaves[n] for n in wanted], up)
        assert all(torch.equal(a, full[n]) for a, n in zip(grads, wanted)), wanted
    assert not _ops().head_cross_entropy(x, w, target, bias=b).requires_grad


@pytest.mark.parametrize("scale", [1e-35, 1e-12, 1e12, 0.0])
def test_gradients_of_any_size(scale):
    """dz is held in 16-bit pieces in units of the largest gradient: small and large losses' weights lose nothing."""
    for kind in ("f32", "bf16"):
        x, w, b, up, g = _inputs(kind, 40, 32, 150)
        target = torch.randint(150, (40,), device=DEV, generator=g)
        _check(x, w, b, (up * scale).float(), target)


def test_gradients_against_differences():
    x, w, b, up, g = _inputs("f32", 12, 20, 50, 2, bias=True)
    target = torch.randint(50, (12,), device=DEV, generator=g)
    lists = _lists(g, 12, 50, 6)
    for targets, more in ((target, {}), (lists, {"temperature": 2.0})):
        got = _pass(x, w, b, up, targets, **more)
        for name, i in (("dx", 0), ("dw", 1), ("db", 2)):
            args = [x.double(), w.double(), b.double()]
            way = torch.randn(args[i].shape, device=DEV, generator=g, dtype=torch.float64)
            step = 2.0 ** -8

            def loss(sign):
                moved = [(t + sign * step * way if j == i else t).float() for j, t in enumerate(args)]
                return float((_pass(*moved, up, targets, **more)["loss"].double() * up).sum())
            slope = (loss(1) - loss(-1)) / (2 * step)
            # losses of up to 16, good for 2^-20 of that; third differences of a logit moved by a few sigma of sqrt(K): below 1000 a row
            size = float(up.sum())
            assert abs(slope - float((got[name].double() * way).sum())) <= size * (16 * 2.0 ** -20 / step + 1000 / 6 * step * step), name


def test_differentiable_once():
    x, w, b, up, g = _inputs("f32", 8, 16, 30)
    target = torch.zeros(8, dtype=torch.long, device=DEV)
    for weight in (w, w.t().contiguous().t()):
        leaf = x.detach().requires_grad_()
        (dx,) = torch.autograd.grad(_ops().head_cross_entropy(leaf, weight, target).square().sum(), leaf, create_graph=True)
        with pytest.raises(RuntimeError):
            dx.sum().backward()


def test_another_stream_and_replays_of_a_graph():
    x, w, b, up, g = _inputs("bf16", 200, 96, 3000, bias=True)
    target = torch.randint(3000, (200,), device=DEV, generator=g)
    want = _pass(x, w, b, up, target)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _pass(x, w, b, up, target)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(got[n], want[n]) for n in want)

    from paper_2604_04736_amd import binding as hot
    for rows in (200, 1100):
        x, w, b, up, g = _inputs("bf16", rows, 96, 3000, bias=True)
        target = torch.randint(3000, (rows,), device=DEV, generator=g)
        args = [x[None].clone(), w[None], b[None], target[None].clone()]
        loss, lse = torch.empty(1, rows, device=DEV), torch.empty(1, rows, device=DEV, dtype=torch.float64)
        dx, dw, db = torch.empty_like(args[0]), torch.empty_like(args[1]), torch.empty_like(args[2])
        ws = [torch.empty(hot.hot_head_workspace_bytes(*args, which=k), dtype=torch.uint8, device=DEV) for k in (0, 1)]

        def step():
            hot.hot_head_forward(*args, None, loss, lse, workspace=ws[0])
            hot.hot_head_backward(*args, None, lse, up[None], dx, dw, db, workspace=ws[1])
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for seed in range(3):
            xs = torch.randn(x.shape, device=DEV, generator=g).to(x.dtype)
            ts = torch.randint(3000, (rows,), device=DEV, generator=g)
            ts[torch.rand(rows, device=DEV, generator=g) < 0.3 * seed] = -100
            args[0].copy_(xs[None])
            args[3].copy_(ts[None])
            for t in ws:
                t.fill_(255)                                        # (scratch that holds nan)
            graph.replay()
            torch.cuda.synchronize()
            want = _pass(xs, w, b, up, ts)
            for n, v in (("loss", loss[0]), ("dx", dx[0]), ("dw", dw[0]), ("db", db[0])):
                assert torch.equal(v, want[n]), (n, seed)


def test_offsets_beyond_32_bits():
    vocab, width = 70000, 32768                                     # weights of 4.6 GB
    w = torch.empty(vocab, width, dtype=torch.bfloat16, device=DEV)
    w[:, :] = (torch.randn(1, width, device=DEV) / 200).to(w.dtype)
    w[-5:] = (torch.randn(5, width, device=DEV) / 100).to(w.dtype)
    for rows in (2, 40):
        x = torch.randn(rows, width, device=DEV).to(w.dtype)
        target = torch.full((rows,), vocab - 2, device=DEV)
        up = torch.ones(rows, device=DEV)
        got = _pass(x, w, None, up, target)
        few = torch.cat([w[:1], w[-5:]]).double()
        z = x.double() @ few.T
        weights = torch.tensor([vocab - 5] + [1] * 5, device=DEV, dtype=torch.float64)
        lse = torch.logsumexp(z + weights.log(), 1)
        dz = torch.exp(z - lse[:, None])
        dz[:, 4] -= 1
        off = (width / 16 + 24) * U.U32 * (x.double().abs() @ few.abs().T).amax()
        U.within(got["loss"], lse - z[:, 4], (2 * off + 2 ** -18).expand(rows), "loss")
        ref = dz.T @ x.double()
        bound = (dz.abs() * 2.0 ** -8 + torch.exp(z - lse[:, None]) * (5 * off + 2 ** -18)).T @ x.double().abs() + U.rounded(ref, w.dtype)
        U.within(torch.cat([got["dw"][:1], got["dw"][-5:]]), ref, bound, "dw")
        ref = (dz * weights) @ few
        bound = (dz.abs() * 2.0 ** -8 + torch.exp(z - lse[:, None]) * (5 * off + 2 ** -17)) * weights @ few.abs() + U.rounded(ref, w.dtype)
        U.within(got["dx"], ref, bound, "dx")
        del got


def test_many_rows_of_wide_features():
    rows, width = 70000, 32768                                      # features of 4.6 GB
    x = torch.empty(rows, width, dtype=torch.bfloat16, device=DEV)
    x[:, :] = torch.randn(1, width, device=DEV).to(x.dtype)
    x[-3:] = torch.randn(3, width, device=DEV).to(x.dtype)
    w = (torch.randn(7, width, device=DEV) / 100).to(x.dtype)
    target = torch.full((rows,), -100, device=DEV)
    target[-3:] = torch.tensor([1, 6, 3], device=DEV)
    target[0] = 2
    up = torch.ones(rows, device=DEV)
    got = _pass(x, w, None, up, target)
    seen = torch.tensor([0, rows - 3, rows - 2, rows - 1], device=DEV)
    want = U.head_plain(x[seen][None], w[None], None, U.labels(target[seen][None], 7), up[seen][None])
    for n in ("loss", "dx"):
        U.within(got[n][seen], want[n][0][0], want[n][1][0] + (2.0 ** -8 * want[n][0][0].abs().amax() if n == "dx" else 0), n)
    assert not got["dx"][1:-3].any() and not got["loss"][1:-3].any()


def test_refusals():
    ce, kd = _ops().head_cross_entropy, _ops().head_distillation
    x, w = torch.randn(4, 6, device=DEV), torch.randn(9, 6, device=DEV)
    t = torch.zeros(4, dtype=torch.long, device=DEV)
    i, s = torch.zeros(4, 2, dtype=torch.long, device=DEV), torch.zeros(4, 2, device=DEV)
    for bad in (lambda: ce(x.double(), w.double(), t), lambda: ce(x, w.bfloat16(), t), lambda: ce(x, w, t.int()), lambda: ce(x, w, t.cpu()), lambda: ce(x, w.cpu(), t), lambda: ce(x.cpu(), w, t),
                lambda: ce(x, w, t, bias=torch.zeros(9, device=DEV, dtype=torch.bfloat16)), lambda: kd(x, w, i, s.double())):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: ce(x, w[:, :5], t), lambda: ce(x, w[0], t), lambda: ce(x, w, t[:3]), lambda: ce(x, w, t, bias=torch.zeros(8, device=DEV)), lambda: kd(x, w, i, s[:, :1]),
                lambda: kd(x, w, i[:, :0], s[:, :0]), lambda: kd(x, w, i[:3], s[:3]), lambda: ce(x.expand(3, 4, 6), w.expand(2, 9, 6), t),
                lambda: kd(x, w, torch.zeros(4, 1025, dtype=torch.long, device=DEV), torch.zeros(4, 1025, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    for temperature in (0.0, -1.0, NAN, math.inf):
        with pytest.raises(RuntimeError):
            kd(x, w, i, s, temperature=temperature)
    with pytest.raises(RuntimeError):                               # one set of weights twice: each sample has its own
        ce(x, w.expand(2, 9, 6), t)
