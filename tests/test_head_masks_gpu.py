"""The head's losses where logits are masked with the lowest value of their type, and where all of them lie far from zero."""
import math

import pytest
import torch

import head_norm_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _ops():
    from paper_2604_04736_amd import autograd
    return autograd


def _pass(x, w, b, up, targets, temperature=1.0):
    leaves = [t.detach().requires_grad_() for t in (x, w, b)]
    if isinstance(targets, tuple):
        loss = _ops().head_distillation(leaves[0], leaves[1], *targets, bias=leaves[2], temperature=temperature)
    else:
        loss = _ops().head_cross_entropy(leaves[0], leaves[1], targets, bias=leaves[2])
    return dict(zip(("loss", "dx", "dw", "db"), (loss.detach(), *torch.autograd.grad(loss, leaves, up))))


def _inputs(kind, rows, width, vocab):
    g = torch.Generator(device=DEV).manual_seed(rows + vocab)
    dt = U.TYPES[kind]
    x = torch.randn(rows, width, device=DEV, generator=g).to(dt)
    w = (torch.randn(vocab, width, device=DEV, generator=g) * (2 / math.sqrt(width))).to(dt)
    return x, w, torch.randn(vocab, device=DEV, generator=g).to(dt), torch.rand(rows, device=DEV, generator=g) + 0.5, g


SIZES = [(9, 300), (20, 40000), (70, 1000), (400, 20000)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_a_label_masked_with_the_lowest_value(kind, rows, vocab):
    """A finite loss, that word's distance, and the gradients that a bias of -inf gives; the other rows as before."""
    x, w, b, up, g = _inputs(kind, rows, 40, vocab)
    masked = torch.rand(vocab, device=DEV, generator=g) < 0.5
    masked[:vocab // 3] = True
    target = torch.nonzero(~masked).flatten()[torch.randint(int((~masked).sum()), (rows,), device=DEV, generator=g)]
    hit = torch.arange(rows, device=DEV) % 3 == 0
    target[hit] = torch.nonzero(masked).flatten()[torch.randint(int(masked.sum()), (int(hit.sum()),), device=DEV, generator=g)]
    lowest = torch.finfo(b.dtype).min
    far, gone = (_pass(x, w, b.masked_fill(masked, value), up, target) for value in (lowest, -math.inf))
    assert all(torch.equal(far[n], gone[n]) for n in ("dx", "dw", "db"))
    assert torch.equal(far["loss"][~hit], gone["loss"][~hit]) and (gone["loss"][hit] == math.inf).all()
    # z of the label and the largest logit: below 2^6 each; float32 logits of that size, and a loss rounded once
    bound = 4 * U.U32 * -lowest + 2 ** 7 + (40 / 16 + 24) * U.U32 * -lowest * (kind == "f16")
    U.within(far["loss"][hit], torch.full((int(hit.sum()),), -float(lowest), dtype=torch.float64, device=DEV), bound, "loss")
    # a teacher's words, some of them masked
    index = target[:, None].repeat(1, 3)
    index[:, 1] = int(torch.nonzero(~masked)[1])
    index[:, 2] = int(torch.nonzero(masked)[2])
    logit = torch.tensor([[1.0, 0.5, -1.0]], device=DEV).repeat(rows, 1)
    far, gone = (_pass(x, w, b.masked_fill(masked, value), up, (index, logit)) for value in (lowest, -math.inf))
    assert all(torch.equal(far[n], gone[n]) for n in ("dx", "dw", "db"))
    p = torch.softmax(logit[0].double(), 0)
    share = torch.where(hit, p[0] + p[2], p[2])
    U.within(far["loss"], -lowest * share, bound * share + 32 * U.U32 * -lowest + 2 ** 8, "a teacher's words")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("lists", [False, True])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_every_word_masked_with_the_lowest_value(kind, lists, rows, vocab):
    """z = x . w + lowest is the lowest value itself: all words are as likely."""
    temperature = 2.0 if lists else 1.0
    x, w, b, up, g = _inputs(kind, rows, 40, vocab)
    if lists:
        targets = (torch.randint(vocab, (rows, 4), device=DEV, generator=g), torch.randn(rows, 4, device=DEV, generator=g))
        p, p_log_p, _ = U.teacher(*targets, temperature, vocab)
    else:
        targets = torch.randint(vocab, (rows,), device=DEV, generator=g)
        p, p_log_p, _ = U.labels(targets, vocab)
    _same_distance(x, w, torch.full_like(b, torch.finfo(b.dtype).min), up, targets, p, p_log_p, temperature, torch.zeros(vocab, dtype=torch.float64, device=DEV))


def _same_distance(x, w, b, up, targets, p, p_log_p, temperature, z):
    """Results where all rows' logits are z - max z, a float's exact differences [vocab] (64 bits), against 64 bits."""
    got = _pass(x, w, b, up, targets, temperature)
    log_q = torch.log_softmax(z / temperature, 0)
    q, t2 = log_q.exp(), temperature ** 2
    terms = torch.where(p > 0, p * log_q, torch.zeros_like(p))
    loss = t2 * (p_log_p - terms.sum(1))
    distance = torch.where(p > 0, p * (z.max() - z) / temperature, torch.zeros_like(p)).sum(1)
    off = t2 * 24 * U.U32 * (math.log(len(z)) + p_log_p.abs() + distance + 4)
    U.within(got["loss"], loss, off + U.U32 * loss.abs(), "loss")
    u, f32 = U.HALF_UNIT[x.dtype], x.dtype == torch.float32
    gt = (up.double() * temperature)[:, None]
    dz = gt * (q - p)
    held = 2 * U.U32 if f32 else 4 * u * u + 2 * U.U32
    dz_off = gt * (16 * U.U32 * q * ((z.max() - z) / temperature + math.log(len(z)) + 4) + 4 * U.U32 * (q + p)) + held * dz.abs() + 2.0 ** -125 * float(gt.max())     # (probabilities and pieces below the normal numbers are zero)
    dx, dw, db = dz @ w.double(), dz.T @ x.double(), dz.sum(0)
    rows, vocab = p.shape
    chain = (vocab / 16 + 96) * U.U32
    U.within(got["dx"], dx, U.rounded(dx, x.dtype) + 1.01 * (dz_off + chain * dz.abs()) @ w.double().abs(), "dx")
    chain = (rows / 16 + 64) * U.U32
    U.within(got["dw"], dw, U.rounded(dw, x.dtype) + 1.01 * (dz_off + chain * dz.abs()).T @ x.double().abs(), "dw")
    U.within(got["db"], db, U.rounded(db, x.dtype) + 1.01 * (dz_off + chain * dz.abs()).sum(0), "db")


@pytest.mark.parametrize("offset", [0.0, 1e3, -1e5, 2.0 ** 22, 1.9 * 2.0 ** 26, -2.0 ** 27, 2.0 ** 33, 1e30, -1e38])
@pytest.mark.parametrize("temperature", [1.0, 0.25, 64.0, 4096.0])
@pytest.mark.parametrize("rows,vocab", [(9, 300), (70, 3000)])
def test_logits_far_from_zero(offset, temperature, rows, vocab):
    """x = 0, so z is the bias to the last bit: what counts are its distances, a few of the steps of float32 at that offset."""
    x, w, _, up, g = _inputs("f32", rows, 24, vocab)
    x.zero_()
    step = max(math.ulp(abs(offset)) * 2 ** 29, 2.0 ** -6)
    z = torch.randint(0, 8, (vocab,), device=DEV, generator=g).double() * step
    b = (offset + z).float()
    assert torch.equal(b.double() - b.double().max(), z - z.max())
    targets = (torch.randint(vocab, (rows, 5), device=DEV, generator=g), torch.randn(rows, 5, device=DEV, generator=g) * temperature)
    p, p_log_p, _ = U.teacher(*targets, temperature, vocab)
    _same_distance(x, w, b, up, targets, p, p_log_p, temperature, z - z.max())
    if temperature == 1.0:
        target = targets[0][:, 0]
        p, p_log_p, _ = U.labels(target, vocab)
        _same_distance(x, w, b, up, target, p, p_log_p, 1.0, z - z.max())


@pytest.mark.parametrize("offset", [0.0, -1e5, 2.0 ** 22, -2.0 ** 33, 1e30, "lowest"])
@pytest.mark.parametrize("temperature", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("rows,vocab,top", [(9, 300, 3), (70, 3000, 90)])
def test_a_teachers_logits_far_from_zero(offset, temperature, rows, vocab, top):
    """Only a teacher's distances count; words that all have the lowest value are as likely as each other."""
    x, w, b, up, g = _inputs("f32", rows, 24, vocab)
    index = torch.randint(vocab, (rows, top), device=DEV, generator=g)
    if offset == "lowest":
        logit, distance = torch.full((rows, top), torch.finfo(torch.float32).min, device=DEV), torch.zeros(rows, top, device=DEV, dtype=torch.float64)
    else:
        step = max(math.ulp(abs(offset)) * 2 ** 29, 2.0 ** -6)
        distance = torch.randint(0, 8, (rows, top), device=DEV, generator=g).double() * step
        logit = (offset + distance).float()
        assert torch.equal(logit.double() - logit.double().max(), distance - distance.max())
    got = _pass(x, w, b, up, (index, logit), temperature)
    distance -= distance.amax(1, keepdim=True)
    want = U.head_plain(x[None], w[None], b[None], U.teacher(index[None], distance[None], temperature, vocab), up[None], temperature)
    for n in got:
        ref, bound = (t[0] for t in want[n])
        U.within(got[n], ref, bound, n)
