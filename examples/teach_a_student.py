"""From an ensemble to one network, on one GPU: a Bayesian head learns labels, then teaches a deterministic student.

The network is a norm and a head over a vocabulary.  The Bayesian one keeps mu and sigma of every weight; each step draws S weight
samples with the sample layer (their norms and heads are views of the drawn rows), runs layer norm and the head's cross entropy
on all samples at once, and back-propagates into mu and sigma, KL included.  The student learns the ensemble's likeliest words
(the mean of the samples' predictions, its top logits) through the distillation loss, and then answers a single row.

    python examples/teach_a_student.py [--steps 60] [--device cuda:0]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2604_04736_amd.autograd import GaussianSampleLayer, head_cross_entropy, head_distillation, layer_norm  # noqa: E402


def task(rows, width, vocab, device, seed):
    """Features whose word is the nearest of `vocab` directions; one row in eight has no label."""
    g = torch.Generator(device=device).manual_seed(seed)
    directions = torch.randn(vocab, width, device=device, generator=torch.Generator(device=device).manual_seed(0))
    word = torch.randint(vocab, (rows,), device=device, generator=g)
    x = directions[word] + 1.5 * torch.randn(rows, width, device=device, generator=g)
    label = torch.where(torch.rand(rows, device=device, generator=g) < 0.125, -100, word)
    return x, word, label


def slices(width, vocab):
    """Where norm weight, norm bias, head and head bias lie in the flat vector of weights."""
    sizes = [("norm_w", (width,)), ("norm_b", (width,)), ("head", (vocab, width)), ("head_b", (vocab,))]
    at, out = 0, {}
    for name, shape in sizes:
        n = torch.Size(shape).numel()
        out[name] = (at, at + n, shape)
        at += n
    return out, at


def views(w, where):
    return {name: w[..., a:b].unflatten(-1, shape) for name, (a, b, shape) in where.items()}


def main(steps=60, device="cuda:0", samples=4, rows=512, width=64, vocab=500, top=16, temperature=2.0):
    device = torch.device(device)
    where, n = slices(width, vocab)
    x, word, label = task(rows, width, vocab, device, 1)
    labelled = (label != -100).sum()

    # the Bayesian network
    start = torch.zeros(n, device=device)
    start[slice(*where["norm_w"][:2])] = 1.0
    start[slice(*where["head"][:2])] = 0.02 * torch.randn(vocab * width, device=device, generator=torch.Generator(device=device).manual_seed(2))
    mu, sigma = start.clone().requires_grad_(), torch.full((n,), 0.01, device=device, requires_grad=True)
    layer = GaussianSampleLayer(n, samples, dataset_size=45000.0, device=device.index or 0)
    optimizer = torch.optim.Adam([mu, sigma], lr=0.01)
    first = last = None
    for step in range(steps):
        drawn, kl = layer.sample(mu, sigma, step)                         # [samples, n]
        v = views(drawn, where)
        h = layer_norm(x.expand(samples, -1, -1), v["norm_w"], v["norm_b"])
        loss = head_cross_entropy(h, v["head"], label, bias=v["head_b"]).sum() / (samples * labelled)
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        with torch.no_grad():
            sigma.clamp_(min=1e-4)
        first, last = loss.item() if first is None else first, loss.item()

    # its likeliest words, and the student that learns them
    with torch.no_grad():
        v = views(layer.sample(mu, sigma, steps)[0], where)
        h = layer_norm(x.expand(samples, -1, -1), v["norm_w"], v["norm_b"])
        ensemble = (torch.baddbmm(v["head_b"].unsqueeze(1), h, v["head"].transpose(1, 2).contiguous())).softmax(-1).mean(0)
        logit, index = ensemble.log().topk(top, dim=-1)
    student = {name: t.clone().requires_grad_() for name, t in views(start, where).items()}
    optimizer = torch.optim.Adam(student.values(), lr=0.01)
    first_taught = last_taught = None
    for step in range(steps):
        h = layer_norm(x, student["norm_w"], student["norm_b"])
        loss = head_distillation(h, student["head"], index, logit, bias=student["head_b"], temperature=temperature).mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        first_taught, last_taught = loss.item() if first_taught is None else first_taught, loss.item()

    # one new row: how probable the student finds its word
    with torch.no_grad():
        one, its_word, _ = task(1, width, vocab, device, 3)
        surprise = head_cross_entropy(layer_norm(one, student["norm_w"], student["norm_b"]), student["head"], its_word, bias=student["head_b"]).item()
        agree = ((layer_norm(x, student["norm_w"], student["norm_b"]) @ student["head"].T + student["head_b"]).argmax(-1) == ensemble.argmax(-1)).float().mean().item()
    print(f"ensemble: loss {first:.3f} -> {last:.3f} over {steps} steps, KL {kl.item():.0f}")
    print(f"student: divergence {first_taught:.3f} -> {last_taught:.3f}, its likeliest word is the ensemble's on {100 * agree:.0f} % of the rows")
    print(f"a new row: its word has probability {torch.tensor(-surprise).exp():.3f} (uniform: {1 / vocab:.3f})")
    return {"ensemble": (first, last), "student": (first_taught, last_taught), "agree": agree, "surprise": surprise}


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--device", default="cuda:0")
    a = ap.parse_args()
    main(a.steps, a.device)
