"""Plain forms of the layer norm and of the head's losses in 64 bits, and how far float32 or 16-bit results may be from them: each bound adds up the
roundings that a result goes through, from the sizes of the terms that are rounded."""
import math

import torch

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# half a unit in the last place of a number with 24, 8 or 11 significant bits, and half the smallest step near zero
HALF_UNIT = {dtype: torch.finfo(dtype).eps / 2 for dtype in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
U32 = 2.0 ** -24


def within(got, want, bound, name):
    """got (any type) against want (64 bits), element by element; nan and infinities have to be in the same places."""
    got = got.detach().double()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), name + ": nan elsewhere"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), name
    off = ((got - want).abs() - bound)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, (name, float(off.max()), float((got - want).abs()[fine].max()))


def rounded(want, dtype):
    return 1.01 * HALF_UNIT[dtype] * want.abs() + TINY[dtype]


# ------------------------------------------------------------------ layer norm: x [S, R, D], w and b [S, D] or [D]

def norm_plain(x, w, b, eps, dy):
    """y, dx, dw, db in 64 bits and the bounds of a float32 computation rounded to the types at the end."""
    xd, wd = x.double(), (w.double() if w is not None else torch.ones(x.shape[-1], dtype=torch.float64, device=x.device)).unsqueeze(-2)
    bd = (b.double() if b is not None else torch.zeros(x.shape[-1], dtype=torch.float64, device=x.device)).unsqueeze(-2)
    n, rows = x.shape[-1], x.shape[-2]
    mean = xd.mean(-1, keepdim=True)
    r = ((xd - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    h = (xd - mean) * r
    y = h * wd + bd
    # a thread adds up to n / 1024 + 16 elements, ten more additions join the threads: relative to the mean size of what is added
    adds = (n / 1024 + 32) * U32
    h_off = adds * r * xd.abs().mean(-1, keepdim=True) + (adds + 8 * U32) * h.abs() + 4 * U32 * r * xd.abs()
    out = {"y": (y, rounded(y, x.dtype) + 1.01 * (h_off * wd.abs() + 4 * U32 * (bd.abs() + (h * wd).abs())))}
    d = dy.double()
    u = d * wd
    c1, c2 = u.mean(-1, keepdim=True), (u * h).mean(-1, keepdim=True)
    dx = r * (u - c1 - h * c2)
    size1, size2 = u.abs().mean(-1, keepdim=True), (u * h).abs().mean(-1, keepdim=True)
    c2_off = (adds + 4 * U32) * size2 + (u.abs() * h_off).mean(-1, keepdim=True)
    dx_off = r * ((8 * U32) * (u.abs() + size1 + (h * c2).abs()) + adds * size1 + h.abs() * c2_off + h_off * c2.abs()) + (adds + 8 * U32) * dx.abs()
    out["dx"] = (dx, rounded(dx, x.dtype) + 1.01 * dx_off)
    wt = w.dtype if w is not None else x.dtype
    # rows over up to 1024 workgroups: no chain of additions is longer than rows / 16 + 64
    chain = (min(rows * x.shape[0], rows / 16 + 96) + 8) * U32
    dw, db = (d * h).sum(-2), d.sum(-2)
    dw_off = chain * (d * h).abs().sum(-2) + (d.abs() * h_off).sum(-2)
    db_off = chain * d.abs().sum(-2)
    shaped = w if w is not None else b
    if shaped is None or shaped.dim() == 1:
        dw, db, dw_off, db_off = dw.sum(0), db.sum(0), dw_off.sum(0), db_off.sum(0)
    out["dw"] = (dw, rounded(dw, wt) + 1.01 * dw_off)
    out["db"] = (db, rounded(db, wt) + 1.01 * db_off)
    return out


# ------------------------------------------------------------------ head: x [S, R, K] or [1, R, K], w [S, V, K], b [S, V] or None

def teacher(index, logit, temperature, vocab):
    """(p spread over the vocabulary, sum p ln p, which rows count) of a teacher's lists, 64 bits."""
    there = (index >= 0) & ~torch.isneginf(logit.double())
    t = torch.where(there, logit.double() / temperature, -math.inf)
    counts = there.any(-1)
    p = torch.where(counts.unsqueeze(-1), torch.softmax(t, -1), torch.zeros_like(t))
    spread = torch.zeros(*index.shape[:-1], vocab, dtype=torch.float64, device=index.device)
    spread.scatter_add_(-1, index.clamp(min=0), torch.where(there, p, torch.zeros_like(p)))
    return spread, -torch.special.entr(p).sum(-1), counts


def labels(target, vocab, ignore_index=-100):
    counts = target != ignore_index
    spread = torch.zeros(*target.shape, vocab, dtype=torch.float64, device=target.device)
    spread.scatter_(-1, target.clamp(min=0).unsqueeze(-1), counts.double().unsqueeze(-1))
    return spread, torch.zeros(target.shape, dtype=torch.float64, device=target.device), counts


def head_plain(x, w, b, teach, g, temperature=1.0):
    """loss, dx, dw, db in 64 bits and their bounds; teach: (p spread, sum p ln p, counts)."""
    p, p_log_p, counts = teach
    kind, t = x.dtype, temperature
    u = HALF_UNIT[kind]
    xd, wd = x.double(), w.double()
    n, rows, width = w.shape[0], x.shape[1], x.shape[2]
    keep = counts.expand(n, rows)
    xs = torch.where(keep.unsqueeze(-1), xd.expand(n, rows, width), 0.0)
    z = xs @ wd.transpose(1, 2)
    size = xs.abs() @ wd.abs().transpose(1, 2)
    if b is not None:
        z = z + b.double().unsqueeze(1)
        size = size + torch.nan_to_num(b.double().abs(), posinf=0.0).unsqueeze(1)
    # a logit: K / 16 additions of the matrix instruction (each itself a sum of sixteen), three pieces of float32 good for 2^-22 of a product
    z_off = (width / 16 + 24) * U32 * size
    lse = torch.logsumexp(z / t, -1, keepdim=True)
    q = torch.exp(z / t - lse)
    zero_safe = torch.where(p > 0, z, torch.zeros_like(z))
    loss = t * t * (p_log_p + torch.where(keep, lse.squeeze(-1), 0.0) - (p * zero_safe).sum(-1) / t)
    loss = torch.where(keep, loss, torch.zeros_like(loss))
    most_off = torch.where(torch.isfinite(z), z_off, torch.zeros_like(z_off)).amax(-1)
    finite_lse = torch.nan_to_num(lse.squeeze(-1), nan=0.0, posinf=0.0, neginf=0.0)
    loss_off = t * t * (2 * most_off / t + 24 * U32 * (finite_lse.abs() + p_log_p.abs() + (p * zero_safe).abs().sum(-1) / t + 4))
    out = {"loss": (loss, U32 * torch.nan_to_num(loss).abs() + loss_off)}
    if g is None:
        return out
    gk = torch.where(keep, g.double(), 0.0).unsqueeze(-1) * t
    few = rows <= 32 and kind != torch.float32
    dz = gk * (q - p)
    q_off = q * (3 * z_off / t + 2 * most_off.unsqueeze(-1) / t + 16 * U32 * (torch.nan_to_num((z / t).abs(), posinf=0.0) + finite_lse.abs().unsqueeze(-1) + 4))
    held = 2 * U32 if kind == torch.float32 else (4 * u * u + 2 * U32 if few else 1.01 * u)
    biggest = gk.abs().amax()
    dz_off = gk.abs() * (torch.nan_to_num(q_off) + 4 * U32 * (q + p)) + held * dz.abs() + (biggest * 2.0 ** -36 if kind == torch.float16 else 0.0)
    dx = dz @ wd
    dx_off = dz_off @ wd.abs() + (w.shape[1] / 16 + 96) * U32 * (dz.abs() @ wd.abs())
    if x.shape[0] == 1 and n > 1:
        dx, dx_off = dx.sum(0, keepdim=True), dx_off.sum(0, keepdim=True)
    dw = dz.transpose(1, 2) @ xs
    dw_off = dz_off.transpose(1, 2) @ xs.abs() + (rows / 16 + 32) * U32 * (dz.abs().transpose(1, 2) @ xs.abs())
    db, db_off = dz.sum(1), dz_off.sum(1) + (rows / 16 + 64) * U32 * dz.abs().sum(1)
    for name, v, off in (("dx", dx, dx_off), ("dw", dw, dw_off), ("db", db, db_off)):
        out[name] = (v, rounded(v, kind) + 1.01 * off)
    return out
