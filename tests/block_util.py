"""Plain forms of dropout, of a block's end and of attention with a position bias in 64 bits, and how far float32 or 16-bit results may be from them: each
bound adds up the roundings that a result goes through, from the sizes of the terms that are rounded."""
import math

import torch

from head_norm_util import DEV, HALF_UNIT, TINY, TYPES, U32, rounded, within  # noqa: F401

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85


def _products(a, b):
    p = a * b                      # (int64 wraps, its bits are the product's)
    return (p >> 32) & 0xFFFFFFFF, p & 0xFFFFFFFF


def kept(rows, width, keep, seed, step=0, first_sample=0, samples=1, offset=0, device=DEV):
    """([samples, rows, width] of which elements stay, the number that those are multiplied by), from the generator's published definition."""
    octets = -(-width // 8)
    i = offset + torch.arange(rows * octets, device=device)[None]
    c0, c1 = i & 0xFFFFFFFF, (i >> 32) | 0x80000000
    c2 = (first_sample + torch.arange(samples, device=device)[:, None]).expand(samples, i.shape[1])
    c3 = torch.full_like(c2, step)
    c0, c1 = c0.expand_as(c2), c1.expand_as(c2)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        (h0, l0), (h1, l1) = _products(c0, M0), _products(c2, M1)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + W0) & 0xFFFFFFFF, (k1 + W1) & 0xFFFFFFFF
    halves = torch.stack([c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16], -1)
    most = max(1, round(65536 * keep))
    return (halves < most).reshape(samples, rows, octets * 8)[..., :width], 65536 / most


# ------------------------------------------------------------------ a block's end: x and branch [S, R, D], vectors [D] or [S, D]

def _vector(v, like, without):
    return (v.double() if v is not None else torch.full((like.shape[-1],), without, dtype=torch.float64, device=like.device)).unsqueeze(-2)


def _norm(v, v_off, kind, w, b, eps):
    """(normalised rows, r, their bounds) of a norm of v, whose elements are v_off off."""
    n = v.shape[-1]
    adds = (n / 1024 + 32) * U32                       # a thread adds up to sixteen elements, ten more additions join the threads
    mean = v.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(v[..., :1])
    mean_off = v_off.mean(-1, keepdim=True) + adds * v.abs().mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(mean)
    c = v - mean
    c_off = v_off + mean_off + 2 * U32 * (v.abs() + mean.abs())
    square = c.square().mean(-1, keepdim=True)
    square_off = (2 * c.abs() * c_off + c_off.square()).mean(-1, keepdim=True) + adds * square
    r = (square + eps).rsqrt()
    r_off = r * (square_off / (square + eps) + 4 * U32)
    h = c * r
    return h, r, c_off * r + c.abs() * r_off + 2 * U32 * h.abs(), r_off


def _norm_back(u, u_off, h, h_off, r, r_off, kind):
    n = u.shape[-1]
    adds = (n / 1024 + 32) * U32
    c2, size2 = (u * h).mean(-1, keepdim=True), (u * h).abs().mean(-1, keepdim=True)
    c2_off = (u_off * h.abs() + u.abs() * h_off).mean(-1, keepdim=True) + adds * size2
    c1 = u.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(c2)
    c1_off = u_off.mean(-1, keepdim=True) + adds * u.abs().mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(c2)
    inner = u - c1 - h * c2
    off = u_off + c1_off + h_off * c2.abs() + h.abs() * c2_off + 4 * U32 * (u.abs() + c1.abs() + (h * c2).abs())
    return r * inner, r * off + r_off * inner.abs() + 2 * U32 * (r * inner).abs()


def block_plain(x, branch, dh, dy, norm, branch_norm=None, weight=None, bias=None, gate=None, branch_weight=None, branch_bias=None, scale=1.0, mask=None, up=1.0, eps=1e-5):
    """{name: (value, bound)} of h, y and the gradients of all tensors that are there; dh or dy None: zeros."""
    kind = x.dtype
    xd, t = x.double(), branch.double()
    t_off = torch.zeros_like(t)
    if branch_norm:
        bn, br, bn_off, br_off = _norm(t, t_off, branch_norm, None, None, eps)
        bw, bb = _vector(branch_weight, x, 1.0), _vector(branch_bias, x, 0.0)
        t, t_off = bn * bw + bb, bn_off * bw.abs() + 2 * U32 * ((bn * bw).abs() + bb.abs())
    if mask is not None:
        zero = torch.zeros_like(t)
        t, t_off = torch.where(mask, t * up, zero), torch.where(mask, t_off * up + 2 * U32 * (t * up).abs(), zero)
    g = scale * _vector(gate, x, 1.0)
    h = xd + g * t
    h_off = g.abs() * t_off + 3 * U32 * (g * t).abs() + 2 * U32 * h.abs()
    out = {"h": (h, rounded(h, kind) + 1.01 * h_off)}
    du = torch.zeros_like(h) if dh is None else dh.double()
    du_off = torch.zeros_like(du)
    chain = (min(h[..., 0].numel(), h[..., 0].numel() / 16 + 128) + 8) * U32          # rows over up to 1024 workgroups
    if norm:
        n, r, n_off, r_off = _norm(h, h_off, norm, None, None, eps)
        w, b = _vector(weight, x, 1.0), _vector(bias, x, 0.0)
        y = n * w + b
        out["y"] = (y, rounded(y, kind) + 1.01 * (n_off * w.abs() + 2 * U32 * ((n * w).abs() + b.abs())))
        d = torch.zeros_like(h) if dy is None else dy.double()
        _sum(out, "weight", weight, d * n, d.abs() * n_off, chain)
        _sum(out, "bias", bias, d, torch.zeros_like(d), chain)
        back, back_off = _norm_back(d * w, U32 * (d * w).abs(), n, n_off, r, r_off, norm)
        du = du + back
        du_off = back_off + 2 * U32 * du.abs()
    out["dx"] = (du, rounded(du, kind) + 1.01 * du_off)
    _sum(out, "gate", gate, scale * du * t, abs(scale) * (du_off * t.abs() + du.abs() * t_off) + 3 * U32 * (scale * du * t).abs(), chain)
    dt, dt_off = du * g, du_off * g.abs() + 3 * U32 * (du * g).abs()
    if mask is not None:
        dt, dt_off = torch.where(mask, dt * up, torch.zeros_like(dt)), torch.where(mask, dt_off * up + 2 * U32 * (dt * up).abs(), torch.zeros_like(dt))
    if branch_norm:
        _sum(out, "branch_weight", branch_weight, dt * bn, dt_off * bn.abs() + dt.abs() * bn_off, chain)
        _sum(out, "branch_bias", branch_bias, dt, dt_off, chain)
        dt, dt_off = _norm_back(dt * bw, dt_off * bw.abs() + U32 * (dt * bw).abs(), bn, bn_off, br, br_off, branch_norm)
    out["dbranch"] = (dt, rounded(dt, kind) + 1.01 * dt_off)
    return out


def _sum(out, name, vector, terms, off, chain):
    if vector is None:
        return
    total, total_off = terms.sum(-2), off.sum(-2) + chain * terms.abs().sum(-2)
    if vector.dim() == 1:
        total, total_off = total.sum(0), total_off.sum(0)
    out["d" + name] = (total, rounded(total, vector.dtype) + 1.01 * total_off)


# ------------------------------------------------------------------ attention: q [B, H, Nq, d], k and v [B, G, Nk, d], table [T, buckets, H]

def attention_plain(q, k, v, do=None, table=None, which=None, scale=None, causal=False, query_groups=None, key_groups=None):
    """{name: (value, bound)} of o and, with do, of the gradients; which: the bucket of every pair [Nq, Nk].  Rows that are of no group count as zeros, whatever they hold."""
    kind = q.dtype
    batch, heads, nq, width = q.shape
    kv, nk = k.shape[1], k.shape[2]
    per, scale = heads // kv, width ** -0.5 if scale is None else scale
    see = torch.ones(batch, 1, nq, nk, dtype=torch.bool, device=q.device)
    qd, kd, vd = q.double(), k.double(), v.double()
    dod = do.double() if do is not None else None
    if query_groups is not None:
        a, b = (t[torch.arange(batch, device=q.device) % t.shape[0]] for t in (query_groups, key_groups))
        see = ((a[:, :, None] == b[:, None, :]) & (a >= 0)[:, :, None])[:, None]
        zero = torch.zeros((), dtype=torch.float64, device=q.device)
        qd, kd, vd = torch.where((a >= 0)[:, None, :, None], qd, zero), torch.where((b >= 0)[:, None, :, None], kd, zero), torch.where((b >= 0)[:, None, :, None], vd, zero)
        dod = torch.where((a >= 0)[:, None, :, None], dod, zero) if do is not None else None
    if causal:
        see = see & torch.ones(nq, nk, dtype=torch.bool, device=q.device).tril(nk - nq)
    kd, vd = kd.repeat_interleave(per, 1), vd.repeat_interleave(per, 1)
    z = qd @ kd.transpose(-1, -2) * scale
    # a score: width / 4 additions of the matrix instruction at most, the product with scale, and the bias's own rounding when it is taken to base 2
    z_off = (width + 8) * U32 * (abs(scale) * (qd.abs() @ kd.abs().transpose(-1, -2)))
    if table is not None:
        of = torch.arange(batch, device=q.device) // (batch // table.shape[0])
        bias = table.double()[of][:, which].permute(0, 3, 1, 2)
        z = z + bias
        z_off = z_off + 4 * U32 * torch.nan_to_num(bias.abs(), posinf=0.0)
    z_off = z_off + 4 * U32 * torch.nan_to_num(z.abs(), posinf=0.0)
    z = torch.where(see, z, -math.inf)
    there = torch.isfinite(z).any(-1, keepdim=True)
    top = torch.where(there, z.amax(-1, keepdim=True), 0.0)
    e = torch.where(there, torch.exp(z - top), 0.0)
    total = e.sum(-1, keepdim=True)
    p = e / torch.where(there, total, 1.0)
    # of p: two scores' errors (its own and the sum's), the hardware's 2^x (two units), and the sum of all keys
    most = torch.where(torch.isfinite(z), z_off, 0.0).amax(-1, keepdim=True)
    p_rel = 2.02 * most + (nk + 72) * U32
    held = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -16, torch.float16: 2.0 ** -21}[kind]
    step = 2.0 ** -38 if kind == torch.float16 else 0.0           # half a step of the second piece, relative to the largest
    o = p @ vd
    o_raw = (p * (p_rel + held + (nk + 64) * U32)) @ vd.abs() + step * there * vd.abs().sum(-2, keepdim=True)
    out = {"o": (o, rounded(o, kind) + 1.01 * o_raw)}
    if do is None:
        return out
    u = HALF_UNIT[kind]
    o_kept = o_raw + (U32 * o.abs() if kind == torch.float32 else 4 * u * u * o.abs() + (2.0 ** -25 if kind == torch.float16 else 0.0))    # (o and what its rounding left over)
    d = (dod * o).sum(-1, keepdim=True)
    d_off = (dod.abs() * o_kept).sum(-1, keepdim=True) + (width + 8) * U32 * (dod * o).abs().sum(-1, keepdim=True)
    dp = dod @ vd.transpose(-1, -2)
    dp_off = (width + 8) * U32 * (dod.abs() @ vd.abs().transpose(-1, -2))
    dz = p * (dp - d)
    bound = 2 * dod.norm(dim=-1).amax(-1)[:, :, None, None] * vd.norm(dim=-1).amax(-1)[:, :, None, None]
    bound = bound.unflatten(1, (kv, per)).amax(2, keepdim=True).expand(-1, -1, per, -1, -1).flatten(1, 2)
    dz_raw = p * (dp_off + d_off + 4 * U32 * (dp.abs() + d.abs())) + (p_rel + 4 * U32) * dz.abs()
    dz_off = dz_raw + held * dz.abs() + step * bound * (p > 0)
    dq = scale * (dz @ kd)
    dq_off = abs(scale) * (dz_off @ kd.abs() + (nk + 64) * U32 * (dz.abs() @ kd.abs()))
    dv = p.transpose(-1, -2) @ dod
    dv_off = (p * (p_rel + held)).transpose(-1, -2) @ dod.abs() + step * see.double().transpose(-1, -2) @ dod.abs() + (nq * per + 64) * U32 * (p.transpose(-1, -2) @ dod.abs())
    dk = scale * (dz.transpose(-1, -2) @ qd)
    dk_off = abs(scale) * (dz_off.transpose(-1, -2) @ qd.abs() + (nq * per + 64) * U32 * (dz.abs().transpose(-1, -2) @ qd.abs()))
    out["dq"] = (dq, rounded(dq, kind) + 1.01 * dq_off)
    for name, value, off in (("dk", dk, dk_off), ("dv", dv, dv_off)):
        value, off = (t.unflatten(1, (kv, per)).sum(2) for t in (value, off))
        out[name] = (value, rounded(value, kind) + 1.01 * off)
    if table is not None:
        def buckets(t):
            t = t.unflatten(0, (table.shape[0], -1)).sum(1)                               # [T, H, Nq, Nk]
            zero = torch.zeros(table.shape[0], heads, table.shape[1], dtype=torch.float64, device=q.device)
            return zero.index_add_(2, which.reshape(-1), t.flatten(2)).transpose(1, 2)
        total = buckets(dz)
        # sums over 64 pairs and then over tiles, entries and workgroups
        off = buckets(dz_raw) + (nk / 16 + batch + 160) * U32 * buckets(dz.abs())
        out["dtable"] = (total, rounded(total, table.dtype) + 1.01 * off)
    return out


def buckets_of(positions, nq, nk, first_query=0):
    """The bucket of every pair, from what an object of RelativePositions holds."""
    q, k = positions.query_code[first_query:first_query + nq].long(), positions.key_code[:nk].long()
    return positions.bucket[:, 0].long()[q[:, None] - k]
