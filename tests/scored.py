"""Plain statements, in 64 bits, of the scored step, the attention weight and the eviction, and how far a result may be off.

Bounds.  Half a step of a type's rounding is u(t) = finfo(t).eps / 2, relative to the value.  A rotated query of a bf16 cache is rounded
once, so a score moves by at most d_r = u(bf16) * scale * sum_c |q_c k_rc| (a cap's slope is 1 at most), a probability is rounded once
before it meets its value row and the output once at the end:
    |out - exact| <= sum_r p_r (d_r + u) (|v_r| + |out|) + u |out|        (to first order; d_r is well below 1 here)
What fp32 adds is counted with u(f32): a dot product of d terms (d + 2) u sum |q_c k_rc| scale, doubled for tensor cores that cut sums
short instead of rounding them; a score in log2 units, its reference and their difference 4 u (|s| + |lse|) log2(e); a cap 2^-20 of the
cap; an exponential 2^-22; a sum over N terms N u."""
from __future__ import annotations

import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def turned(x, pos0, base):
    """x [n, heads, d] rotated at pos0, pos0 + 1, ... (pairs j, j + d/2), in 64 bits."""
    d = x.shape[-1]
    inv = base ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device=x.device) / d)
    at = (pos0 + torch.arange(x.shape[0], dtype=torch.float64, device=x.device))[:, None, None] * inv
    a, b = x.double().split(d // 2, dim=-1)
    return torch.cat([a * at.cos() - b * at.sin(), b * at.cos() + a * at.sin()], dim=-1)


def ranges(n, rows, prefix, appended, first=None, end=None, device="cuda"):
    """(first, end) rows that each of n tokens sees, out-of-range entries brought to the nearest row."""
    e = torch.arange(prefix + 1, prefix + n + 1, device=device) if appended else torch.full((n,), rows, device=device)
    f = torch.zeros(n, dtype=torch.int64, device=device)
    return (f if first is None else first.long().clamp(min=0)), (e if end is None else end.long().clamp(0, rows))


def scores(q, keys, scale, pos0, softcap=0.0, slopes=None):
    """(s [n, H, rows], sum_c |q_c k_rc| * scale) of rotated queries [n, H, d] on keys [Hkv, rows, d]."""
    n, heads, d = q.shape
    kv, rows = keys.shape[:2]
    x = q.double().view(n, kv, heads // kv, d)
    s = torch.einsum("nkgd,krd->nkgr", x, keys.double()).reshape(n, heads, rows) * scale
    size = torch.einsum("nkgd,krd->nkgr", x.abs(), keys.double().abs()).reshape(n, heads, rows) * scale
    if softcap:
        s = softcap * torch.tanh(s / softcap)
    if slopes is not None:
        far = (pos0 + torch.arange(n, device=q.device)[:, None] - torch.arange(rows, device=q.device)).abs().double()
        s = s - slopes.double().view(1, heads, 1) * far[:, None]
    return s, size


def attend(q, keys, values, seen, scale, pos0, softcap=0.0, slopes=None, dtype=torch.bfloat16, out_dtype=None, tensor_cores=True):
    """(out [n, H, d], lse [n, H], bound of out, bound of lse) for rotated, unrounded queries."""
    n, heads, d = q.shape
    kv, rows = keys.shape[:2]
    s, size = scores(q, keys, scale, pos0, softcap, slopes)
    row = torch.arange(rows, device=q.device)
    hidden = ~((row >= seen[0][:, None]) & (row < seen[1][:, None]))
    s = s.masked_fill(hidden[:, None], -math.inf)
    lse = torch.logsumexp(s, -1)
    some = lse > -math.inf
    p = torch.where(some[..., None], torch.exp(s - torch.where(some, lse, 0.0)[..., None]), 0.0)
    group = heads // kv
    v = values.double()

    def times(w, x):
        return torch.einsum("nkgr,krd->nkgd", w.view(n, kv, group, rows), x).reshape(n, heads, d)

    out = times(p, v)
    u, f = U[dtype], U[torch.float32]
    s0 = torch.where(hidden[:, None], 0.0, s).abs()
    move = (u if dtype == torch.bfloat16 else 16 * f) * size + (2 if tensor_cores else 1) * (d + 2) * f * size
    move = move + 4 * f * 1.4427 * (s0 + torch.where(some, lse, 0.0).abs()[..., None]) + 2.0 ** -22 + (softcap * 2.0 ** -20 if softcap else 0.0)
    if slopes is not None:
        move = move + 4 * f * slopes.double().abs().view(1, heads, 1) * (pos0 + n + rows)
    move = torch.where(hidden[:, None], 0.0, move)
    sums = rows * f
    bound = times(p * (move + (u if dtype == torch.bfloat16 else 0.0) + sums), v.abs()) + out.abs() * ((p * move).sum(-1) + sums)[..., None]
    bound = 1.1 * bound + U[out_dtype or dtype] * out.abs() + 1e-30
    return out, lse, bound, 1.1 * ((p * move).sum(-1) + sums) + 2 * f * lse.abs().clamp(max=1e30)


def mass(q, keys, lse, seen, scale, pos0, softcap=0.0, slopes=None, mass_in=None, decay=1.0, held=None, tensor_cores=True):
    """(mass [Hkv, rows], bound) for the rotated queries as given and the denominators as given."""
    n, heads, d = q.shape
    kv, rows = keys.shape[:2]
    s, size = scores(q, keys, scale, pos0, softcap, slopes)
    row = torch.arange(rows, device=q.device)
    hidden = ~((row >= seen[0][:, None]) & (row < seen[1][:, None]))
    l = lse.double()
    p = torch.where(hidden[:, None] | (l == -math.inf)[..., None], 0.0, torch.exp(s - l[..., None]))
    f = U[torch.float32]
    move = (2 if tensor_cores else 1) * (d + 2) * f * size + 4 * f * 1.4427 * (s.abs() + l.abs()[..., None]) + 2.0 ** -22
    if softcap:
        move = move + softcap * 2.0 ** -20
    if slopes is not None:
        move = move + 4 * f * slopes.double().abs().view(1, heads, 1) * (pos0 + n + rows)
    got = p.view(n, kv, -1, rows).sum((0, 2))
    off = torch.where(p > 0, p * move, 0.0).view(n, kv, -1, rows).sum((0, 2)) + n * heads // kv * f * got
    if mass_in is not None and decay:
        before = mass_in.double()[:, :rows].clone() * decay
        before[:, held:] = 0
        got = got + before
        off = off + 2 * f * before.abs()
    return got, 1.1 * off + f * got.abs() + 1e-30


def kept_rows(mass, rows, n_sink, n_recent, budget):
    """[Hkv, budget]: the rows an eviction keeps."""
    got = []
    for w in mass[:, :rows].double().cpu().tolist():
        between = sorted(range(n_sink, rows - n_recent), key=lambda r: (-(w[r] if w[r] == w[r] else -math.inf), w[r] != w[r], r))
        best = between[:budget - n_sink - n_recent]
        got.append(sorted(best + list(range(n_sink)) + list(range(rows - n_recent, rows))))
    return torch.tensor(got, dtype=torch.int32)
