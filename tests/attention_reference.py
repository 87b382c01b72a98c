"""Attention with a sliding window and sinks in 64 bits on the host, every pair written down, and how far a kernel may be from it.

The bounds count roundings.  u is half a step of fp32 (2^-24), h half a step of the type (`torch.finfo(t).eps / 2`).  A score is
a sum of dh products, off by at most dh u times the sum of their magnitudes, and its exponential by that much relative to itself, plus
an exponential's own error and a maximum taken off (32 u together).  A sum of n terms adds n u.  In bf16 the probabilities and dS are
rounded to bf16 where they are multiplied (h relative each, to probabilities scaled by a running maximum as well), and results are
rounded once to their type."""
import math

import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def sees(first, n, m, window, sinks):
    """[n, m]: which of rows first .. first + n - 1 sees which of m positions"""
    i, j = first + torch.arange(n)[:, None], torch.arange(m)[None, :]
    return (j <= i) & ((j > i - window) | (j < sinks))


def forward(q, k, v, mask, dtype):
    """q [n, H, dh], k and v [m, Hkv, dh] in 64 bits, mask [n, m] -> o [n, H, dh], lse [n, H], and the bounds of both"""
    n, H, dh = q.shape
    G, c, h = H // k.shape[1], 1.0 / math.sqrt(dh), half_step(dtype)
    o, lse, eo, el = (torch.zeros((n, H) + s, dtype=torch.float64) for s in ((dh,), (), (dh,), ()))
    for x in range(H):
        kk, vv = k[:, x // G], v[:, x // G]
        s = (q[:, x] @ kk.T * c).masked_fill(~mask, -math.inf)
        empty = ~mask.any(1)
        lse[:, x] = torch.logsumexp(s, 1)
        p = torch.where(mask, torch.exp(s - lse[:, x, None]), 0.0)
        p[empty] = 0.0
        o[:, x] = p @ torch.where(mask.any(0)[:, None], vv, 0.0)
        size = (q[:, x].abs() @ kk.abs().T * c).masked_fill(~mask, 0.0).amax(1)
        rel = U * (2 * dh * size + mask.sum(1) + 32) + (h if dtype != torch.float32 else 0.0)
        eo[:, x] = 2 * rel[:, None] * (p @ torch.where(mask.any(0)[:, None], vv.abs(), 0.0)) + h * o[:, x].abs()
        el[:, x] = U * (2 * dh * size + mask.sum(1) + 32) + 2 * U * lse[:, x].abs().nan_to_num(posinf=0.0)
    return o, lse, eo, el


def backward(q, k, v, o, g, lse, mask, dtype):
    """the gradient of sum(o * g) from q, k, v and the given o and lse (rows x heads) -> dq, dk, dv and their bounds"""
    n, H, dh = q.shape
    G, c, h = H // k.shape[1], 1.0 / math.sqrt(dh), half_step(dtype)
    extra = h if dtype != torch.float32 else 0.0
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    eq, ek, ev = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for x in range(H):
        y = x // G
        kk, vv, qq, gg = k[:, y], v[:, y], q[:, x], g[:, x]
        p = torch.where(mask, torch.exp(qq @ kk.T * c - lse[:, x, None]), 0.0)
        D = (gg * o[:, x]).sum(1, keepdim=True)
        ds = p * (gg @ vv.T - D)
        size = (qq.abs() @ kk.abs().T * c).masked_fill(~mask, 0.0).amax(1, keepdim=True)
        rel = U * (2 * dh * size + 32 + lse[:, x, None].abs())
        inner = gg.abs() @ vv.abs().T + (gg.abs() * o[:, x].abs()).sum(1, keepdim=True)
        e_ds = rel * ds.abs() + p * U * (dh + 2) * inner + extra * ds.abs()
        terms_q = U * mask.sum(1, keepdim=True)
        terms_k = U * G * mask.sum(0)[:, None]
        dq[:, x] = ds @ kk * c
        eq[:, x] = (e_ds + terms_q * ds.abs()) @ kk.abs() * c
        dk[:, y] += ds.T @ qq * c
        ek[:, y] += e_ds.T @ qq.abs() * c + terms_k * (ds.abs().T @ qq.abs()) * c
        dv[:, y] += p.T @ gg
        ev[:, y] += ((rel + extra) * p).T @ gg.abs() + terms_k * (p.T @ gg.abs())
    return dq, dk, dv, eq + h * dq.abs(), ek + h * dk.abs(), ev + h * dv.abs()


def inside(got, want, bound, what=""):
    """Every element of `got` is within `bound` of `want`.  Nothing passes that is not shown to: where `want` is finite `got` has to be
    finite too (a NaN compares as neither inside nor outside), an infinity has to be that infinity and a NaN a NaN."""
    got, want = got.double().cpu(), want.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    near = torch.isfinite(want) & torch.isfinite(got) & ((got - want).abs() <= bound + 1e-30)
    out = ~(same | near)
    at = out.nonzero()[:3].tolist()
    assert not bool(out.any()), f"{what}: {int(out.sum())} of {out.numel()} out of bounds, among them {[(i, float(got[tuple(i)]), float(want[tuple(i)])) for i in at]}"


def definition(q, k, v, mask):
    """o and lse in 64 bits for inputs of any value: a sum runs over the pairs of the mask alone, so that a value that is not finite
    reaches exactly the rows that see it.  A row that sees nothing has o = 0 and lse = -inf; one whose visible scores are all -inf has
    o = NaN (0 / 0) and lse = -inf."""
    n, H, dh = q.shape
    G, c = H // k.shape[1], 1.0 / math.sqrt(dh)
    o, lse = torch.zeros((n, H, dh), dtype=torch.float64), torch.full((n, H), -math.inf, dtype=torch.float64)
    for i in range(n):
        j = mask[i].nonzero()[:, 0]
        if len(j):
            kk, vv = k[j].repeat_interleave(G, 1), v[j].repeat_interleave(G, 1)          # [keys, H, dh]
            s = (q[i] * kk).sum(2) * c
            top = s.amax(0)                                                              # NaN where a score is
            p = torch.exp(s - top)                                                       # NaN where top is infinite
            p = torch.where(torch.isinf(top) & (top < 0), torch.zeros_like(p), p)        # all -inf: a sum of zeros
            total = p.sum(0)
            o[i] = (p[:, :, None] * vv).sum(0) / total[:, None]
            lse[i] = top + torch.log(total)
    return o, lse
