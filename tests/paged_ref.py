"""The prompt, paged-cache and eviction calls restated in 64 bits, with bounds on how far the kernels may be off.

A bound counts the roundings that a kernel is allowed: the 16-bit rounding of P and of the output (half a step each), the
fp32 sums of D products, and the fp32 exponentials.
"""
import math

import torch

F64 = torch.float64


def tree_mask(parents):
    n = len(parents)
    see = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        j = i
        while j >= 0:
            see[i, j] = True
            j = int(parents[j])
    return see


def causal_mask(n, ctx):
    return torch.arange(ctx + n)[None, :] <= ctx + torch.arange(n)[:, None]


def attention(q, k, v, see, scale):
    """q [n, Hq, D], k and v [m, Hkv, D], see [n, m].  Output, lse, and the bounds of their errors for inputs of q's type."""
    dt = q.dtype
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    dev = q.device
    see = see.to(dev)
    out = torch.zeros(n, Hq, D, dtype=F64, device=dev)
    lse = torch.zeros(n, Hq, dtype=F64, device=dev)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    half = torch.finfo(dt).eps / 2
    for h in range(Hq):
        Q, K, V = q[:, h].to(F64), k[:, h // G].to(F64), v[:, h // G].to(F64)
        V = torch.where(see.any(0)[:, None], V, torch.zeros((), dtype=F64, device=dev))
        s = (Q @ K.T * scale).masked_fill(~see, -math.inf)
        z = torch.logsumexp(s, 1)
        p = torch.where(see, torch.exp(s - z[:, None]), torch.zeros((), dtype=F64, device=dev))
        o, A = p @ V, p @ V.abs()
        # a sum of D fp32 products, each addition off by 2^-23 of what it has reached at most
        reach = (Q.abs() @ K.abs().T * scale).masked_fill(~see, 0.0).amax(1)
        e = 2.0 * (D * 2.0 ** -23 * reach + 2.0 ** -20 * (1 + z.abs()))
        out[:, h], lse[:, h] = o, z
        # fp16 P below 2^-32 of the largest weight is lost; fp16 outputs below 2^-14 lose bits
        lost = s.shape[1] * 2.0 ** -31 * V.abs().amax() + 2.0 ** -25 if dt == torch.float16 else 0.0
        out_tol[:, h] = half * (o.abs() + A) * (1 + half) + e[:, None] * (A + o.abs()) + lost
        lse_tol[:, h] = e
    return out, lse, out_tol, lse_tol


def slots(table, b, length, page):
    j = torch.arange(length, device=table.device)
    return table[b].long()[j // page] * page + j % page


def check(got, want, tol, what):
    err = (got.to(F64) - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), "%s: %d of %d off; worst %g against %g" % (what, int(bad.sum()), bad.numel(), float(err.max()), float(tol.max()))


def weights(q, k, lse, see, scale):
    """[Hkv, m]: the weight that the rows give to each key, and the bound of its error in fp32."""
    n, Hq, D = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    total = torch.zeros(Hkv, k.shape[0], dtype=F64, device=q.device)
    tol = torch.zeros_like(total)
    see = see.to(q.device)
    for h in range(Hq):
        Q, K, z = q[:, h].to(F64), k[:, h // G].to(F64), lse[:, h].to(F64)
        on = see & torch.isfinite(z)[:, None]
        p = torch.where(on, torch.exp(Q @ K.T * scale - torch.where(torch.isfinite(z), z, 0.0)[:, None]), 0.0)
        reach = Q.abs() @ K.abs().T * scale + z.abs()[:, None]
        e = 2.0 * (D * 2.0 ** -23 * torch.where(on, reach, 0.0) + 2.0 ** -20)
        total[h // G] += p.sum(0)
        tol[h // G] += (p * (e + 2.0 ** -24 * n * G)).sum(0)  # n G fp32 additions at most
    return total, tol


def evict_order(weights, positions, next_pos, recent, budget):
    """Which slots of one (request, head) stay, by the definition: host lists."""
    def place(s):
        if positions[s] >= next_pos - recent:
            return (0, 0, 0.0, s)
        return (1, 1, 0.0, s) if math.isnan(weights[s]) else (1, 0, -weights[s], s)

    rank = sorted(range(len(weights)), key=place)
    kept = set(rank[:budget])
    holes = [s for s in range(budget) if s not in kept]
    movers = [s for s in range(budget, len(weights)) if s in kept]
    return list(zip(movers, holes))
