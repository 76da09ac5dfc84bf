"""The 8-bit cache's calls restated: e4m3 from its definition, the append rule block by block, attention over the values in 64 bits."""
import math

import torch

from paged_ref import F64, attention

BLOCK = 16
RANGE = {torch.bfloat16: (-117, 120), torch.float16: (-15, 8)}


def _positive():
    """The values of codes 0 .. 126: four bits of exponent (bias 7), three of fraction."""
    return [(c & 7) / 8 * 2.0 ** -6 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)]


VALUES = torch.tensor(_positive(), dtype=F64)


def decode(codes):
    c = codes.cpu().long()
    v = torch.cat([VALUES, torch.tensor([math.nan], dtype=F64)])[c & 127]
    return torch.where(c >= 128, -v, v)


def encode(x):
    """Nearest code, ties to the even one; at most 448 in magnitude; NaN to NaN."""
    x = x.to(F64).cpu()
    a = x.abs().nan_to_num(0.0).clamp(max=448.0)
    lo = (torch.searchsorted(VALUES, a, right=True) - 1).clamp(max=125)
    d = (a - VALUES[lo]) - (VALUES[lo + 1] - a)
    code = torch.where((d > 0) | ((d == 0) & (lo % 2 == 1)), lo + 1, lo)
    code = torch.where(torch.signbit(x), code + 128, code)
    return torch.where(x.isnan(), 127, code).to(torch.uint8)


def exponent(values, dtype):
    """The least exponent of the type's range with every finite |value| <= 448 x 2^e."""
    lo, hi = RANGE[dtype]
    most = max([abs(v) for v in values if math.isfinite(v)], default=0.0)
    e = lo
    while e < hi and most > math.ldexp(448.0, e):
        e += 1
    return e


def block_codes(x, e, dtype):
    """Codes of new values x (a tensor) at exponent e."""
    x = torch.where(x.to(F64).isinf(), math.nan, x.to(F64)) * 2.0 ** -e
    if e == RANGE[dtype][1]:
        x = torch.where(x.abs() > 240.0, torch.copysign(torch.full_like(x, 240.0), x), x)
    return encode(x)


def append(codes, exps, table, x, off, ctx, page):
    """One of K and V: codes [pages, page, Hkv, D] and exps [pages, page / 16, Hkv] on the CPU, in place."""
    dtype, Hkv = x.dtype, x.shape[1]
    flat, eflat = codes.view(-1, Hkv, codes.shape[3]), exps.view(-1, Hkv)
    for b in range(len(ctx)):
        n, c = off[b + 1] - off[b], ctx[b]
        for s0 in range(c // BLOCK * BLOCK, c + n if n else 0, BLOCK):
            row = int(table[b][s0 // page]) * page + s0 % page
            first, last = max(c, s0), min(c + n, s0 + BLOCK)
            new = x[off[b] + first - c:off[b] + last - c]
            for h in range(Hkv):
                e = exponent(new[:, h].double().flatten().tolist(), dtype)
                if first > s0:
                    old = min(max(int(eflat[row // BLOCK, h]), RANGE[dtype][0]), RANGE[dtype][1])
                    if e > old:
                        live = flat[row:row + first - s0, h]
                        flat[row:row + first - s0, h] = encode(decode(live) * 2.0 ** (old - e))
                    e = max(e, old)
                flat[row + first - s0:row + last - s0, h] = block_codes(new[:, h], e, dtype)
                eflat[row // BLOCK, h] = e


def values(codes, exps):
    """[pages, page, Hkv, D] in 64 bits."""
    e = exps.cpu().double().repeat_interleave(BLOCK, 1)
    return decode(codes) * (2.0 ** e)[..., None]


def coded_attention(q, k, v, ve, see, scale):
    """paged_ref.attention over the values k, v [m, Hkv, D] (64 bits) of a cache; ve [m, Hkv] their exponents.  The bounds also count
    what fp16 weights lose (2^-32 of the largest weight x 2^ve a key, times a code of 448 at most) and the exponents' sums."""
    out, lse, out_tol, lse_tol = attention(q, k, v, see, scale)
    G = q.shape[1] // k.shape[1]
    see = see.to(q.device)
    for h in range(q.shape[1]):
        s = (q[:, h].to(F64) @ k[:, h // G].T * scale).masked_fill(~see, -math.inf)
        w = torch.exp(s - lse[:, h, None]) * 2.0 ** ve[:, h // G].double()
        lost = torch.nan_to_num(w).amax(1) * s.shape[1] * 448.0 * 2.0 ** -32
        far = 2.0 ** -22 * ve[:, h // G].double().abs().amax()
        out_tol[:, h] += lost[:, None] + far * (out_tol[:, h] * 2.0 ** 8 + out[:, h].abs())
    return out, lse, out_tol, lse_tol
