"""Rotary positions of queries and keys (``rs_rotary``): the frequencies' table and the call over tensors."""
import math
from fractions import Fraction

import torch

from . import respec as rs

_CODES = {torch.bfloat16: rs.RS_BF16, torch.float16: rs.RS_F16}
_LAYOUTS = dict(half=rs.RS_ROTARY_HALF, interleaved=rs.RS_ROTARY_INTERLEAVED)
_PI = Fraction(314159265358979323846264338327950288419716939937510, 10 ** 50)


def frequencies(rot, base=10000.0, factor=1.0, trained=None, low=1.0, high=4.0):
    """Radians a position of the rot / 2 pairs: base^(-2 i / rot), in 64 bits.  For contexts `factor` times as long as the `trained`
    one: waves that fit into it fewer than `low` times are stretched by the factor, those that fit `high` times or more are kept, and
    those between go from one to the other in proportion.  Without `trained` all are stretched."""
    if rot < 2 or rot % 2:
        raise ValueError("rot=%d: an even number expected" % rot)
    if not (base > 0 and factor > 0 and low < high):
        raise ValueError("base=%g, factor=%g, low=%g, high=%g: positive ones expected, low below high" % (base, factor, low, high))
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        keep = 0.0 if trained is None else min(1.0, max(0.0, (trained * f / (2 * math.pi) - low) / (high - low)))
        out.append(f * (keep + (1.0 - keep) / factor))
    return torch.tensor(out, dtype=torch.float64)


def turns(freq):
    """The table that the kernel takes: each frequency as a fraction of a turn, in units of 2^-64 (int64 words, on freq's device).
    Made on the host, once per model (64 frequencies 0.8 ms, and a wait for those on a device)."""
    f = freq.double().tolist()
    if not all(abs(x) < 2.0 ** 96 for x in f):  # (for larger ones pi would need more digits)
        raise ValueError("freq: values below 2^96 expected")
    # exact but for the last bit: a quotient in 64-bit floating point would be off by 2^-52, 2^-21 of a turn at position 2^31
    words = [round(Fraction(x) / (2 * _PI) * 2 ** 64) % 2 ** 64 for x in f]
    return torch.tensor([w - 2 ** 64 if w >= 2 ** 63 else w for w in words], dtype=torch.int64, device=freq.device)


class Rotary:
    """The positions of one model: heads of D values, of which the first rot are turned; `scale` multiplies the turned values."""

    def __init__(self, D, rot=None, layout="half", freq=None, scale=1.0, device="cuda"):
        rot = D if rot is None else rot
        if layout not in _LAYOUTS:
            raise ValueError("layout=%r: one of %s expected" % (layout, sorted(_LAYOUTS)))
        if not (8 <= D <= 512 and D % 8 == 0 and 2 <= rot <= D and rot % 2 == 0):
            raise ValueError("D=%d, rot=%d: a multiple of 8 up to 512 and an even number up to it expected" % (D, rot))
        freq = frequencies(rot) if freq is None else freq
        if freq.numel() != rot // 2:
            raise ValueError("freq: %d values expected, not %d" % (rot // 2, freq.numel()))
        self.D, self.rot, self.layout, self.scale = D, rot, layout, float(scale)
        self.freq = freq.to(torch.float64).cpu()
        self.turns = turns(self.freq).to(device)

    def __call__(self, q, k, pos, out=None, inverse=False):
        """q [T, Hq, D] and k [T, Hkv, D] (rows may be parts of wider ones; either may be None) at the positions pos [T] int32.
        Returns (q, k) turned: new tensors, or those in `out`, which may be q and k themselves.  inverse: by the negative angles,
        still times `scale`, which is the gradient.  Where q or k requires a gradient the results have theirs, and `out` is refused."""
        x = q if q is not None else k
        if x is None:
            raise ValueError("q or k expected")
        if x.dtype not in _CODES:
            raise ValueError("q and k of bfloat16 or float16 expected")
        T = x.shape[0]
        if pos.dtype != torch.int32 or pos.dim() != 1 or pos.numel() != T:
            raise ValueError("pos: %d values of int32 expected, not %s of %s" % (T, list(pos.shape), pos.dtype))
        out = (None, None) if out is None else out
        args, outs = [], []
        for name, t, o in (("q", q, out[0]), ("k", k, out[1])):
            if t is None:
                args += [None, 0, None, 0]
                outs.append(None)
                continue
            if o is None:
                o = torch.empty(t.shape, dtype=t.dtype, device=t.device)
            for y in (t, o):
                if y.dim() != 3 or y.shape[0] != T or y.shape[2] != self.D or y.dtype != x.dtype or y.shape != t.shape:
                    raise ValueError("%s: [%d, heads, %d] of %s expected, not %s of %s" % (name, T, self.D, x.dtype, list(y.shape), y.dtype))
            args += [t, _apart(t), o, _apart(o)]
            outs.append(o)
        if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (q, k, *out)):
            if any(o is not None for o in out):
                raise ValueError("out: results with a gradient are new tensors")
            return _Turned.apply(self, q, k, pos, inverse)
        heads = [0 if t is None else t.shape[1] for t in (q, k)]
        rs.rs_rotary(*args, _CODES[x.dtype], pos, T, *heads, self.D, self.rot, _LAYOUTS[self.layout], self.turns, self.scale, int(inverse))
        return tuple(outs)


class _Turned(torch.autograd.Function):
    """A linear map: its gradient is the same call with the opposite angles."""

    @staticmethod
    def forward(ctx, rotary, q, k, pos, inverse):
        ctx.set_materialize_grads(False)
        ctx.rotary, ctx.inverse = rotary, inverse
        ctx.save_for_backward(pos)
        out = rotary(q, k, pos, inverse=inverse)
        ctx.mark_non_differentiable(*(o for o, needed in zip(out, ctx.needs_input_grad[1:3]) if o is not None and not needed))
        return out

    @staticmethod
    def backward(ctx, dq, dk):
        dq, dk = (_rows(g) if g is not None and needed else None for g, needed in zip((dq, dk), ctx.needs_input_grad[1:3]))
        if dq is None and dk is None:
            return None, None, None, None, None
        return (None, *ctx.rotary(dq, dk, ctx.saved_tensors[0], inverse=not ctx.inverse), None, None)


def _rows(x):
    """x as the call takes it: a gradient may be broadcast or transposed."""
    fits = x.stride(2) == 1 and x.stride(1) == x.shape[2] and _apart(x) >= x.shape[1] * x.shape[2] and _apart(x) % 8 == 0 and x.data_ptr() % 16 == 0
    return x if fits else x.contiguous()


def _apart(x):
    return x.stride(0) if x.shape[0] > 1 else x.shape[1] * x.shape[2]
