"""Ragged batches over a 4-bit paged cache, with float64 references on the CPU.  As in paged_util, slots that hold no token of the batch
are poisoned (NaN parameters, codes 255) and block-table entries of pages that no key needs name pages that do not exist."""
import math

import torch

from paged_util import Batch

MIN_SCALE = 2.0 ** -60


def down_to_bf16(x):
    """The largest bfloat16 not above x (float64, within float32's range), as float64."""
    y = x.float().to(torch.bfloat16)
    below = torch.nextafter(y, torch.full_like(y, -math.inf))
    return torch.where(y.double() > x, below, y).double()


def quantise4(x):
    """The format's definition in float64: rows [..., d] -> (bytes [..., d / 2], parameters bfloat16 [..., 2, 2])."""
    h = x.double().unflatten(-1, (2, x.shape[-1] // 2))
    m = down_to_bf16(h.amin(-1))
    s = ((h.amax(-1) - m) / 15).to(torch.bfloat16).double().clamp(min=MIN_SCALE)
    c = torch.round((h - m[..., None]) / s[..., None]).clamp(0, 15).to(torch.uint8)
    return c[..., 0, :] | c[..., 1, :] << 4, torch.stack([s, m], -1).to(torch.bfloat16)


def values4(codes, p):
    """float64 values of cached rows."""
    p = p.double()
    lo, hi = (codes & 15).double(), (codes >> 4).double()
    return torch.cat([lo * p[..., 0, 0, None] + p[..., 0, 1, None], hi * p[..., 1, 0, None] + p[..., 1, 1, None]], -1)


class Batch4(Batch):
    """offset: added to K and V per head dim, times N(0, 1), so that rows are not centred."""

    def __init__(self, *, dtype, offset=0.0, rows=None, **kw):
        super().__init__(dtype=dtype, fmt=dtype, **kw)
        self.fmt, g = "int4", torch.Generator().manual_seed(kw.get("seed", 0) + 991)
        for name in "kv":
            owned = ~torch.isnan(self.codes[name][:, :1, :, :1].float())  # [n_pages, 1, page, 1]
            x = self.values[name] + offset * torch.randn(self.d, generator=g, dtype=torch.float64)
            if rows is not None:
                x = rows(name, x)
            codes, p = quantise4(x.float() if dtype == "f32" else x.to(torch.bfloat16).float())
            self.values[name] = values4(codes, p)
            self.codes[name] = torch.where(owned, codes, torch.full_like(codes, 255))
            self.scales[name] = torch.where(owned[..., None], p, torch.full_like(p, math.nan))

    def reference(self, scale=None):
        """(out, tol) as Batch.reference.  tol, beside float32's share there, which here is taken of the products' own terms (code * s and m
        apart, together at most 2 |m| + |value| each): for bfloat16 queries a rounding of the output to bfloat16 (half a step, 2^-8), and of what
        the tensor cores take to float16 (half a step, 2^-11, once for a weight and once for a value; of K in calls of more than 16 rows,
        which moves a score by at most 2^-11 of the sum of its terms' magnitudes, a weight by twice that)."""
        scale = self.d ** -0.5 if scale is None else scale
        out = torch.full((self.n, self.nq, self.d), math.nan, dtype=torch.float64)
        tol = torch.zeros_like(out)
        group, half = self.nq // self.nkv, self.d // 2
        few = self.max_new() * group <= 16
        for b in range(self.B):
            a, n = self.lens[b], self.new[b]
            if not n:
                continue
            idx = torch.tensor([self.row_of(b, t) for t in range(a + n)])
            k, v = (self.values[x][idx[:, 0], :, idx[:, 1]] for x in "kv")  # [T, nkv, d]
            # magnitudes of the two terms of a value
            km, vm = (x.abs() + 2 * self.scales[y][idx[:, 0], :, idx[:, 1]][..., 1].double().abs().repeat_interleave(half, -1) for x, y in ((k, "k"), (v, "v")))
            t, p = torch.arange(a + n), torch.arange(a, a + n)[:, None]
            see = t <= p
            if self.window:
                see &= (t > p - self.window) | (t < self.sinks)
            q = self.q[self.cu[b]:self.cu[b] + n].double()
            rows = slice(self.cu[b], self.cu[b] + n)
            for h in range(self.nq):
                g, qh = h // group, q[:, h]
                w = torch.softmax((qh @ k[:, g].t() * scale).masked_fill(~see, -math.inf), -1)
                o = w @ v[:, g]
                mag = (qh.abs() @ km[:, g].abs().t() * scale).masked_fill(~see, 0).amax(-1, keepdim=True)
                rel = 2 * (self.d + 8) * 2.0 ** -24 * mag + 2.0 ** -18 + 2 * (a + n) * 2.0 ** -24
                aw = w @ vm[:, g]
                if self.dtype == torch.bfloat16:
                    rel = rel + 2 * 2.0 ** -11 + (0 if few else 2 * 2.0 ** -11 * mag)
                out[rows, h] = o
                tol[rows, h] = rel * aw + (1.01 * 2.0 ** -8 * o.abs() if self.dtype == torch.bfloat16 else 0)
        return out, tol


