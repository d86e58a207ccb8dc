"""Ragged batches over scattered pages for the paged-cache operators, with a float64 reference on the CPU.

Every page slot that holds no token of the batch is poisoned (NaN values, NaN scales), and block-table entries of pages that
no key needs name pages that do not exist, so that anything read outside the visible keys shows.
"""
import math

import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
E4M3_NAN = 0x7F


def quantise(x, fmt):
    """Row-wise quantisation by the formats' definition, in float64; x: [..., d] -> (codes, float32 scales)."""
    x = x.double()
    top = x.abs().amax(-1)
    if fmt == "int8":
        s = torch.where(top > 0, (top / 127).float().double(), torch.ones_like(top))
        return torch.round(x * torch.where(top > 0, 127 / top, top)[..., None]).clamp(-127, 127).to(torch.int8), s.float()
    s = torch.tensor([2.0 ** math.ceil(math.log2(t / 448)) if t > 0 else 1.0 for t in top.flatten().tolist()], dtype=torch.float64).view(top.shape)
    s = torch.where(448 * s < top, 2 * s, torch.where(224 * s >= top, s / 2, s))  # log2 next to a power of two
    s = torch.where(top > 0, s, torch.ones_like(s))
    return (x / s[..., None]).float().to(torch.float8_e4m3fn), s.float()


class Batch:
    def __init__(self, *, dtype, fmt, nq, nkv, d, page, lens, new, window=0, sinks=0, lead=0, behind=0, seed=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.fmt, self.nq, self.nkv, self.d, self.page = DTYPES[dtype], fmt, nq, nkv, d, page
        self.lens, self.new, self.window, self.sinks = list(lens), list(new), window, sinks
        self.B = len(lens)
        cu = [lead]
        for n in new:
            cu.append(cu[-1] + n)
        self.cu, self.n = cu, cu[-1] + behind
        need = [-(-(a + n) // page) for a, n in zip(lens, new)]
        self.width = max(1, max(need)) + 1
        self.n_pages = sum(need) + 2
        perm = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((self.B, self.width), -7, dtype=torch.int32)
        at = 0
        for b, k in enumerate(need):
            self.table[b, :k] = perm[at:at + k].int()
            at += k
            if window and new[b]:  # pages wholly between the sinks and the first query's window may have been given back
                first = max(0, lens[b] - window + 1)
                for j in range(k):
                    if j * page >= sinks and (j + 1) * page <= first:
                        self.table[b, j] = 1 << 20
        self.q = (torch.randn((self.n, nq, d), generator=g) * spread).to(self.dtype)
        self.values, self.codes, self.scales = {}, {}, {}
        owned = torch.zeros((self.n_pages, page), dtype=torch.bool)
        at = 0
        for b, k in enumerate(need):
            for t in range(lens[b] + new[b]):
                owned[perm[at + t // page], t % page] = True
            at += k
        own4 = owned[:, None, :, None]
        for name in ("k", "v"):
            x = torch.randn((self.n_pages, nkv, page, d), generator=g) * torch.exp(0.4 * torch.randn((self.n_pages, nkv, page, 1), generator=g))
            x = x.to(self.dtype).float()
            if fmt in ("e4m3", "int8"):
                codes, s = quantise(x, fmt)
                self.values[name] = codes.float().double() * s.double()[..., None]
                self.scales[name] = torch.where(owned[:, None, :], s, torch.full_like(s, math.nan))
                if fmt == "e4m3":
                    codes = torch.where(own4, codes.view(torch.uint8), torch.full_like(codes.view(torch.uint8), E4M3_NAN)).view(torch.float8_e4m3fn)
                self.codes[name] = codes
            else:
                x = x.to(DTYPES[fmt])
                self.values[name] = x.double()
                self.codes[name] = torch.where(own4, x, torch.full_like(x, math.nan))
                self.scales[name] = None
        self.real = {b: perm[sum(need[:b]):sum(need[:b + 1])] for b in range(self.B)}

    def row_of(self, b, t):
        return int(self.real[b][t // self.page]), t % self.page

    def max_new(self):
        return max(1, max(self.new))

    def max_context(self):
        return max(1, max(a + n for a, n in zip(self.lens, self.new)))

    def device(self, dev="cuda"):
        def put(t):
            return None if t is None else t.to(dev)
        return dict(q=put(self.q), k_pages=put(self.codes["k"]), v_pages=put(self.codes["v"]), k_scales=put(self.scales["k"]),
                    v_scales=put(self.scales["v"]), cu=torch.tensor(self.cu, dtype=torch.int32, device=dev),
                    lens=torch.tensor(self.lens, dtype=torch.int32, device=dev), table=self.table.to(dev),
                    err=torch.zeros(1, dtype=torch.int32, device=dev))

    def reference(self, scale=None):
        """(out, tol) [n, nq, d] float64; rows of nobody are NaN / 0.  tol bounds a correct kernel's error (see below)."""
        scale = self.d ** -0.5 if scale is None else scale
        out = torch.full((self.n, self.nq, self.d), math.nan, dtype=torch.float64)
        tol = torch.zeros_like(out)
        group = self.nq // self.nkv
        for b in range(self.B):
            a, n = self.lens[b], self.new[b]
            if not n:
                continue
            idx = torch.tensor([self.row_of(b, t) for t in range(a + n)])
            k, v = (self.values[x][idx[:, 0], :, idx[:, 1]] for x in ("k", "v"))  # [T, nkv, d]
            t, p = torch.arange(a + n), torch.arange(a, a + n)[:, None]
            see = t <= p
            if self.window:
                see &= (t > p - self.window) | (t < self.sinks)
            q = self.q[self.cu[b]:self.cu[b] + n].double()
            for h in range(self.nq):
                kh, vh, qh = k[:, h // group], v[:, h // group], q[:, h]
                s = (qh @ kh.t() * scale).masked_fill(~see, -math.inf)
                w = torch.softmax(s, -1)
                rows = slice(self.cu[b], self.cu[b] + n)
                out[rows, h] = w @ vh
                # float32 arithmetic: a score is a sum of d products (and a few scalings), off by at most (d + 8) 2^-24 of the
                # sum of its terms' magnitudes; softmax weights follow with twice that, plus 2^-20 for the exponential and its
                # argument's rounding at these score sizes (|s| < 32: 32 * 2^-24 = 2^-19); sums over T keys add T 2^-24.
                mag = (qh.abs() @ kh.abs().t() * scale).masked_fill(~see, 0).amax(-1, keepdim=True)
                rel = 2 * (self.d + 8) * 2.0 ** -24 * mag + 2.0 ** -18 + 2 * (a + n) * 2.0 ** -24
                aw = w @ vh.abs()
                e = rel * aw
                if self.dtype == torch.bfloat16:  # weights rounded to bf16 (half a step: 2^-8 of each), the output too
                    e = e + 1.01 * 2.0 ** -8 * (aw + (w @ vh).abs())
                tol[rows, h] = e
        return out, tol


def check_attention(batch, got, scale=None):
    ref, tol = batch.reference(scale)
    live = ~torch.isnan(ref[:, 0, 0])
    got = got.double().cpu()[live]
    bad = (got - ref[live]).abs() > tol[live]
    assert torch.isfinite(got).all(), "non-finite output"
    worst = ((got - ref[live]).abs() / tol[live]).max().item()
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} values off, worst {worst:.2f} of the tolerance"
    return live
