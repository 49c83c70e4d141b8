"""References of the operators around the selection, in 64 bits from their definitions, and the bounds that their outputs are held to.

Bounds (u = 2^-24, half a step of fp32, and r = half a step of the tensors' type: 2^-24 or 2^-8)
  logit    x_ij = q_i k_j / sqrt(d) over d products summed in fp32 in any order, the scale's rounding and one more multiplication:
           |error| <= e_i = (d + 4) u max_j sum_c |q_ic k_jc| / sqrt(d)
  softmax  exponentials of 32 bits and sums of n terms: each p_ij is off by a factor within 1 +- 2 (e_i + n u + 32 u): once for
           its own exponent, once for the normaliser; 32 u covers the exponential's own error (2 units in the last
           place, and 2^-22 relative of the exponent's argument, whose size is below 2^5 where p counts)
  output   |error| <= (that + r of the probabilities' rounding where the values are bf16) * sum_j p_ij |v_jc|, plus the accumulation's
           n u of the same sum, plus r |out| for the last rounding
  lse      e_i + (n + 32) u + 2 u |lse|;   weights: the factor above, summed, and u of the whole
"""
import math

import torch

U = 2.0 ** -24


def half_step(dtype) -> float:
    return torch.finfo(dtype).eps / 2


def attention(q, k, v, limits, present=None):
    """q [R, d] against k, v [n, d] in float64; row i sees keys j < limits[i] with present[j].
    Returns out, lse, p, bounds (dict).  What a row does not see is taken out before any arithmetic."""
    n, d = k.shape
    q = q.double()
    seen = torch.arange(n, device=q.device)[None, :] < limits[:, None]
    if present is not None:
        seen &= present[None, :]
    any_seen = seen.any(0)
    k = torch.where(any_seen[:, None], k.double(), torch.zeros((), dtype=torch.float64, device=q.device))
    v = torch.where(any_seen[:, None], v.double(), torch.zeros((), dtype=torch.float64, device=q.device))
    # a key that some rows see and others do not: those that do not see it must not meet its infinities
    fine_k, fine_v = torch.nan_to_num(k, 0, 0, 0), torch.nan_to_num(v, 0, 0, 0)
    x = (q @ fine_k.T) / math.sqrt(d)
    x = torch.where(seen, x, torch.full_like(x, -math.inf))
    lse = torch.logsumexp(x, 1)
    p = torch.where(seen, torch.exp(x - torch.where(torch.isfinite(lse), lse, torch.zeros_like(lse))[:, None]), torch.zeros_like(x))
    out = p @ fine_v
    e = (d + 4) * U * (torch.where(seen, q.abs() @ fine_k.abs().T, torch.zeros_like(x)).amax(1) if n else torch.zeros(len(q), device=q.device)) / math.sqrt(d)
    factor = 2 * (e + (n + 32) * U)
    return out, lse, p, {"e": e, "factor": factor, "abs": p @ fine_v.abs(), "n": n}


def output_bound(ref, bounds, dtype):
    r = half_step(dtype)
    inner = bounds["factor"] + bounds["n"] * U + (r if dtype != torch.float32 else 0.0)
    return inner[:, None] * bounds["abs"] * (1 + r) + r * ref.abs() + 1e-30


def lse_bound(lse, bounds):
    return bounds["e"] + (bounds["n"] + 32) * U + 2 * U * torch.where(torch.isfinite(lse), lse.abs(), torch.zeros_like(lse))


def assert_close(got, ref, bound, what):
    got = got.double()
    same = (got == ref) | (torch.isnan(got) & torch.isnan(ref))
    err = torch.where(same, torch.zeros_like(ref), (got - ref).abs())
    worst = (err - bound).max().item() if err.numel() else 0.0
    assert not torch.isnan(err).any() and worst <= 0, f"{what}: off by {err.max().item():.3g}, {worst:.3g} more than its bound"


# ---- rotary positions ------------------------------------------------------------------------
def frequencies(rot, base, scaling="none", factor=1.0, original=0.0, low=1.0, high=4.0):
    f = []
    for i in range(rot // 2):
        b = base * factor ** (rot / (rot - 2)) if scaling == "base" and rot > 2 else base
        w = b ** (-2 * i / rot)
        if scaling == "linear":
            w /= factor
        if scaling == "bands":
            t = min(max((original * w / (2 * math.pi) - low) / (high - low), 0.0), 1.0)
            w *= t + (1 - t) / factor
        f.append(w)
    return f


def rotated(x, positions, freqs, order, scale=1.0):
    """x [tokens, heads, d], float64."""
    y = x.double().cpu()
    z = y.clone()
    rot = 2 * len(freqs)
    for i, f in enumerate(freqs):
        j, k = (i, i + rot // 2) if order == "half" else (2 * i, 2 * i + 1)
        a = (positions.double().cpu() * f)[:, None]
        z[..., j] = (y[..., j] * torch.cos(a) - y[..., k] * torch.sin(a)) * scale
        z[..., k] = (y[..., k] * torch.cos(a) + y[..., j] * torch.sin(a)) * scale
    return z


def rotary_bound(x, positions, freqs, scale, dtype):
    """|error| of a turned value: the angle is off by at most 2^-31 pi turns of truncation, 2^-24 pi of its rounding and 2^-50 of the
    reference's own product with the position; sine and cosine by 2 units; scale, products and sum one rounding each;
    then one to the type."""
    big = x.double().abs().amax(-1, keepdim=True).cpu()
    angle = math.pi * (2.0 ** -30 + 2.0 ** -24) + positions.double().abs().cpu()[:, None, None] * 2.0 ** -50
    return 2 * big * abs(scale) * (angle + 8 * U) * (1 + half_step(dtype)) + half_step(dtype) * 2 * big * max(1.0, abs(scale))


# ---- the paged cache ---------------------------------------------------------------------------
class Cache:
    """Pools, table and per-row bookkeeping of a small paged cache on the GPU, rows of unused pages filled with NaN."""

    def __init__(self, gen, dtype, batch, hk, d, page, max_pages, layout="phsd", layers=1, spare=2, fill=float("nan")):
        self.dtype, self.batch, self.hk, self.d, self.page, self.max_pages, self.layout = dtype, batch, hk, d, page, max_pages, layout
        self.num_pages = batch * max_pages + spare
        self.cap = page * max_pages
        self.table = torch.randperm(self.num_pages, generator=gen)[: batch * max_pages].view(batch, max_pages).to(torch.int32).cuda()
        shape = (self.num_pages, hk, page, d) if layout == "phsd" else (self.num_pages, page, hk, d)
        self.k = [torch.full(shape, fill, dtype=dtype, device="cuda") for _ in range(layers)]
        self.v = [torch.full(shape, fill, dtype=dtype, device="cuda") for _ in range(layers)]

    def slot(self, pool, b, h, row):
        page = int(self.table[b, row // self.page])
        return pool[page, h, row % self.page] if self.layout == "phsd" else pool[page, row % self.page, h]

    def rows(self, pool, b, h, n):
        """The first n rows of a unit [n, d] and whether their pages exist."""
        pages = self.table[b].long().cpu()
        ok = (pages >= 0) & (pages < self.num_pages)
        x = pool[pages.clamp(0, self.num_pages - 1).cuda()]
        x = x[:, h] if self.layout == "phsd" else x[:, :, h]
        return x.reshape(-1, self.d)[:n], ok.repeat_interleave(self.page)[:n].cuda()

    def fill(self, gen, lengths, scale=1.0):
        """Random rows 0 .. lengths[b][h] - 1 of every unit."""
        for pool in self.k + self.v:
            for b in range(self.batch):
                for h in range(self.hk):
                    n = int(lengths[b][h])
                    x = (scale * torch.randn((n, self.d), generator=gen)).to(self.dtype).cuda()
                    r = torch.arange(n)
                    pages = self.table[b].long().cpu()[r // self.page]
                    good = (pages >= 0) & (pages < self.num_pages)
                    p, s = pages[good].cuda(), (r % self.page)[good].cuda()
                    if self.layout == "phsd":
                        pool[p, h, s] = x[good.cuda()]
                    else:
                        pool[p, s, h] = x[good.cuda()]
