"""References of the 8-bit cache, the norms with rotary positions and the drafts, in 64 bits from their definitions."""
import torch

import operators_util as ou
from paper_2503_17922_b200 import binding as wkv

U = ou.U
MOST = {"e4m3": 448.0, "i8": 127.0}


def powers(e):
    """2^e, exact: from the language's own powers."""
    table = torch.tensor([2.0 ** k for k in range(-200, 201)], dtype=torch.float64, device=e.device)
    return table[(e + 200).long()]


def quantised(x, kind):
    """Scale bytes and what rows x [..., d] stand for once they are codes; NaN rows where an element is infinite or NaN."""
    y = x.double()
    big = y.abs().amax(-1)
    fine = torch.isfinite(big)
    big = torch.where(fine, big, torch.ones_like(big))
    e = torch.ceil(torch.log2((big / MOST[kind]).clamp(min=2.0 ** -190)))
    e = torch.where(big > MOST[kind] * powers(e), e + 1, e)              # (the logarithm's own rounding)
    e = torch.where(big <= MOST[kind] * powers(e - 1), e - 1, e).clamp(-100, 100)
    y = torch.where(fine[..., None], y, torch.zeros_like(y)) / powers(e)[..., None]
    step = torch.ones_like(y)
    if kind == "e4m3":                                                   # three bits behind the first, which is 2^-6 at least
        step = powers(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    y = (torch.round(y / step) * step).clamp(-MOST[kind], MOST[kind]) * powers(e)[..., None]
    return torch.where(fine, e + 127, torch.full_like(e, 255)).to(torch.uint8), torch.where(fine[..., None], y, torch.full_like(y, float("nan")))


def decoded(codes, kind):
    return codes.view(torch.float8_e4m3fn if kind == "e4m3" else torch.int8).double()


def values(codes, scales, kind):
    """What codes [..., d] and scale bytes [...] stand for, 64 bits."""
    y = decoded(codes, kind) * powers(scales.int() - 127)[..., None]
    return torch.where((scales == 255)[..., None], torch.full_like(y, float("nan")), y)


class Cache8:
    """Pools of codes, scales, table and bookkeeping of a small 8-bit cache on the GPU; unused rows hold 0x7f (NaN as E4M3) and scale 255."""

    def __init__(self, gen, kind, batch, hk, d, page, max_pages, layout="phsd", layers=1, spare=2):
        self.kind, self.batch, self.hk, self.d, self.page, self.max_pages, self.layout = kind, batch, hk, d, page, max_pages, layout
        self.num_pages, self.cap = batch * max_pages + spare, page * max_pages
        self.table = torch.randperm(self.num_pages, generator=gen)[: batch * max_pages].view(batch, max_pages).to(torch.int32).cuda()
        shape = (self.num_pages, hk, page, d) if layout == "phsd" else (self.num_pages, page, hk, d)
        self.codes = [[torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda") for _ in range(2)] for _ in range(layers)]
        self.scales = [[torch.full((self.num_pages, hk, page), 255, dtype=torch.uint8, device="cuda") for _ in range(2)] for _ in range(layers)]

    def describe(self, dtype, hq, max_new=1, cu_new=None):
        cache = wkv.PagedCache8(kind=self.kind, dtype=dtype, batch=self.batch, n_q_heads=hq, n_kv_heads=self.hk, head_dim=self.d, page_size=self.page,
                                num_pages=self.num_pages, block_table=self.table, max_new=max_new, cu_new=cu_new, layout=self.layout)
        return cache, [wkv.Layer8(cache, c[0], c[1], s[0], s[1]) for c, s in zip(self.codes, self.scales)]

    def places(self, b, rows):
        """Pages and slots of rows (long, on the host), and which of them have a page."""
        pages = self.table[b].long().cpu()[rows // self.page]
        return pages, rows % self.page, (pages >= 0) & (pages < self.num_pages)

    def raw(self, layer, kv, b, h, n):
        """Codes [n, d] and scales [n] of a unit's first rows, and whether their pages exist."""
        pages, slots, ok = self.places(b, torch.arange(n))
        pages = pages.clamp(0, self.num_pages - 1).cuda()
        slots = slots.cuda()
        pool = self.codes[layer][kv]
        return pool[pages, h, slots] if self.layout == "phsd" else pool[pages, slots, h], self.scales[layer][kv][pages, h, slots], ok.cuda()

    def rows(self, layer, kv, b, h, n):
        codes, scales, ok = self.raw(layer, kv, b, h, n)
        return values(codes, scales, self.kind), ok

    def put(self, layer, kv, b, h, rows, codes, scales):
        pages, slots, ok = self.places(b, rows)
        pages, slots, ok = pages[ok].cuda(), slots[ok].cuda(), ok.cuda()
        if self.layout == "phsd":
            self.codes[layer][kv][pages, h, slots] = codes[ok]
        else:
            self.codes[layer][kv][pages, slots, h] = codes[ok]
        self.scales[layer][kv][pages, h, slots] = scales[ok]

    def fill(self, gen, lengths):
        """Random rows of different sizes: codes as they come (none of them NaN), scales 2^-9 .. 2^-3."""
        for layer in range(len(self.codes)):
            for kv in range(2):
                for b in range(self.batch):
                    for h in range(self.hk):
                        n = int(lengths[b][h])
                        if self.kind == "e4m3":
                            codes = (torch.randn((n, self.d), generator=gen) * 60).to(torch.float8_e4m3fn).view(torch.uint8)
                        else:
                            codes = (torch.randn((n, self.d), generator=gen) * 40).round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
                        scales = torch.randint(118, 125, (n,), generator=gen).to(torch.uint8)
                        self.put(layer, kv, b, h, torch.arange(n), codes.cuda(), scales.cuda())


# ---- norms with rotary positions -----------------------------------------------------------------
def turned(x, weight, eps, offset, positions, axis, freqs, order, scale=1.0):
    """x [tokens, heads, d] at positions [axes, tokens]: the norm (eps None: without), then the rotation (freqs None: without); 64 bits, on the
    host.  Returns the result and the largest magnitude of every row in front of the rotation."""
    y = x.double().cpu()
    if eps is not None:
        y = y / torch.sqrt((y ** 2).mean(-1, keepdim=True) + eps)
        if weight is not None:
            y = y * (weight.double().cpu() + offset)
    big = y.abs().amax(-1, keepdim=True)
    z = y.clone()
    for i, f in enumerate(freqs or []):
        j, k = (i, i + len(freqs)) if order == "half" else (2 * i, 2 * i + 1)
        a = (positions[axis[i]].double().cpu() * f)[:, None]
        z[..., j] = (y[..., j] * torch.cos(a) - y[..., k] * torch.sin(a)) * scale
        z[..., k] = (y[..., k] * torch.cos(a) + y[..., j] * torch.sin(a)) * scale
    return z, big


def turned_bound(big, positions, d, scale, normed):
    """|error| in 32 bits, before the rounding to the type.  Norm: a sum of d squares (d u, halved by the root), division, root, reciprocal, two
    products and the weight's sum: (d / 2 + 8) u of the value.  Rotation as in rotary_bound, over the largest position."""
    own = (d / 2 + 8) * U if normed else 0.0
    far = positions.double().abs().amax(0).cpu()[:, None, None] if positions is not None else 0.0
    angle = 3.141592653589794 * (2.0 ** -30 + 2.0 ** -24) + far * 2.0 ** -50
    return 2 * big * max(1.0, abs(scale)) * (own + angle + 8 * U)


# ---- drafts --------------------------------------------------------------------------------------
def words_of(sees):
    """Truth values [m, m] -> int32 words [m, ceil(m / 32)]."""
    m = sees.shape[-1]
    out = torch.zeros((sees.shape[0], (m + 31) // 32), dtype=torch.int64)
    for j in range(m):
        out[:, j // 32] |= sees[:, j].long() << (j % 32)
    return torch.where(out >= 2 ** 31, out - 2 ** 32, out).to(torch.int32)


def tree_of(parents):
    """What the tokens of a tree see of it: [m, m]."""
    m = len(parents)
    sees = torch.zeros((m, m), dtype=torch.bool)
    for i, p in enumerate(parents):
        if 0 <= p < i:
            sees[i] = sees[p]
        sees[i, i] = True
    return sees


def attention_seen(q, k, v, seen):
    """ou.attention for any `seen` [R, n]; what a row does not see is taken out before any arithmetic."""
    R, n = seen.shape
    order_k, order_v = torch.nan_to_num(k.double(), 0, 0, 0), torch.nan_to_num(v.double(), 0, 0, 0)
    x = q.double() @ order_k.T / k.shape[1] ** 0.5
    x = torch.where(seen, x, torch.full_like(x, float("-inf")))
    lse = torch.logsumexp(x, 1)
    p = torch.where(seen, torch.exp(x - torch.where(torch.isfinite(lse), lse, torch.zeros_like(lse))[:, None]), torch.zeros_like(x))
    d = k.shape[1]
    e = (d + 4) * U * (torch.where(seen, q.double().abs() @ order_k.abs().T, torch.zeros_like(x)).amax(1) if n else torch.zeros(R, device=q.device)) / d ** 0.5
    return p @ order_v, lse, p, {"e": e, "factor": 2 * (e + (n + 32) * U), "abs": p @ order_v.abs(), "n": n}
