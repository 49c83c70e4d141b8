"""GPU tests of the operators around the selection: rotary positions, the prompt's attention, the paged cache in use.  Each is held to
a reference in 64 bits with the bounds of operators_util; what a call must leave alone is filled beforehand and looked at."""
import numpy as np
import pytest
import torch

import operators_util as ou
from paper_2503_17922_b200 import binding as wkv

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
INF, NAN = float("inf"), float("nan")


def gen(seed=1):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g).to(dtype).cuda()


# ---- whole prompts ---------------------------------------------------------------------------
def heads_tensor(g, dtype, B, h, n, d, layout, pad=0):
    """[B, h, n, d] stored in the given order, `pad` elements between rows."""
    if layout == "bhnd":
        return randn(g, B, h, n, d + pad, dtype=dtype)[..., :d]
    return randn(g, B, n, h, d + pad, dtype=dtype)[..., :d].transpose(1, 2)


class Prompt:
    def __init__(self, dtype, hq, hk, d, lens, layout="bhnd", alpha=4, seed=1, pad=0):
        g = gen(seed)
        self.lens, self.hq, self.hk, self.d, self.packed, self.alpha = lens, hq, hk, d, layout == "packed", alpha
        self.dtype = DT[dtype]
        n, B = max(lens), len(lens)
        self.cu = np.concatenate([[0], np.cumsum(lens)]).tolist()
        self.prob = wkv.Problem(dtype=dtype, batch=B, n_q_heads=hq, n_kv_heads=hk, head_dim=d, l_obs=alpha, window=8, task=0, top_p=0,
                                max_seqlen=n, budgets=[n] * B, cu_seqlens=self.cu if self.packed else None,
                                kv_layout="bnhd" if self.packed else layout)
        if self.packed:
            mk = lambda h, p=0: randn(g, sum(lens), h, d + p, dtype=self.dtype)[..., :d]
        else:
            mk = lambda h, p=0: heads_tensor(g, self.dtype, B, h, n, d, layout, p)
        self.q, self.k, self.v = mk(hq, pad), mk(hk), mk(hk)
        self.out = torch.full_like(self.q, 77.0) if pad == 0 else torch.full(self.q.shape, 77.0, dtype=self.dtype, device="cuda")
        self.lse = torch.full((B, hq, n), 77.0, device="cuda")
        self.lse_obs = torch.full((B, hq, alpha), 77.0, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def part(self, t, b, h):
        return t[self.cu[b]:self.cu[b + 1], h] if self.packed else t[b, h, : self.lens[b]]

    def run(self, **kw):
        wkv.wkv_attend_prompt(self.prob, self.q, self.k, self.v, self.out, self.lse, self.lse_obs, self.status, **kw)

    def check(self, rows=None):
        torch.cuda.synchronize()
        assert int(self.status) == 0
        G = self.hq // self.hk
        for b, n in enumerate(self.lens):
            limits = torch.arange(1, n + 1, device="cuda")
            at = limits - 1 if rows is None else torch.tensor([r for r in rows if r < n], device="cuda")
            for h in range(self.hq):
                ref, lse, _, bd = ou.attention(self.part(self.q, b, h)[at], self.part(self.k, b, h // G), self.part(self.v, b, h // G), limits[at])
                ou.assert_close(self.part(self.out, b, h)[at], ref, ou.output_bound(ref, bd, self.dtype), f"out {b} {h}")
                ou.assert_close(self.lse[b, h, at], lse, ou.lse_bound(lse, bd), f"lse {b} {h}")
                assert (self.lse[b, h, n:] == 77.0).all()
                for i in range(self.alpha):
                    r = n - self.alpha + i
                    want = self.lse[b, h, r] if r >= 0 else torch.tensor(-INF, device="cuda")
                    assert self.lse_obs[b, h, i] == want


PROMPTS = [
    # dtype, hq, hk, d, lens, layout, alpha, pad
    ("f32", 4, 2, 64, [1], "bhnd", 4, 0),
    ("f32", 4, 2, 64, [130, 130], "bnhd", 1, 0),
    ("f32", 3, 3, 20, [65, 65], "bhnd", 4, 4),
    ("f32", 6, 2, 128, [1, 3, 200, 64], "packed", 4, 0),
    ("f32", 2, 1, 256, [97], "bhnd", 8, 0),
    ("bf16", 4, 2, 64, [1], "bhnd", 4, 0),
    ("bf16", 4, 1, 128, [2, 2], "bnhd", 4, 0),
    ("bf16", 8, 8, 128, [129], "bhnd", 16, 8),
    ("bf16", 4, 2, 64, [257, 257], "bnhd", 8, 0),
    ("bf16", 6, 1, 128, [385], "bhnd", 4, 0),
    ("bf16", 12, 2, 128, [1, 300, 127, 2, 640], "packed", 16, 0),
    ("bf16", 5, 5, 64, [64, 1, 191], "packed", 2, 8),
    ("bf16", 7, 1, 80, [150], "bhnd", 4, 0),
    ("bf16", 16, 2, 96, [33, 140], "packed", 4, 0),
    ("bf16", 4, 2, 256, [131], "bhnd", 4, 0),
    ("bf16", 130, 1, 64, [40], "bhnd", 4, 0),
    ("bf16", 32, 8, 128, [1000], "bnhd", 32, 0),
]


@pytest.mark.parametrize("case", PROMPTS, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_prompt(case):
    dtype, hq, hk, d, lens, layout, alpha, pad = case
    p = Prompt(dtype, hq, hk, d, lens, layout, alpha, pad=pad)
    p.run()
    p.check()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_long_prompt_rows(dtype, d):
    p = Prompt(dtype, 4, 2, d, [5000, 2111], "packed", 8)
    p.run()
    p.check(rows=[0, 1, 127, 128, 500, 2047, 2048, 2110, 3333, 4863, 4864, 4998, 4999])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("bf16", 96), ("f32", 64)])
def test_prompt_rows_do_not_see_what_follows(dtype, d):
    """Infinities and NaN in keys and values behind a row, and in the sequence behind in a packed batch, do not reach it; those
    that a row does see reach it."""
    p = Prompt(dtype, 4, 2, d, [300, 200], "packed", 4)
    p.run()
    torch.cuda.synchronize()
    clean, clean_lse = p.out.clone(), p.lse.clone()
    at = 170
    p.v[at, 0, 3], p.v[at, 0, 5], p.v[at, 1, 7] = NAN, INF, -INF
    p.k[260, 0, :] = NAN
    p.v[300:, 0] = NAN
    p.k[300:, 1] = INF
    p.run()
    torch.cuda.synchronize()
    assert torch.equal(p.out[:at], clean[:at]) and torch.equal(p.lse[:1, :, :260], clean_lse[:1, :, :260])
    assert torch.isnan(p.out[at:300, :2, 3]).all()
    assert (p.out[at:260, :2, 5] == INF).all() and (p.out[at:300, 2:, 7] == -INF).all()
    others = [c for c in range(d) if c not in (3, 5)]
    assert torch.equal(p.out[at:260, :2][..., others], clean[at:260, :2][..., others])
    assert torch.isnan(p.out[260:300, :2]).all()
    assert torch.equal(p.out[260:300, 2:][..., :7], clean[260:300, 2:][..., :7])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_prompt_large_logits(dtype, d):
    """Logits of thousands: the running maximum moves by more than the exponent's range from tile to tile."""
    p = Prompt(dtype, 4, 2, d, [700], "bhnd", 4)
    p.q *= 32
    p.k *= torch.linspace(0.1, 4, 700, device="cuda").view(1, 1, -1, 1).to(p.dtype)
    p.run()
    p.check()


def test_prompt_is_the_same_alone_and_in_a_batch():
    a = Prompt("bf16", 8, 2, 128, [400, 150], "packed", 4)
    a.run()
    b = Prompt("bf16", 8, 2, 128, [150], "packed", 4)
    b.q, b.k, b.v = a.q[400:], a.k[400:], a.v[400:]
    b.run()
    torch.cuda.synchronize()
    assert torch.equal(a.out[400:], b.out)
    assert torch.equal(a.lse[1, :, :150], b.lse[0])


# ---- rotary positions ------------------------------------------------------------------------
ROPES = [
    # rot, order, scaling, factor, scale
    (64, "half", "none", 1.0, 1.0), (64, "interleaved", "linear", 8.0, 1.0), (128, "half", "bands", 8.0, 1.25),
    (128, "interleaved", "base", 4.0, 1.0), (6, "half", "none", 1.0, 1.0), (6, "interleaved", "bands", 4.0, 0.5), (36, "half", "base", 2.0, 1.0),
    (2, "half", "none", 1.0, 1.0),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rot,order,scaling,factor,scale", ROPES)
def test_rotate_prompt(dtype, rot, order, scaling, factor, scale):
    p = Prompt(dtype, 6, 2, 128, [1, 37, 80], "packed", 4)
    rope = wkv.Rope(rot, 500000.0, order=order, scaling=scaling, factor=factor, original_length=8192, scale=scale)
    freqs = ou.frequencies(rot, 500000.0, scaling, factor, 8192)
    at = torch.cat([torch.arange(n) for n in p.lens])
    far = torch.randint(0, 2 ** 31 - 1, (118,), generator=gen(5)).to(torch.int32)
    for positions in (None, far):
        q_out, k_out = torch.full_like(p.q, 77.0), torch.full_like(p.k, 77.0)
        wkv.wkv_rotate_prompt(p.prob, rope, p.q, p.k, q_out, k_out, positions=None if positions is None else positions.cuda())
        torch.cuda.synchronize()
        pos = at if positions is None else positions
        for got, x in ((q_out, p.q), (k_out, p.k)):
            ou.assert_close(got.cpu(), ou.rotated(x, pos, freqs, order, scale), ou.rotary_bound(x, pos, freqs, scale, p.dtype), "rotated")
            assert torch.equal(got[..., rot:], x[..., rot:])
    # in place, and one tensor alone
    q, k = p.q.clone(), p.k.clone()
    wkv.wkv_rotate_prompt(p.prob, rope, q, None, q, None, positions=far.cuda())
    wkv.wkv_rotate_prompt(p.prob, rope, None, k, None, k, positions=far.cuda())
    torch.cuda.synchronize()
    assert torch.equal(q, q_out) and torch.equal(k, k_out)


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_rotate_dense_layouts(layout):
    p = Prompt("bf16", 4, 2, 64, [50, 50], layout, 4, pad=8)
    rope = wkv.Rope(64, 10000.0)
    q_out = torch.empty_strided(p.q.shape, p.q.stride(), dtype=p.dtype, device="cuda")
    k_out = torch.empty_like(p.k)
    wkv.wkv_rotate_prompt(p.prob, rope, p.q, p.k, q_out, k_out)
    torch.cuda.synchronize()
    pos, freqs = torch.arange(50), ou.frequencies(64, 10000.0)
    for got, x in ((q_out, p.q), (k_out, p.k)):
        for b in range(2):
            ref = ou.rotated(x[b].transpose(0, 1), pos, freqs, "half")
            ou.assert_close(got[b].transpose(0, 1).cpu(), ref, ou.rotary_bound(x[b].transpose(0, 1), pos, freqs, 1.0, p.dtype), "rotated")


# ---- new tokens into the cache ---------------------------------------------------------------
def chunk_of(g, dtype, heads, d, news, packed):
    return randn(g, sum(news), heads, d, dtype=dtype) if packed else randn(g, len(news), heads, max(news), d, dtype=dtype)


def tokens_of(x, b, news, packed):
    """[m_b, heads, d] of sequence b."""
    if packed:
        lo = sum(news[:b])
        return x[lo:lo + news[b]]
    return x[b].transpose(0, 1)[: news[b]]


def paged(c, hq, max_new, cu=None):
    return wkv.PagedCache(dtype="f32" if c.dtype == torch.float32 else "bf16", batch=c.batch, n_q_heads=hq, n_kv_heads=c.hk, head_dim=c.d,
                          page_size=c.page, num_pages=c.num_pages, block_table=c.table, max_new=max_new, cu_new=cu, layout=c.layout)


def cu_of(news):
    return np.concatenate([[0], np.cumsum(news)]).tolist()


@pytest.mark.parametrize("dtype,d,page,layout,news,packed,rot,order", [
    ("bf16", 128, 16, "phsd", [1, 1, 1], False, 128, "half"),
    ("bf16", 64, 7, "pshd", [5, 0, 12], True, 64, "interleaved"),
    ("f32", 80, 24, "phsd", [3, 3, 3], False, 20, "half"),
    ("f32", 64, 1, "pshd", [2, 9, 1], True, 10, "interleaved"),
    ("bf16", 96, 64, "phsd", [70, 1, 33], True, 0, "half"),
])
def test_append(dtype, d, page, layout, news, packed, rot, order):
    g = gen(3)
    hk, hq = 2, 6
    max_pages = 100 // page + 3
    c = ou.Cache(g, DT[dtype], 3, hk, d, page, max_pages, layout, fill=9.0)
    lengths = torch.tensor([[0, 3], [17, 20], [c.cap - news[2] + 1, c.cap - 1]], dtype=torch.int32)      # the last sequence: rows that do not fit
    c.table[1, 20 // page] = -1 if page < 20 else c.num_pages                                   # rows without a page
    k, v, q = (chunk_of(g, DT[dtype], h, d, news, packed) for h in (hk, hk, hq))
    T = sum(news) if packed else 3 * max(news)
    positions = torch.randint(0, 1 << 20, (T,), generator=g).to(torch.int32)
    freqs = ou.frequencies(rot, 10000.0) if rot else []
    rope = wkv.Rope(rot, 10000.0, order=order) if rot else None
    cache = paged(c, hq, max(news), cu_of(news) if packed else None)
    q_out = torch.full_like(q, 77.0)
    lengths_out = torch.full((3, hk), -5, dtype=torch.int32, device="cuda")
    rp = torch.full((3, hk, c.cap), -5, dtype=torch.int32, device="cuda")
    rw = torch.full((3, hk, c.cap), -5.0, device="cuda")
    want_k, want_v = c.k[0].clone(), c.v[0].clone()
    pos_dev = positions.cuda() if packed else positions.view(3, -1).cuda()
    wkv.wkv_append_kv_paged(cache, k, v, lengths.cuda(), c.k[0], c.v[0], q=q, q_out=q_out, positions=pos_dev, rope=rope, lengths_out=lengths_out,
                            row_positions=rp, row_weights=rw)
    torch.cuda.synchronize()
    pos_tokens = positions[:, None].expand(-1, 1) if packed else positions.view(3, 1, -1).transpose(1, 2).reshape(-1, 1)
    first = 0
    for b, m in enumerate(news):
        pos = positions[first:first + m] if packed else positions.view(3, -1)[b, :m]
        first += m
        bound = lambda x: ou.rotary_bound(x, pos, freqs, 1.0, DT[dtype]) if rot else torch.zeros(1, dtype=torch.float64)
        qb = tokens_of(q, b, news, packed)
        if m:
            ou.assert_close(tokens_of(q_out, b, news, packed).cpu(), ou.rotated(qb, pos, freqs, order), bound(qb), "q")
        for h in range(hk):
            n = int(lengths[b, h])
            assert int(lengths_out[b, h]) == min(n + m, c.cap)
            kept = min(m, c.cap - n)
            assert torch.equal(rp[b, h, n:n + kept].cpu(), pos[:kept]) and (rw[b, h, n:n + kept] == 0).all()
            assert (rp[b, h, :n] == -5).all() and (rp[b, h, n + kept:] == -5).all() and (rw[b, h, :n] == -5).all()
            kb, vb = tokens_of(k, b, news, packed)[:, h], tokens_of(v, b, news, packed)[:, h]
            for i in range(kept):
                if not 0 <= int(c.table[b, (n + i) // page]) < c.num_pages:
                    continue
                slot = c.slot(c.k[0], b, h, n + i)
                ou.assert_close(slot.cpu().view(1, 1, -1), ou.rotated(kb[i].view(1, 1, -1), pos[i:i + 1], freqs, order),
                                ou.rotary_bound(kb[i].view(1, 1, -1), pos[i:i + 1], freqs, 1.0, DT[dtype]) if rot else torch.zeros(1, dtype=torch.float64), "k")
                assert torch.equal(c.slot(c.v[0], b, h, n + i), vb[i])
                c.slot(want_k, b, h, n + i).copy_(slot)
                c.slot(want_v, b, h, n + i).copy_(vb[i])
    assert torch.equal(c.k[0], want_k) and torch.equal(c.v[0], want_v)      # nothing else was written


# ---- new tokens over the cache ------------------------------------------------------------------
class Attend:
    def __init__(self, dtype, hq, hk, d, page, layout, lengths, news, packed, seed=1, max_pages=None, scale=1.0, max_new=None):
        g = gen(seed)
        self.dtype = DT[dtype]
        B = len(lengths)
        self.lengths = torch.tensor(lengths, dtype=torch.int32)
        self.news, self.packed, self.hq, self.hk = news, packed, hq, hk
        most = int(self.lengths.max())
        self.c = ou.Cache(g, self.dtype, B, hk, d, page, max_pages or max(1, -(-most // page)) + 1, layout)
        self.c.fill(g, lengths, scale)
        self.q = chunk_of(g, self.dtype, hq, d, news, packed)
        self.out = torch.full_like(self.q, 77.0)
        self.max_new = max_new or max(max(news), 1)
        self.cache = paged(self.c, hq, self.max_new, cu_of(news) if packed else None)
        self.ws = self.cache.alloc_workspace()
        self.lse = torch.full((B, hq, self.max_new), 77.0, device="cuda")
        self.w_in = torch.rand((B, hk, self.c.cap), generator=g).cuda()
        self.w_out = torch.full((B, hk, self.c.cap), 77.0, device="cuda")

    def run(self, weights=True, lse=True, w_in=True, **kw):
        wkv.wkv_attend_paged(self.cache, self.q, self.c.k[0], self.c.v[0], self.lengths.cuda(), self.out, self.ws,
                             lse=self.lse if lse else None, weights_in=self.w_in if weights and w_in else None,
                             weights_out=self.w_out if weights else None, **kw)

    def check(self, weights=True, lse=True, w_in=True):
        torch.cuda.synchronize()
        assert wkv.device_status(self.ws) == 0
        G = self.hq // self.hk
        for b, m in enumerate(self.news):
            out = tokens_of(self.out, b, self.news, self.packed)
            q = tokens_of(self.q, b, self.news, self.packed)
            if not self.packed and m < self.q.shape[2]:
                assert (self.out[b, :, m:] == 77.0).all()
            for h in range(self.hk):
                n = min(max(int(self.lengths[b, h]), 0), self.c.cap)
                k, ok = self.c.rows(self.c.k[0], b, h, n)
                v, _ = self.c.rows(self.c.v[0], b, h, n)
                limits = torch.arange(n - m + 1, n + 1, device="cuda").repeat(G)
                qs = q[:, h * G:(h + 1) * G].transpose(0, 1).reshape(G * m, q.shape[-1])
                ref, lses, p, bd = ou.attention(qs, k, v, limits, ok)
                got = out[:, h * G:(h + 1) * G].transpose(0, 1).reshape(G * m, q.shape[-1])
                if m:
                    ou.assert_close(got, ref, ou.output_bound(ref, bd, self.dtype), f"out {b} {h}")
                    gl = self.lse[b, h * G:(h + 1) * G]
                    if lse:
                        ou.assert_close(gl[:, :m].reshape(-1), lses, ou.lse_bound(lses, bd), f"lse {b} {h}")
                        assert (gl[:, m:] == 77.0).all()
                if weights:
                    base = self.w_in[b, h, :n].double() if w_in else torch.zeros(n, dtype=torch.float64, device="cuda")
                    want = base + p.sum(0)
                    bound = (bd["factor"][:, None] * p).sum(0) + G * m * ou.U * p.sum(0) + 2 * ou.U * want + 1e-37 if m else torch.zeros_like(want)
                    ou.assert_close(self.w_out[b, h, :n], want, bound, f"weights {b} {h}")
                    assert (self.w_out[b, h, n:] == 77.0).all()


ATTENDS = [
    # dtype, hq, hk, d, page, layout, lengths, news, packed
    ("f32", 4, 2, 64, 16, "phsd", [[1, 1]], [1], False),
    ("f32", 4, 2, 64, 24, "pshd", [[700, 699], [1, 0], [65, 64]], [1, 1, 1], False),
    ("f32", 6, 2, 80, 7, "phsd", [[300, 290], [5, 7]], [5, 7], True),
    ("f32", 2, 1, 256, 32, "phsd", [[333]], [40], False),
    ("bf16", 8, 2, 128, 16, "phsd", [[992, 990]], [1], False),
    ("bf16", 32, 8, 128, 64, "pshd", [[2000 - h for h in range(8)], [1] * 8, [0] * 8, [129 + h for h in range(8)]], [1] * 4, False),
    ("bf16", 4, 1, 64, 8, "phsd", [[4097], [15]], [1, 1], False),
    ("bf16", 12, 2, 128, 24, "pshd", [[517, 515], [64, 65]], [2, 2], False),
    ("bf16", 8, 2, 96, 13, "phsd", [[260, 255], [31, 33]], [3, 0], True),
    ("bf16", 7, 1, 80, 1, "phsd", [[77]], [2], False),
    ("bf16", 4, 2, 256, 16, "phsd", [[300, 301]], [1], False),
    ("bf16", 16, 1, 128, 32, "phsd", [[1025]], [1], False),
    ("bf16", 40, 1, 64, 32, "phsd", [[130]], [1], False),
    ("bf16", 8, 2, 128, 16, "phsd", [[600, 598], [300, 300], [1, 2]], [100, 300, 1], True),
    ("bf16", 8, 2, 128, 128, "pshd", [[1000, 998], [333, 330]], [200, 200], False),
    ("bf16", 12, 2, 64, 32, "phsd", [[700, 698], [5, 5], [260, 260]], [150, 0, 260], True),
    ("bf16", 4, 4, 128, 64, "pshd", [[513] * 4], [129], False),
    ("bf16", 8, 2, 128, 24, "phsd", [[401, 400]], [130], False),
    ("bf16", 6, 1, 80, 16, "phsd", [[260]], [90], False),
    ("bf16", 4, 1, 128, 256, "phsd", [[900]], [70], False),
    ("bf16", 8, 2, 128, 16, "phsd", [[3, 200]], [64], False),            # more new tokens than rows
    ("bf16", 8, 2, 128, 16, "phsd", [[3, 0]], [5], False),
]


@pytest.mark.parametrize("case", ATTENDS, ids=lambda c: "-".join(map(str, c)).replace(" ", "")[:70])
def test_attend(case):
    a = Attend(*case)
    a.run()
    a.check()


@pytest.mark.parametrize("case", [ATTENDS[1], ATTENDS[4], ATTENDS[13]], ids=["f32", "one", "chunk"])
@pytest.mark.parametrize("what", [dict(weights=False), dict(weights=False, lse=False), dict(lse=False), dict(w_in=False)])
def test_attend_optional_parts(case, what):
    a = Attend(*case)
    a.run(**what)
    a.check(**what)
    if what.get("lse") is False:
        assert (a.lse == 77.0).all()


@pytest.mark.parametrize("case", [ATTENDS[1], ATTENDS[5], ATTENDS[14]], ids=["f32", "one", "chunk"])
def test_weights_add_up_in_place(case):
    a = Attend(*case)
    a.run()
    torch.cuda.synchronize()
    w = a.w_in.clone()
    wkv.wkv_attend_paged(a.cache, a.q, a.c.k[0], a.c.v[0], a.lengths.cuda(), a.out, a.ws, weights_in=w, weights_out=w)
    torch.cuda.synchronize()
    n = a.lengths.cuda().unsqueeze(-1)
    there = torch.arange(a.c.cap, device="cuda") < n
    assert torch.equal(w, torch.where(there, a.w_out, a.w_in))


@pytest.mark.parametrize("dtype,d,page,layout,new", [("f32", 64, 16, "phsd", 1), ("bf16", 128, 16, "phsd", 1), ("bf16", 128, 16, "pshd", 140),
                                                     ("bf16", 64, 128, "phsd", 70), ("bf16", 80, 8, "phsd", 40), ("bf16", 128, 7, "phsd", 90)])
def test_rows_without_a_page_are_not_attended(dtype, d, page, layout, new):
    a = Attend(dtype, 8, 2, d, page, layout, [[500, 499], [400, 400]], [new, new], False)
    a.c.table[0, 1] = -1
    a.c.table[1, 0] = a.c.num_pages
    a.c.table[1, 399 // page] = 2 ** 31 - 1
    a.run()
    a.check()
    a.c.table[:] = -3
    a.run()
    a.check()
    assert (a.out == 0).all() and (a.lse == -INF).all()


@pytest.mark.parametrize("dtype,d,page,new", [("f32", 64, 16, 6), ("bf16", 128, 16, 4), ("bf16", 128, 16, 150), ("bf16", 64, 128, 150), ("bf16", 96, 24, 50)])
def test_queries_do_not_see_later_rows(dtype, d, page, new):
    """NaN and infinities in the chunk's own later rows and behind the cache's end (every unused row is NaN) do not reach a query."""
    a = Attend(dtype, 4, 2, d, page, "phsd", [[400, 399]], [new], False)
    a.run()
    torch.cuda.synchronize()
    clean, lse = a.out.clone(), a.lse.clone()
    at = [400 - new // 2, 399 - new // 2]            # rows of the two heads
    for h in range(2):
        a.c.slot(a.c.v[0], 0, h, at[h])[1] = NAN
        a.c.slot(a.c.v[0], 0, h, at[h])[2] = INF
    i = new - new // 2                               # the first query that sees them
    a.run()
    torch.cuda.synchronize()
    assert torch.equal(a.out[:, :, :i], clean[:, :, :i]) and torch.equal(a.lse, lse)
    assert torch.isnan(a.out[:, :, i:, 1]).all() and (a.out[:, :, i:, 2] == INF).all()
    assert torch.equal(a.out[:, :, i:, 3:], clean[:, :, i:, 3:])


def test_lengths_beyond_the_table_and_below_zero():
    a = Attend("bf16", 4, 2, 64, 16, "phsd", [[80, 80]], [1], False, max_pages=5)
    a.lengths[:] = torch.tensor([[1000, -7]])
    a.run()
    a.check()


def test_a_stale_device_copy_stays_inside():
    """cu_new on the device that says more than the host copy did: nothing outside the arrays sized by the host copy."""
    a = Attend("bf16", 4, 2, 64, 16, "phsd", [[80, 80], [60, 60]], [3, 4], True)
    guard = torch.full((7 + 16, 4, 64), 77.0, dtype=torch.bfloat16, device="cuda")
    a.out = guard[:7]
    a.cache.cu_dev.copy_(torch.tensor([0, 6, 1000], dtype=torch.int32))
    a.run(weights=False)
    torch.cuda.synchronize()
    assert (guard[7:] == 77.0).all()


# ---- eviction -----------------------------------------------------------------------------------
def evict_reference(w, pos, n, keep, recent):
    """Rows kept in their new places: list of source rows, by the order in the header."""
    newest = max(pos[:n], default=0)
    key = lambda r: (not pos[r] > newest - recent, -(w[r] if w[r] == w[r] else -INF), w[r] != w[r], r)
    stays = set(sorted(range(n), key=key)[:keep])
    fill = iter(r for r in range(keep, n) if r in stays)
    return [r if r in stays else next(fill) for r in range(keep)]


class Evict:
    def __init__(self, dtype, d, page, layout, lengths, layers, seed=1, max_pages=None):
        g = gen(seed)
        self.lengths = torch.tensor(lengths, dtype=torch.int32)
        B, hk = self.lengths.shape
        most = int(self.lengths.max())
        self.c = ou.Cache(g, DT[dtype], B, hk, d, page, max_pages or max(1, -(-most // page)) + 1, layout, layers, fill=5.0)
        for pool in self.c.k + self.c.v:
            pool.copy_(torch.randn(pool.shape, generator=g).to(pool.dtype))
        self.w = torch.exp(2 * torch.randn((B, hk, self.c.cap), generator=g))
        self.pos = torch.argsort(torch.rand((B, hk, self.c.cap), generator=g), -1).to(torch.int32)
        self.cache = paged(self.c, hk, 1)
        self.ws = self.cache.alloc_workspace()

    def run_and_check(self, budget, recent, in_place=False, budgets=None, v=True):
        c, B, hk = self.c, *self.lengths.shape
        before_k, before_v = [x.clone() for x in c.k], [x.clone() for x in c.v]
        w, pos, n_in = self.w.cuda(), self.pos.cuda(), self.lengths.cuda()
        w_out, pos_out, n_out = (w, pos, n_in) if in_place else (torch.full_like(w, 77.0), torch.full_like(pos, -7), torch.full_like(n_in, -7))
        bud = None if budgets is None else torch.tensor(budgets, dtype=torch.int32, device="cuda")
        wkv.wkv_evict_kv_paged(self.cache, c.k, c.v if v else None, w, pos, n_in, budget, recent, w_out, pos_out, n_out, self.ws, budgets=bud)
        torch.cuda.synchronize()
        want_k, want_v = [x.clone() for x in before_k], [x.clone() for x in before_v]
        for b in range(B):
            for h in range(hk):
                n = min(max(int(self.lengths[b, h]), 0), c.cap)
                keep = min(n, max(budget if budgets is None else budgets[b], 0))
                src = evict_reference(self.w[b, h].tolist(), self.pos[b, h].tolist(), n, keep, recent)
                assert int(n_out[b, h]) == keep
                at = torch.tensor(src, dtype=torch.long)
                assert torch.equal(w_out[b, h, :keep].cpu().view(torch.int32), self.w[b, h][at].view(torch.int32))
                assert torch.equal(pos_out[b, h, :keep].cpu(), self.pos[b, h][at])
                if in_place:
                    assert torch.equal(w[b, h, keep:].cpu().view(torch.int32), self.w[b, h, keep:].view(torch.int32))
                else:
                    assert (w_out[b, h, keep:] == 77.0).all() and (pos_out[b, h, keep:] == -7).all()
                for r, s in enumerate(src):
                    if r == s or not all(0 <= int(c.table[b, x // c.page]) < c.num_pages for x in (r, s)):
                        continue
                    for before, want in list(zip(before_k, want_k)) + (list(zip(before_v, want_v)) if v else []):
                        c.slot(want, b, h, r).copy_(c.slot(before, b, h, s))
        for got, want in zip(c.k + c.v, want_k + want_v):
            assert torch.equal(got, want)


EVICTS = [
    # dtype, d, page, layout, lengths, layers, budget, recent
    ("bf16", 128, 16, "phsd", [[100, 99]], 2, 90, 8),
    ("bf16", 64, 7, "pshd", [[200, 30], [0, 1], [64, 65]], 1, 64, 0),
    ("f32", 20, 24, "phsd", [[300, 280]], 3, 17, 5),
    ("f32", 64, 64, "pshd", [[50, 50]], 1, 0, 5),
    ("bf16", 256, 32, "phsd", [[130, 131]], 1, 129, 200),
    ("bf16", 96, 1, "phsd", [[33, 2]], 1, 1, 1),
    ("bf16", 64, 16, "phsd", [[2500, 1024], [1025, 2048]], 1, 1000, 30),
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", EVICTS, ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_evict(case, in_place):
    dtype, d, page, layout, lengths, layers, budget, recent = case
    Evict(dtype, d, page, layout, lengths, layers).run_and_check(budget, recent, in_place)


def test_evict_twice_gives_the_same():
    """Without in-place state a repeated call does the same again: what moved is still behind the kept rows."""
    e = Evict("bf16", 64, 16, "phsd", [[300, 200]], 2)
    e.run_and_check(150, 10)
    e.run_and_check(150, 10)


def test_evict_ties_zeros_nan_and_infinities():
    e = Evict("bf16", 64, 16, "phsd", [[200, 150]], 1)
    e.w[0, 0] = 1.0                                          # all equal: the lowest rows stay
    e.w[0, 1, ::3] = 0.0
    e.w[0, 1, 1::6] = -0.0
    e.w[0, 1, 5], e.w[0, 1, 6], e.w[0, 1, 7], e.w[0, 1, 8] = NAN, INF, -INF, -NAN
    e.run_and_check(60, 4)
    e.w[:] = NAN
    e.run_and_check(60, 0)


def test_evict_budgets_of_their_own_positions_and_missing_pages():
    e = Evict("bf16", 64, 16, "phsd", [[200, 150], [90, 80], [20, 300]], 2)
    e.pos[0] = 7                                             # every row recent: the weights decide
    e.pos[1] = -2 ** 31
    e.pos[2, 1, 100] = 2 ** 31 - 1
    e.c.table[2, 3] = -1
    e.c.table[0, 11] = 2 ** 31 - 1
    e.run_and_check(123, 3, budgets=[50, -4, 100])
    e.run_and_check(40, 2 ** 31 - 1)


def test_evict_keys_only_and_lengths_out_of_range():
    e = Evict("bf16", 64, 16, "phsd", [[150, 80]], 1, max_pages=6)
    e.lengths[:] = torch.tensor([[1000, -3]])
    e.run_and_check(50, 3, v=False)


def test_evict_a_list_beyond_shared_memory():
    e = Evict("bf16", 8, 64, "phsd", [[60000]], 1)
    c = e.c
    w, pos, n = e.w.cuda(), e.pos.cuda(), e.lengths.cuda()
    src = evict_reference(e.w[0, 0].tolist(), e.pos[0, 0].tolist(), 60000, 30001, 100)
    before = c.rows(c.k[0], 0, 0, 60000)[0].clone()
    wkv.wkv_evict_kv_paged(e.cache, c.k, c.v, w, pos, n, 30001, 100, w, pos, n, e.ws)
    torch.cuda.synchronize()
    assert int(n) == 30001
    assert torch.equal(w[0, 0, :30001].cpu(), e.w[0, 0][torch.tensor(src)])
    assert torch.equal(c.rows(c.k[0], 0, 0, 30001)[0], before[torch.tensor(src).cuda()])
    assert torch.equal(c.rows(c.k[0], 0, 0, 60000)[0][30001:], before[30001:])


# ---- a run of them, as an engine uses them ---------------------------------------------------------
@pytest.mark.parametrize("dtype,hq,hk,d,page", [("bf16", 8, 2, 128, 16), ("f32", 4, 2, 64, 24), ("bf16", 12, 2, 64, 32)])
def test_prompt_to_decode(dtype, hq, hk, d, page):
    """Rotate and attend a prompt, select its windows with the attention's own normalisers, gather into pages, seed the rows'
    state, then decode tokens with eviction; the cache is held against a plain model of it after every step."""
    n, alpha, window, budget = 600, 16, 8, 128
    g = gen(11)
    p = Prompt(dtype, hq, hk, d, [n], "bhnd", alpha)
    p.prob = wkv.Problem(dtype=dtype, batch=1, n_q_heads=hq, n_kv_heads=hk, head_dim=d, l_obs=alpha, window=window, task=0, top_p=0,
                         max_seqlen=n, budgets=[budget], kv_layout="bhnd")
    prob, rope = p.prob, wkv.Rope(d, 10000.0)
    wkv.wkv_rotate_prompt(prob, rope, p.q, p.k, p.q, p.k)
    p.run()
    p.check(rows=[0, 1, 300, n - 1])
    # the selection with these normalisers is the selection with the framework's own
    q_obs = p.q[:, :, n - alpha:].contiguous()
    work, o = prob.alloc_workspace(), prob.alloc_outputs(1)
    tokens = torch.zeros((1, hk, prob.nr_max), device="cuda")
    wkv.wkv_select_leader_windows(prob, q_obs, p.k, o["window_scores"], o["window_idx"], o["kept_len"], work)
    own_idx = o["window_idx"].clone()
    wkv.wkv_score_windows_lse(prob, q_obs, p.k, p.lse_obs, o["window_scores"], tokens, work)
    wkv.wkv_select_topk_windows(prob, o["window_scores"], o["window_idx"], o["kept_len"])
    torch.cuda.synchronize()
    assert torch.equal(own_idx, o["window_idx"])
    c = ou.Cache(g, DT[dtype], 1, hk, d, page, (budget + 40) // page + 1, "phsd", fill=0.0)
    cache = paged(c, hq, 1)
    wkv.wkv_gather_kv_paged(prob, [p.k], [p.v], o["window_idx"], c.k, c.v, c.table, page, c.num_pages, hk * page * d, page * d, d)
    positions = torch.full((1, hk, c.cap), -1, dtype=torch.int32, device="cuda")
    weights = torch.full((1, hk, c.cap), -1.0, device="cuda")
    wkv.wkv_seed_rows(prob, o["window_idx"], tokens, positions, weights)
    torch.cuda.synchronize()
    model = []
    for h in range(hk):
        idx = o["window_idx"][0, h].tolist()
        rows = [w * window + x for w in idx if w >= 0 for x in range(window) if w * window + x < n - alpha] + list(range(n - alpha, n))
        assert len(rows) == int(o["kept_len"][0, h])
        m = len(rows)
        assert positions[0, h, :m].tolist() == rows and (positions[0, h, m:] == -1).all()
        want = [tokens[0, h, r].item() if r < n - alpha else 0.0 for r in rows]
        assert weights[0, h, :m].tolist() == want and (weights[0, h, m:] == -1).all()
        assert torch.equal(c.rows(c.k[0], 0, h, m)[0], p.k[0, h][torch.tensor(rows).cuda()])
        model.append(rows)
    lengths, ws = o["kept_len"].clone(), cache.alloc_workspace()
    grown, out = torch.zeros_like(lengths), torch.zeros((1, hq, 1, d), dtype=DT[dtype], device="cuda")
    freqs = ou.frequencies(d, 10000.0)
    for step in range(30):
        q, k, v = (randn(g, 1, h, 1, d, dtype=DT[dtype]) for h in (hq, hk, hk))
        pos = torch.tensor([[n + step]], dtype=torch.int32, device="cuda")
        wkv.wkv_append_kv_paged(cache, k, v, lengths, c.k[0], c.v[0], q=q, q_out=q, positions=pos, rope=rope, lengths_out=grown,
                                row_positions=positions, row_weights=weights)
        wkv.wkv_attend_paged(cache, q, c.k[0], c.v[0], grown, out, ws, weights_in=weights, weights_out=weights)
        lengths.copy_(grown)
        if step % 10 == 9:
            held = [weights[0, h].tolist() for h in range(hk)]
            wkv.wkv_evict_kv_paged(cache, c.k, c.v, weights, positions, lengths, 100, 20, weights, positions, lengths, ws)
        torch.cuda.synchronize()
        for h in range(hk):
            model[h].append(n + step)
            if step % 10 == 9:
                src = evict_reference(held[h], model[h], len(model[h]), 100, 20)
                model[h] = [model[h][r] for r in src]
            m = len(model[h])
            assert int(lengths[0, h]) == m and positions[0, h, :m].tolist() == model[h]
        if step % 10 != 9:
            G = hq // hk
            for h in range(hk):
                kk, vv = c.rows(c.k[0], 0, h, len(model[h]))[0], c.rows(c.v[0], 0, h, len(model[h]))[0]
                ref, _, _, bd = ou.attention(q[0, h * G:(h + 1) * G, 0], kk, vv, torch.full((G,), len(model[h]), device="cuda"))
                ou.assert_close(out[0, h * G:(h + 1) * G, 0], ref, ou.output_bound(ref, bd, DT[dtype]), f"step {step} head {h}")
    assert wkv.device_status(ws) == 0


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 130), ("f32", 3)])
def test_decode_step_captured_and_replayed(dtype, new):
    """A step of append, attend and evict in a CUDA graph, on another stream, with lengths that change between replays."""
    a = Attend(dtype, 8, 2, 64, 16, "phsd", [[300, 299], [200, 200]], [new, new], False, max_pages=40)
    c = a.c
    g = gen(4)
    k, v = (chunk_of(g, a.dtype, 2, 64, [new, new], False) for _ in range(2))
    pos = torch.arange(new, dtype=torch.int32, device="cuda").expand(2, -1).contiguous() + 400
    rope = wkv.Rope(64, 10000.0)
    state = {"w": a.w_in.clone(), "p": torch.arange(c.cap, dtype=torch.int32, device="cuda").expand(2, 2, -1).contiguous(),
             "n": a.lengths.cuda() - new, "n1": torch.zeros((2, 2), dtype=torch.int32, device="cuda")}
    start = {x: y.clone() for x, y in state.items()}
    pools = [c.k[0].clone(), c.v[0].clone()]
    q_out = torch.empty_like(a.q)

    def step():
        wkv.wkv_append_kv_paged(a.cache, k, v, state["n"], c.k[0], c.v[0], q=a.q, q_out=q_out, positions=pos, rope=rope, lengths_out=state["n1"],
                                row_positions=state["p"], row_weights=state["w"])
        wkv.wkv_attend_paged(a.cache, q_out, c.k[0], c.v[0], state["n1"], a.out, a.ws, weights_in=state["w"], weights_out=state["w"])
        wkv.wkv_evict_kv_paged(a.cache, c.k, c.v, state["w"], state["p"], state["n1"], 280, 10, state["w"], state["p"], state["n"], a.ws)

    results = []
    for replayed in (False, True):
        for x in state:
            state[x].copy_(start[x])
        c.k[0].copy_(pools[0])
        c.v[0].copy_(pools[1])
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            if replayed:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    step()
                for _ in range(3):
                    graph.replay()
            else:
                for _ in range(3):
                    step()
        torch.cuda.synchronize()
        results.append([a.out.clone()] + [state[x].clone() for x in ("w", "p", "n")] + [c.k[0].clone(), c.v[0].clone()])
    for x, y in zip(*results):
        assert torch.equal(x.view(torch.uint8) if x.dtype != torch.int32 else x, y.view(torch.uint8) if y.dtype != torch.int32 else y)
    assert wkv.device_status(a.ws) == 0


@pytest.mark.parametrize("case", [
    # few items over long caches: blocks share items and join their pieces
    ("bf16", 8, 2, 128, 64, "pshd", [[5000, 4990], [2100, 700], [1, 0], [3, 2600]], [40, 300, 0, 200], True),
    ("bf16", 4, 1, 64, 128, "phsd", [[9000]], [33], False),
    ("bf16", 12, 1, 128, 16, "phsd", [[2500], [4100]], [500, 7], True),
    ("bf16", 64, 1, 128, 32, "phsd", [[3333]], [1], False),
], ids=["ragged", "one", "g6", "token"])
def test_attend_shared_work(case):
    a = Attend(*case)
    assert a.c.cap >= 2048
    a.run()
    a.check()


def test_attend_shared_work_with_infinities_and_missing_pages():
    a = Attend("bf16", 8, 2, 128, 64, "phsd", [[4000, 3990]], [200], False)
    a.run(weights=False)
    torch.cuda.synchronize()
    clean = a.out.clone()
    a.c.slot(a.c.v[0], 0, 0, 3900)[3] = NAN
    a.c.slot(a.c.v[0], 0, 1, 3890)[5] = INF
    a.run(weights=False)
    torch.cuda.synchronize()
    assert torch.equal(a.out[:, :4, :100], clean[:, :4, :100]) and torch.isnan(a.out[:, :4, 100:, 3]).all()
    assert torch.equal(a.out[:, 4:, :100], clean[:, 4:, :100]) and (a.out[:, 4:, 100:, 5] == INF).all()
    assert torch.equal(a.out[:, :4, :, 4:], clean[:, :4, :, 4:])
    a.c.slot(a.c.v[0], 0, 0, 3900)[3] = 0.5
    a.c.slot(a.c.v[0], 0, 1, 3890)[5] = 0.5
    a.c.table[0, 20:40] = -1
    a.run()
    a.check()


@pytest.mark.parametrize("case", [
    # head dimensions that are not a whole number of the tensor cores' steps, or of 64 columns
    ("bf16", 4, 2, 8, [140], "bhnd", 4, 0),
    ("bf16", 6, 3, 24, [333, 128], "packed", 4, 0),
    ("bf16", 8, 2, 40, [129, 129], "bnhd", 8, 8),
    ("bf16", 12, 2, 72, [513], "bhnd", 4, 0),
    ("bf16", 8, 1, 80, [1, 400, 260], "packed", 16, 8),
    ("bf16", 6, 2, 96, [257, 257], "bnhd", 8, 0),
    ("bf16", 3, 3, 104, [300], "bhnd", 4, 0),
    ("bf16", 5, 1, 120, [200, 31], "packed", 4, 8),
], ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_prompt_head_dimensions(case):
    dtype, hq, hk, d, lens, layout, alpha, pad = case
    p = Prompt(dtype, hq, hk, d, lens, layout, alpha, pad=pad)
    p.run()
    p.check()


def test_head_dimension_80_does_not_see_what_follows():
    p = Prompt("bf16", 4, 2, 80, [300, 200], "packed", 4)
    p.run()
    torch.cuda.synchronize()
    clean = p.out.clone()
    at = 170
    p.v[at, 0, 3], p.v[at, 0, 70], p.v[at, 1, 79] = NAN, INF, -INF
    p.k[260, 0, :] = NAN
    p.v[300:, 0] = NAN
    p.run()
    torch.cuda.synchronize()
    assert torch.equal(p.out[:at], clean[:at]) and torch.isnan(p.out[at:300, :2, 3]).all()
    assert (p.out[at:260, :2, 70] == INF).all() and (p.out[at:300, 2:, 79] == -INF).all()
    assert torch.equal(p.out[at:300, 2:, :79], clean[at:300, 2:, :79])


@pytest.mark.parametrize("case", [
    # pages that are no part of a key tile; shared work with such pages and head dimensions; weights over more than one block of keys
    ("bf16", 8, 2, 128, 40, "phsd", [[1000, 998], [333, 330]], [200, 33], True),
    ("bf16", 8, 2, 64, 48, "pshd", [[700, 650], [5, 5]], [150, 2], True),
    ("bf16", 4, 1, 96, 192, "phsd", [[900]], [70], False),
    ("bf16", 12, 2, 80, 24, "pshd", [[2600, 2500], [60, 61], [2333, 0]], [140, 60, 333], True),
    ("bf16", 4, 2, 40, 8, "phsd", [[2900, 2890]], [300], False),
    ("bf16", 9, 3, 128, 200, "phsd", [[513] * 3], [129], False),
    ("bf16", 8, 1, 256, 16, "phsd", [[700]], [90], False),
    ("bf16", 17, 1, 64, 12, "phsd", [[640], [63]], [2, 1], True),
], ids=lambda c: "-".join(map(str, c)).replace(" ", "")[:70])
def test_attend_pages_and_head_dimensions(case):
    a = Attend(*case)
    a.run()
    a.check()
    a.c.table[0, 1] = -1
    a.run()
    a.check()


def test_weights_of_a_chunk_beside_keys_that_nobody_sees():
    """Rows behind the last query's position (more rows than the chunk accounts for cannot be: the last query sees the last row), and
    infinities in keys that only some queries see: the others' weights stay as they are."""
    a = Attend("bf16", 8, 2, 128, 24, "phsd", [[600, 590]], [100], False)
    a.run()
    torch.cuda.synchronize()
    clean = a.w_out.clone()
    a.c.slot(a.c.k[0], 0, 0, 599)[:] = NAN                       # seen by the last query alone
    a.run()
    torch.cuda.synchronize()
    assert torch.isnan(a.w_out[0, 0, :600]).all() and torch.equal(a.w_out[0, 1], clean[0, 1])
    assert torch.isnan(a.out[0, :4, 99]).all() and torch.isfinite(a.out[0, :4, :99]).all()


@pytest.mark.parametrize("case", [
    # fp32: keys split over two, four and eight blocks of a cluster, 16 to 128 rows a block, sequences shorter than the splits
    ("f32", 4, 2, 64, [1024], "bhnd", 8, 0),
    ("f32", 4, 2, 128, [1500], "bnhd", 8, 4),
    ("f32", 2, 2, 80, [700, 3, 64, 1], "packed", 4, 0),
    ("f32", 8, 1, 96, [2100], "bhnd", 4, 0),
    ("f32", 16, 16, 128, [1100], "bnhd", 1, 0),
    ("f32", 1, 1, 256, [500], "bhnd", 4, 0),
    ("f32", 7, 1, 8, [333], "bhnd", 4, 0),
], ids=lambda c: "-".join(map(str, c)).replace(" ", ""))
def test_prompt_fp32_splits(case):
    dtype, hq, hk, d, lens, layout, alpha, pad = case
    p = Prompt(dtype, hq, hk, d, lens, layout, alpha, pad=pad)
    p.run()
    p.check(rows=None if max(lens) < 600 else [0, 1, 63, 64, 127, 128, 600, 699, 1023, 1024, 1099, 1499, 2098, 2099])


def test_fp32_splits_do_not_see_what_follows():
    p = Prompt("f32", 4, 2, 64, [900], "bhnd", 4)
    p.run()
    torch.cuda.synchronize()
    clean = p.out.clone()
    p.v[0, 0, 500, 3], p.v[0, 0, 500, 5], p.k[0, 1, 700] = NAN, INF, NAN
    p.run()
    torch.cuda.synchronize()
    assert torch.equal(p.out[0, :2, :500], clean[0, :2, :500]) and torch.equal(p.out[0, 2:, :700], clean[0, 2:, :700])
    assert torch.isnan(p.out[0, :2, 500:, 3]).all() and (p.out[0, :2, 500:, 5] == INF).all() and torch.isnan(p.out[0, 2:, 700:]).all()


@pytest.mark.parametrize("case", [
    # fp32 splits with 128 rows a block; 17 to 32 rows on the tensor cores, of few and many items, short and long, ending inside a page
    ("f32", 8, 2, 128, 16, "phsd", [[3001, 2990], [2500, 2400]], [200, 200], False),
    ("bf16", 8, 2, 128, 64, "pshd", [[2500, 2400], [17, 5], [130, 129]], [5, 8, 6], True),
    ("bf16", 4, 1, 64, 16, "phsd", [[333], [90]], [8, 8], False),
    ("bf16", 16, 1, 128, 128, "phsd", [[5000]], [2], False),
    ("bf16", 16, 4, 128, 16, "pshd", [[2222] * 4] * 9, [6] * 9, False),
], ids=lambda c: "-".join(map(str, c)).replace(" ", "")[:70])
def test_attend_row_counts(case):
    a = Attend(*case)
    a.run()
    a.check()


@pytest.mark.parametrize("dtype,max_new", [("bf16", 2), ("bf16", 100), ("f32", 2), ("f32", 100)])
def test_no_new_tokens_at_all(dtype, max_new):
    """A packed chunk of nothing: tensors without elements, whose addresses are null."""
    a = Attend(dtype, 8, 2, 64, 16, "phsd", [[100, 90], [40, 0]], [0, 0], True, max_new=max_new)
    assert a.q.numel() == 0
    a.run()
    torch.cuda.synchronize()
    there = torch.arange(a.c.cap, device="cuda") < a.lengths.cuda().unsqueeze(-1)
    assert torch.equal(a.w_out, torch.where(there, a.w_in, torch.full_like(a.w_in, 77.0))) and (a.lse == 77.0).all()
    a.run(weights=False)
    lengths, out = a.lengths.cuda(), torch.zeros_like(a.lengths).cuda()
    before = a.c.k[0].clone()
    kv = a.q[:, :2]
    positions = torch.zeros(0, dtype=torch.int32, device="cuda")
    wkv.wkv_append_kv_paged(a.cache, kv, kv, lengths, a.c.k[0], a.c.v[0], q=a.q, q_out=a.q, positions=positions, rope=wkv.Rope(64), lengths_out=out)
    torch.cuda.synchronize()
    assert torch.equal(out, lengths) and torch.equal(a.c.k[0].view(torch.uint8), before.view(torch.uint8)) and wkv.device_status(a.ws) == 0


@pytest.mark.parametrize("dtype,d,stride,new", [("bf16", 128, 400_000_000, 1), ("bf16", 128, 400_000_000, 9), ("f32", 64, 200_000_000, 3)])
def test_pools_beyond_32_bits(dtype, d, stride, new):
    """Pages whose offsets pass 2^31 and 2^32: the same bits as in a small pool with the same table."""
    g = gen(21)
    small = Attend(dtype, 8, 2, d, 64, "phsd", [[600, 599]], [new], False, max_pages=10)
    c = small.c
    shape = tuple(c.k[0].shape)
    assert shape[0] == 12 and int(c.table.max()) * stride > (2 ** 32 if dtype == "bf16" else 2 ** 31)
    flat = [torch.empty(11 * stride + shape[1] * shape[2] * d, dtype=c.dtype, device="cuda") for _ in range(2)]
    far = [f.as_strided(shape, (stride, shape[2] * d, d, 1)) for f in flat]
    far_cache = wkv.PagedCache(dtype=dtype, batch=1, n_q_heads=8, n_kv_heads=2, head_dim=d, page_size=64, num_pages=12, block_table=c.table,
                               max_new=new, layout=(stride, shape[2] * d, d))
    for x, y in zip(far, (c.k[0], c.v[0])):
        x.copy_(y)
    k, v = (chunk_of(g, c.dtype, 2, d, [new], False) for _ in range(2))
    pos = torch.arange(new, dtype=torch.int32, device="cuda").view(1, -1) + 700
    rope = wkv.Rope(d)
    results = []
    for cache, pools in ((small.cache, (c.k[0], c.v[0])), (far_cache, far)):
        w, p = small.w_in.clone(), torch.arange(c.cap, dtype=torch.int32, device="cuda").expand(1, 2, -1).contiguous()
        n0, n1, n2 = small.lengths.cuda(), torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros((1, 2), dtype=torch.int32, device="cuda")
        out, ws, q_out = torch.full_like(small.q, 77.0), cache.alloc_workspace(), torch.empty_like(small.q)
        wkv.wkv_append_kv_paged(cache, k, v, n0, pools[0], pools[1], q=small.q, q_out=q_out, positions=pos, rope=rope, lengths_out=n1, row_positions=p,
                                row_weights=w)
        wkv.wkv_attend_paged(cache, q_out, pools[0], pools[1], n1, out, ws, weights_in=w, weights_out=w)
        wkv.wkv_evict_kv_paged(cache, [pools[0]], [pools[1]], w, p, n1, 300, 20, w, p, n2, ws)
        torch.cuda.synchronize()
        assert wkv.device_status(ws) == 0 and (n2 == 300).all()
        results.append([out, q_out, w, p, n1, pools[0], pools[1]])
    for x, y in zip(*results):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype,n", [("bf16", 200), ("bf16", 90), ("f32", 150)])
def test_prompt_queries_beyond_32_bits(dtype, n):
    """Queries and outputs whose last tokens lie behind 2^31 elements."""
    p = Prompt(dtype, 4, 2, 64, [n], "bhnd", 4)
    p.run()
    stride = 2 ** 31 // (n - 4) // 64 * 64
    far = [torch.empty((n - 1) * stride + 4 * 64, dtype=p.q.dtype, device="cuda").as_strided((1, 4, n, 64), (0, 64, stride, 1)) for _ in range(2)]
    far[0].copy_(p.q)
    wkv.wkv_attend_prompt(p.prob, far[0], p.k, p.v, far[1])
    torch.cuda.synchronize()
    assert torch.equal(far[1].contiguous(), p.out)
    rope, turned = wkv.Rope(64), torch.empty_like(p.q)
    wkv.wkv_rotate_prompt(p.prob, rope, p.q, None, turned, None)
    wkv.wkv_rotate_prompt(p.prob, rope, far[0], None, far[0], None)
    torch.cuda.synchronize()
    assert torch.equal(far[0].contiguous(), turned)


def test_calls_on_two_streams_at_once():
    """Each with a workspace of its own: the same bits as one after the other."""
    calls = [Attend("bf16", 8, 2, 128, 64, "pshd", [[5000, 4990], [2100, 700]], [40, 300], True),
             Attend("bf16", 32, 8, 128, 64, "pshd", [[2000] * 8, [1500] * 8], [1, 1], False),
             Attend("f32", 8, 2, 64, 16, "phsd", [[900, 899]], [7], False)]
    prompts = [Prompt("bf16", 8, 2, 128, [2500], "bhnd", 4), Prompt("f32", 4, 2, 64, [700], "bhnd", 4)]
    for a in calls + prompts:
        a.run()
    torch.cuda.synchronize()
    alone = [[x.clone() for x in (a.out, a.lse)] + ([a.w_out.clone()] if isinstance(a, Attend) else []) for a in calls + prompts]
    streams = [torch.cuda.Stream() for _ in calls + prompts]
    for a in calls + prompts:
        a.out.fill_(77.0)
    torch.cuda.synchronize()
    for _ in range(10):
        for a, s in zip(calls + prompts, streams):
            with torch.cuda.stream(s):
                a.run()
    torch.cuda.synchronize()
    for a, want in zip(calls + prompts, alone):
        for x, y in zip([a.out, a.lse] + ([a.w_out] if isinstance(a, Attend) else []), want):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_prompt_and_rotation_captured_and_replayed():
    p = Prompt("bf16", 8, 2, 96, [700, 333], "packed", 8)
    f = Prompt("f32", 4, 2, 64, [600], "bhnd", 8)
    rope, turned = wkv.Rope(64), torch.empty_like(p.q)

    def step():
        wkv.wkv_rotate_prompt(p.prob, rope, p.q, None, turned, None)
        wkv.wkv_attend_prompt(p.prob, turned, p.k, p.v, p.out, p.lse, p.lse_obs, p.status)
        f.run()
    step()
    torch.cuda.synchronize()
    want = [x.clone() for x in (turned, p.out, p.lse, p.lse_obs, f.out)]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
        for x in (turned, p.out, f.out):
            x.fill_(77.0)
        for _ in range(3):
            graph.replay()
    torch.cuda.synchronize()
    for x, y in zip((turned, p.out, p.lse, p.lse_obs, f.out), want):
        assert torch.equal(x, y)
    assert int(p.status) == 0


@pytest.mark.parametrize("budget,layers,n", [(300, 1, 303), (290, 4, 320), (0, 2, 9), (1, 2, 9), (310, 8, 320), (250, 32, 255), (63, 1, 320)])
def test_evict_few_rows(budget, layers, n):
    """With few rows to move, by the budget and the table's size, they are moved without a second kernel: the same as by one of its own.
    With a budget per sequence, whose numbers the host does not see, only the table's size counts."""
    g = gen(31)
    c = ou.Cache(g, torch.bfloat16, 2, 2, 64, 16, 20, "phsd", layers=layers)
    lengths = [[n, max(n - 3, 0)], [min(budget, n), n // 2]]
    c.fill(g, lengths)
    c.table[1, 0] = -1
    cache = paged(c, 4, 1)
    ws = cache.alloc_workspace()
    w = torch.rand((2, 2, c.cap), generator=g).cuda()
    p = torch.randperm(c.cap, generator=g).to(torch.int32).cuda().expand(2, 2, -1).contiguous()
    lens = torch.tensor(lengths, dtype=torch.int32).cuda()
    results, launches = [], []
    for budgets in (None, torch.full((2,), budget, dtype=torch.int32, device="cuda")):
        k, v = [x.clone() for x in c.k], [x.clone() for x in c.v]
        w1, p1, n1 = w.clone(), p.clone(), lens.clone()
        before = wkv.lib().wkv_launch_count()
        wkv.wkv_evict_kv_paged(cache, k, v, w1, p1, n1, budget if budgets is None else 0, 5, w1, p1, n1, ws, budgets=budgets)
        launches.append(wkv.lib().wkv_launch_count() - before)
        torch.cuda.synchronize()
        results.append(k + v + [w1, p1, n1])
    for x, y in zip(*results):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    most = [min(budget, c.cap - budget), c.cap // 2 + 1]
    assert launches == [1 if x <= 256 and x * 8 * 2 * layers <= 4096 else 2 for x in most]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("order", ["half", "interleaved"])
@pytest.mark.parametrize("d,rot", [(72, 2), (72, 62), (72, 66), (72, 70), (72, 72), (40, 36), (128, 120), (128, 126), (8, 6)])
def test_rotate_odd_parts_leave_the_rest_alone(dtype, order, d, rot):
    """Turned parts that end inside 16 bytes: infinities and NaN in the rest and beside it come out as they are, and the turned
    part is, in bits, what it is in a head that ends with it."""
    p = Prompt(dtype, 3, 1, d, [37], "bhnd", 4)
    p.q[..., rot:] = INF
    if rot + 1 < d:
        p.q[..., rot + 1] = NAN
    rope = wkv.Rope(rot, 10000.0, order=order)
    turned = torch.full_like(p.q, 77.0)
    wkv.wkv_rotate_prompt(p.prob, rope, p.q, None, turned, None)
    torch.cuda.synchronize()
    if rot < d:
        assert torch.equal(turned[..., rot:].contiguous().view(torch.uint8), p.q[..., rot:].contiguous().view(torch.uint8))
    angle = torch.arange(37, dtype=torch.float64).view(-1, 1) * torch.tensor(ou.frequencies(rot, 10000.0, "none", 1.0, 0.0), dtype=torch.float64)
    cos, sin = torch.cos(angle).cuda(), torch.sin(angle).cuda()
    x = p.q[..., :rot].double()
    a, b = (x[..., : rot // 2], x[..., rot // 2:]) if order == "half" else (x[..., 0::2], x[..., 1::2])
    u, v = a * cos - b * sin, b * cos + a * sin
    want = torch.cat([u, v], -1) if order == "half" else torch.stack([u, v], -1).flatten(-2)
    size = torch.cat([a.abs() + b.abs()] * 2, -1) if order == "half" else torch.stack([a.abs() + b.abs()] * 2, -1).flatten(-2)
    # sine and cosine from an angle of 32 bits (2^-31 of half a turn, times pi) and their own rounding (2 units), the products' and the sum's
    bound = size * (2.0 ** -29 + 4 * 2.0 ** -24) + (want.abs() * 2.0 ** -8 if dtype == "bf16" else 0)
    ou.assert_close(turned[..., :rot], want, bound, "turned part")
    wkv.wkv_rotate_prompt(p.prob, rope, p.q, None, p.q, None)
    torch.cuda.synchronize()
    assert torch.equal(p.q.view(torch.uint8), turned.view(torch.uint8))
