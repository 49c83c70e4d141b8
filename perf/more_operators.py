"""More operators around the window selection, as timed cases: the norms of queries and keys with their rotary positions in one
pass, a cache of 8-bit rows (new tokens and selected windows quantised as they are written, read back, attended over), and
attention for a tree of drafted tokens.

Where `own` is false, `run` computes them from elementary tensor operations; where it is true, it calls the entry points of
`paper_2503_17922_b200.binding`.

Fields of a case:
  op         "turn"     per-head norms and rotary positions of a prompt's queries and keys
             "store"    new tokens: norms, rotary positions, keys and values quantised into the cache, and the new rows read back
             "fill"     selected windows and observation rows of prompts quantised into the cache, and the rows read back
             "attend"   attention of new tokens over an 8-bit cache, optionally adding up the weight that each row receives
             "tree"     attention of drafted tokens over the cache: each sees the rows before the draft and its own ancestors
  dtype      "bf16" or "f32": of queries, new keys and values, outputs;  cache: "e4m3", "i8" or (tree) "plain", rows of `dtype`
  batch, q_heads, kv_heads, d: attention shape
  n          prompt length (turn, fill) or rows in the cache, new ones included: the longest
  ragged     lengths between n / 2 and n; prompts and chunks of new tokens are packed [T, heads, d]
  layout     "bhnd" or "bnhd" (token-major) for dense prompts, "phsd" or "pshd" (token-major) for pages
  new        new tokens of a sequence (the most, when ragged);  page: rows of a page
  weights    attend: with accumulated weights
  norm       turn, store: with norms;  rot: rotated dimensions;  order: "half" or "interleaved";  axes: position axes
  at         store: position of a sequence's first new token
  alpha, omega, share   fill: observation rows, rows of a window, percent of the windows kept;  layers: of the group

A row of the 8-bit cache is d codes and one exponent e: element = code * 2^e, with the least e >= -100 for which no code passes
the type's largest (448 or 127), and codes rounded to nearest, ties to even.
"""
import math

import torch

own = False

_LARGEST = {"bytes": 7.0e8, "flops": 3.2e11}     # what the largest listed cases cannot do without
_BASE = 500000.0
_EPS = 1e-6


def _case(op, **kw):
    c = dict(op=op, dtype="bf16", batch=1, q_heads=32, kv_heads=8, d=128, ragged=False)
    c.update(kw)
    return c


def listed():
    return [
        # a unit test's or a toy model's prompt in fp32: nothing but latency
        _case("turn", name="tiny-turn-f32", dtype="f32", q_heads=4, kv_heads=2, d=64, n=1024, layout="bhnd", norm=True, rot=64, order="half", axes=1),
        # a full context whose positions have three axes (a video among the text)
        _case("turn", name="turn-32k-axes", n=32768, layout="bnhd", norm=True, rot=128, order="half", axes=3),
        # a decoding batch's next tokens into an 8-bit cache
        _case("store", name="store-batch", cache="e4m3", batch=32, n=8192, new=1, page=64, layout="pshd", ragged=True, norm=True, rot=128, order="half",
              axes=1, at=7000),
        # chunks of a batch's next prompt parts, half of each head rotated
        _case("store", name="store-chunk", cache="i8", batch=4, n=16384, new=512, page=128, layout="phsd", ragged=True, norm=False, rot=64,
              order="interleaved", axes=1, at=15000),
        # the 12 percent that one layer keeps of an 8 K prompt
        _case("fill", name="fill-8k", cache="e4m3", n=8192, page=16, layout="phsd", alpha=32, omega=8, share=12, layers=1),
        # prompts of odd lengths, six query heads per key head, two layers of a group
        _case("fill", name="fill-ragged", cache="i8", batch=8, q_heads=12, kv_heads=2, n=12289, page=64, layout="pshd", ragged=True, alpha=16, omega=32,
              share=30, layers=2),
        # one sequence's next token over the 12 percent of an 8 K prompt that were kept: latency
        _case("attend", name="one-token-8bit", cache="e4m3", n=992, new=1, page=16, layout="phsd", weights=False),
        # a decoding batch over long caches of different lengths, whose rows' weights are added up for the eviction
        _case("attend", name="token-batch-8bit", cache="i8", batch=32, n=8192, new=1, page=64, layout="pshd", ragged=True, weights=True),
        # chunks of a batch's next prompt parts over what is cached already: the largest
        _case("attend", name="chunk-16k-8bit", cache="e4m3", batch=4, n=16384, new=512, page=128, layout="phsd", ragged=True, weights=False),
        # one sequence's draft of a dozen tokens over a short cache: latency
        _case("tree", name="one-tree", cache="plain", n=992, new=12, page=16, layout="phsd"),
        # a batch's drafts over long 8-bit caches of different lengths
        _case("tree", name="tree-batch-8bit", cache="e4m3", batch=16, n=8192, new=64, page=64, layout="pshd", ragged=True),
        # fp32, pages of an odd number of rows
        _case("tree", name="tiny-tree-f32", dtype="f32", cache="plain", batch=3, q_heads=4, kv_heads=2, d=64, n=1027, new=9, page=24, layout="phsd", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))


def draw(rng):
    while True:
        op = rng.choice(["turn", "store", "fill", "attend", "attend", "tree", "tree"])
        kv_heads = rng.choice([1, 2, 3, 4, 8])
        c = _case(op, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), batch=_log_int(rng, 1, 32),
                  q_heads=kv_heads * rng.choice([1, 2, 3, 4, 6, 8]), kv_heads=kv_heads, d=rng.choice([64, 80, 96, 128]),
                  ragged=rng.random() < 0.5)
        if op == "turn":
            c.update(n=_log_int(rng, 1, 16384), layout="bnhd" if c["ragged"] else rng.choice(["bhnd", "bnhd"]))
        else:
            c.update(n=_log_int(rng, 1, 16384), page=rng.choice([8, 16, 24, 32, 64, 128]), layout=rng.choice(["phsd", "pshd"]),
                     cache=rng.choice(["e4m3", "i8"]))
        if op in ("turn", "store"):
            c.update(norm=rng.random() < 0.7, rot=2 * rng.randint(1, c["d"] // 2), order=rng.choice(["half", "interleaved"]), axes=rng.choice([1, 1, 2, 3]))
        if op == "store":
            c.update(new=min(c["n"], 1 if rng.random() < 0.4 else _log_int(rng, 1, 512)), at=_log_int(rng, 1, 1000000))
        if op == "fill":
            c.update(alpha=rng.choice([1, 8, 16, 32, 64]), omega=rng.choice([4, 8, 13, 32, 64]), share=rng.randint(0, 60), layers=rng.randint(1, 4))
        if op == "attend":
            c.update(new=min(c["n"], 1 if rng.random() < 0.5 else _log_int(rng, 1, 512)), weights=rng.random() < 0.5)
        if op == "tree":
            c.update(new=min(c["n"], _log_int(rng, 1, 256)), cache=rng.choice(["plain", "e4m3", "i8"]))
        w = work(c)
        f32_limit = 0.1 if c["dtype"] == "f32" else 1.0
        if w["bytes"] <= _LARGEST["bytes"] and w["flops"] <= f32_limit * _LARGEST["flops"] and _scores(c) <= 2 ** 31 and _cache_bytes(c) <= 2e9:
            return c


# ---- sizes -----------------------------------------------------------------------------------
def _lengths(c):
    """Rows of every sequence: all n, or spread over n / 2 .. n."""
    n, B = c["n"], c["batch"]
    if not c["ragged"]:
        return [n] * B
    return [max(1, n - ((b * 5 + 2) % B) * (n // 2) // B) for b in range(B)]


def _news(c):
    """New tokens of every sequence: all `new`, or spread over 1 .. new (never more than the sequence has rows)."""
    if not c["ragged"]:
        return [c["new"]] * c["batch"]
    return [min(n, 1 + (c["new"] - 1) * ((b * 3 + 1) % c["batch"] + 1) // c["batch"]) for b, n in enumerate(_lengths(c))]


def _cu(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


def _elem(c):
    return 4 if c["dtype"] == "f32" else 2


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _row_bytes(c):
    """Of a row of the cache: its elements, and one byte of scale where they are codes."""
    return c["d"] * _elem(c) if c["cache"] == "plain" else c["d"] + 1


def _scores(c):
    """Scores that the plain form holds at once."""
    return c["batch"] * c["q_heads"] * c["new"] * c["n"] if c["op"] in ("attend", "tree") else 0


def _cache_bytes(c):
    if c["op"] == "turn":
        return 0
    return 10.0 * c.get("layers", 1) * c["batch"] * (c["n"] + c["page"]) * c["kv_heads"] * c["d"]


def _windows(c, n):
    """Windows of a prompt of n tokens, and how many of them are kept."""
    kw = (n - c["alpha"] + c["omega"] - 1) // c["omega"] if n > c["alpha"] else 0
    return kw, kw * c["share"] // 100


def work(case):
    c = case
    e, d, hq, hk = _elem(c), c["d"], c["q_heads"], c["kv_heads"]
    lens = _lengths(c)
    if c["op"] == "turn":
        return {"bytes": 2.0 * sum(lens) * (hq + hk) * d * e, "flops": sum(lens) * (hq + hk) * (3.0 * c["rot"] + (4.0 * d if c["norm"] else 0.0))}
    if c["op"] == "fill":
        # rows are read, written as codes, read back and written as they stand for
        rows = sum(min(n, _windows(c, n)[1] * c["omega"] + c["alpha"]) for n in lens)
        return {"bytes": 2.0 * c["layers"] * rows * hk * (d * e + 2.0 * _row_bytes(c) + 2.0 * d), "flops": 2.0 * c["layers"] * rows * hk * 3.0 * d}
    news = _news(c)
    q = sum(news) * hq * d * e
    if c["op"] == "store":
        per_row = 3.0 * c["rot"] + (4.0 * d if c["norm"] else 0.0)
        return {"bytes": 2.0 * q + 2.0 * sum(news) * hk * (d * e + 2.0 * _row_bytes(c) + 2.0 * d),
                "flops": sum(news) * ((hq + hk) * per_row + 6.0 * hk * d)}
    if c["op"] == "tree":
        pairs = sum(m * (n - m + 1) for m, n in zip(news, lens))         # a token sees what is before the draft, and itself at least
        state = 0.0
    else:
        pairs = sum(m * n - m * (m - 1) / 2 for m, n in zip(news, lens))
        state = 8.0 * hk * sum(lens) if c["weights"] else 0.0
    return {"bytes": 2.0 * q + 2.0 * sum(lens) * hk * _row_bytes(c) + state, "flops": 4.0 * d * hq * pairs}


# ---- what a program has in hand before the call ----------------------------------------------------
def _frequencies(c):
    """Angle per position of every rotated pair (on the host, 64 bits)."""
    return _BASE ** (-2.0 * torch.arange(c["rot"] // 2, dtype=torch.float64) / c["rot"])


def _axis_of_pair(c):
    """Each axis turns a stretch of the pairs."""
    pairs = c["rot"] // 2
    return [min(c["axes"] - 1, i * c["axes"] // pairs) for i in range(pairs)]


def _times_power(x, e):
    """x * 2^e in 32 bits, exactly: the power by its bits (-126 <= e <= 127)."""
    return x * ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _quantised(x, kind):
    """Codes (as 8-bit floats or integers) and exponents of rows [..., d]."""
    y = x.float()
    m, k = torch.frexp(y.abs().amax(-1))
    most, bits = (0.875, 9) if kind == "e4m3" else (0.9921875, 7)           # 448 and 127 as m * 2^k
    e = (k - bits + (m > most)).clamp(min=-100)
    y = _times_power(y, -e.unsqueeze(-1))
    return (y.to(torch.float8_e4m3fn) if kind == "e4m3" else y.round().to(torch.int8)), e


def _pools8(c, pool, normal):
    """A layer's pools of codes with their scales [pages, heads, slots], as bytes: rows of different sizes, as heads have them."""
    codes, scales = [], []
    for _ in range(2):
        x, e = _quantised(normal(*pool) * torch.exp2(normal(*pool[:-1], 1)), c["cache"])
        codes.append(x.view(torch.uint8))
        scales.append((e if c["layout"] == "phsd" else e.transpose(1, 2)).add(127).to(torch.uint8).contiguous())
    return codes, scales


def _trees(c, news, g):
    """For every new token the earlier ones that it descends from, itself included: [B, new, new]; tokens hang on a token before
    them, a few on the last of the context."""
    B, m = c["batch"], c["new"]
    at = torch.rand((B, m), generator=g, device="cuda").cpu()
    root = (torch.rand((B, m), generator=g, device="cuda") < 0.1).cpu()
    sees = torch.zeros((B, m, m), dtype=torch.bool)
    b = torch.arange(B)
    for i in range(m):
        if i > 0:
            parent = (at[:, i] * i).long().clamp(max=i - 1)
            sees[:, i] = sees[b, parent] & ~root[:, i].unsqueeze(-1)
        sees[:, i, i] = True
    there = torch.arange(m) < torch.tensor(news).view(B, 1)
    return (sees & there.unsqueeze(-1)).cuda()


def _words(sees):
    """[..., m] truth values -> int32 words of 32, bit j of a word the j-th."""
    m = sees.shape[-1]
    words = (m + 31) // 32
    x = torch.zeros(sees.shape[:-1] + (words * 32,), dtype=torch.int64, device=sees.device)
    x[..., :m] = sees.long()
    x = (x.unflatten(-1, (words, 32)) << torch.arange(32, device=sees.device)).sum(-1)
    return torch.where(x >= 2 ** 31, x - 2 ** 32, x).to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _dtype(c)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dt)

    B, hq, hk, d = c["batch"], c["q_heads"], c["kv_heads"], c["d"]
    s = {"case": c, "lens": _lengths(c)}
    if c["op"] in ("turn", "store"):
        s["freq"] = _frequencies(c)
        s["q_weight"], s["k_weight"] = (1.0 + 0.2 * normal(d)).to(dt), (1.0 + 0.2 * normal(d)).to(dt)
    if c["op"] in ("turn", "fill"):
        n, T = c["n"], sum(s["lens"])
        s["cu"] = _cu(s["lens"]) if c["ragged"] else None

        def heads(h):
            if c["ragged"]:
                return normal(T, h, d)
            return normal(B, h, n, d) if c["layout"] in ("bhnd", "phsd") else normal(B, n, h, d).transpose(1, 2)

    if c["op"] == "turn":
        s["q"], s["k"] = heads(hq), heads(hk)
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        at = torch.cat([torch.arange(m) for m in s["lens"]]) if c["ragged"] else torch.arange(n).expand(B, n)
        # rows, columns and frames of a picture in the middle: the other axes repeat, the first goes on
        s["positions"] = torch.stack([at] + [at // 7 % (31 + 16 * x) for x in range(1, c["axes"])]).to(torch.int32).contiguous().cuda()
    else:
        page, n = c["page"], c["n"]
        max_pages = (n + page - 1) // page + 1
        num_pages = B * max_pages + 3
        s["max_pages"], s["num_pages"], s["capacity"] = max_pages, num_pages, max_pages * page
        order = torch.randperm(num_pages, generator=g, device="cuda")[: B * max_pages]
        s["table"] = order.view(B, max_pages).to(torch.int32)
        pool = (num_pages, hk, page, d) if c["layout"] == "phsd" else (num_pages, page, hk, d)
        if c["cache"] == "plain":
            s["k_pool"], s["v_pool"] = normal(*pool), normal(*pool)
        else:
            s["codes"], s["scales"] = zip(*[_pools8(c, pool, normal) for _ in range(c.get("layers", 1))])
    if c["op"] == "fill":
        s["k"], s["v"] = [heads(hk) for _ in range(c["layers"])], [heads(hk) for _ in range(c["layers"])]
        kept = [_windows(c, m) for m in s["lens"]]
        s["k_max"] = max(1, max(k for _, k in kept))
        idx = torch.full((B, hk, s["k_max"]), -1, dtype=torch.int64, device="cuda")
        rows = torch.zeros((B, hk), dtype=torch.int64, device="cuda")
        for b, (kw, k) in enumerate(kept):
            r = s["lens"][b] - c["alpha"]
            if k > 0:
                some = torch.argsort(torch.rand((hk, kw), generator=g, device="cuda"), dim=-1)[:, :k].sort(-1).values
                idx[b, :, :k] = some
                rows[b] = k * c["omega"] - (some[:, -1] == kw - 1) * (kw * c["omega"] - r)
            rows[b] += min(c["alpha"], s["lens"][b])
        s["window_idx"], s["kept"] = idx.to(torch.int32), rows.to(torch.int32)
        s["most"] = max(min(m, k * c["omega"] + c["alpha"]) for m, (_, k) in zip(s["lens"], kept))
        s["budgets"] = [c["alpha"] + k * c["omega"] for _, k in kept]
        s["rows"] = [torch.zeros((B, hk, s["most"], d), dtype=torch.bfloat16, device="cuda") for _ in range(2 * c["layers"])]
    if c["op"] in ("store", "attend", "tree"):
        # a head whose selection held the prompt's short last window has a few rows fewer
        rows = torch.tensor(s["lens"], device="cuda").view(B, 1) - torch.arange(hk, device="cuda").view(1, hk) % 3
        s["news"] = _news(c)
        news = torch.tensor(s["news"], device="cuda").view(B, 1)
        rows = torch.maximum(rows, news)
        s["cu"] = _cu(s["news"]) if c["ragged"] else None
        T = sum(s["news"])

        def chunk(h):
            return normal(T, h, d) if c["ragged"] else normal(B, h, c["new"], d)

        s["q"] = chunk(hq)
        s["q_out"] = torch.empty_like(s["q"])
        if c["op"] == "store":
            rows = rows - news
            s["k"], s["v"] = chunk(hk), chunk(hk)
            first = torch.repeat_interleave(torch.tensor(_cu(s["news"])[:-1]), torch.tensor(s["news"]))
            at = c["at"] + torch.arange(T) - first
            s["positions"] = torch.stack([at] + [at // 7 % (31 + 16 * x) for x in range(1, c["axes"])]).to(torch.int32).contiguous().cuda()
            if not c["ragged"]:
                s["positions"] = s["positions"].view(c["axes"], B, c["new"])
            s["lengths_out"] = torch.zeros((B, hk), dtype=torch.int32, device="cuda")
            s["rows"] = [torch.zeros((B, hk, c["new"], d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        s["lengths"] = rows.to(torch.int32).contiguous()
        if c["op"] != "store":
            s["lse"] = torch.zeros((B, hq, c["new"]), device="cuda")
        if c["op"] == "attend" and c["weights"]:
            s["weights"] = torch.rand((B, hk, s["capacity"]), generator=g, device="cuda")
            s["weights_out"] = torch.zeros_like(s["weights"])
        if c["op"] == "tree":
            s["sees"] = _trees(c, s["news"], g)
            words = _words(s["sees"])
            s["masks"] = _packed(words.unsqueeze(1), s["news"])[:, 0].contiguous() if c["ragged"] else words
    if own:
        s["calls"] = _handles(c, s)
    return s


def _handles(c, s):
    """The calls with their arguments laid out once, as an engine keeps them per layer."""
    from paper_2503_17922_b200 import binding as wkv
    shape = dict(dtype=c["dtype"], batch=c["batch"], n_q_heads=c["q_heads"], n_kv_heads=c["kv_heads"], head_dim=c["d"])
    more = {}
    if c["op"] in ("turn", "store"):
        more = dict(rope=wkv.Rope(c["rot"], _BASE, order=c["order"]), axes=wkv.RopeAxes(_axis_of_pair(c), c["axes"]) if c["axes"] > 1 else None,
                    norm=wkv.HeadNorm(s["q_weight"], s["k_weight"], eps=_EPS) if c["norm"] else None,
                    positions=s["positions"] if c["axes"] > 1 else s["positions"][0])
    if c["op"] in ("turn", "fill"):
        prob = wkv.Problem(l_obs=c.get("alpha", 1), window=c.get("omega", 8), task=0, top_p=0, max_seqlen=c["n"],
                           budgets=s.get("budgets") or [c["n"]] * c["batch"], cu_seqlens=s["cu"],
                           kv_layout="bhnd" if c["layout"] in ("bhnd", "phsd") else "bnhd", **shape)
    if c["op"] == "turn":
        return [wkv.prepare_norm_rotate_prompt(prob, s["q"], s["k"], s["q_out"], s["k_out"], **more)]
    paged = dict(page_size=c["page"], num_pages=s["num_pages"], block_table=s["table"], max_new=c.get("new", 1),
                 cu_new=s["cu"] if c["op"] != "fill" else None, layout=c["layout"], **shape)
    if c["cache"] == "plain":
        cache = wkv.PagedCache(**paged)
        return [wkv.prepare_attend_draft_paged(cache, s["masks"], s["q"], s["k_pool"], s["v_pool"], s["lengths"], s["q_out"],
                                              cache.alloc_workspace(), lse=s["lse"])]
    cache = wkv.PagedCache8(kind=c["cache"], **paged)
    layers = [wkv.Layer8(cache, k, v, k_scales, v_scales) for (k, v), (k_scales, v_scales) in zip(s["codes"], s["scales"])]
    if c["op"] == "fill":
        return [wkv.prepare_gather_kv_paged8(prob, cache, layers, s["k"], s["v"], s["window_idx"])] + [
            wkv.prepare_read_kv_paged8(cache, layer, s["kept"], s["rows"][2 * i], s["rows"][2 * i + 1]) for i, layer in enumerate(layers)]
    if c["op"] == "store":
        return [wkv.prepare_append_kv_paged8(cache, layers[0], s["k"], s["v"], s["lengths"], q=s["q"], q_out=s["q_out"],
                                             lengths_out=s["lengths_out"], **more),
                wkv.prepare_read_kv_paged8(cache, layers[0], s["lengths_out"], s["rows"][0], s["rows"][1], first=s["lengths"])]
    return [wkv.prepare_attend_paged8(cache, layers[0], s["q"], s["lengths"], s["q_out"], cache.alloc_workspace(), lse=s["lse"],
                                      weights_in=s.get("weights"), weights_out=s.get("weights_out"), draft=s.get("masks"))]


# ---- one pass ----------------------------------------------------------------------------------
def run(state):
    s, op = state, state["case"]["op"]
    if own:
        for call in s["calls"]:
            call.run()
        if op == "turn":
            return {"q": s["q_out"], "k": s["k_out"]}
        if op == "store":
            return {"q": s["q_out"], "k_rows": s["rows"][0], "v_rows": s["rows"][1], "lengths": s["lengths_out"]}
        if op == "fill":
            return {"rows": s["rows"]}
        return {"out": s["q_out"], "lse": s["lse"], "weights": s.get("weights_out")}
    return {"turn": _turn, "store": _store, "fill": _fill, "attend": _attend, "tree": _attend}[op](s)


def _padded(x, cu, most):
    """Packed [T, h, d] -> [B, h, most, d]; rows behind a sequence's last are repetitions of some row (masked or unused)."""
    at = torch.tensor(cu[:-1], device=x.device).view(-1, 1) + torch.arange(most, device=x.device).view(1, -1)
    return x[at.clamp(max=x.shape[0] - 1)].transpose(1, 2)


def _packed(x, lens):
    """[B, h, most, d] -> packed [T, h, d]."""
    there = torch.arange(x.shape[2], device=x.device).view(1, -1) < torch.tensor(lens, device=x.device).view(-1, 1)
    return x.transpose(1, 2)[there]


def _angles(s):
    """[..., rot / 2] for positions [axes, ...], 64 bits."""
    axis = torch.tensor(_axis_of_pair(s["case"]), device="cuda")
    return s["positions"].double().movedim(0, -1)[..., axis] * s["freq"].cuda()


def _turned(x, weight, angle, c):
    """x [..., d]: its norm, then the first `rot` dimensions rotated by `angle`; in 32 bits."""
    y = x.float()
    if c["norm"]:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + _EPS) * weight.float()
    rot = c["rot"]
    cos, sin = angle.cos().float(), angle.sin().float()
    if c["order"] == "half":
        a, b = y[..., : rot // 2], y[..., rot // 2: rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1)


def _turn(s):
    c = s["case"]
    angle = _angles(s).unsqueeze(1)                                       # [T, 1, .] or [B, 1, n, .]
    return {"q": _turned(s["q"], s["q_weight"], angle, c).to(_dtype(c)), "k": _turned(s["k"], s["k_weight"], angle, c).to(_dtype(c))}


def _places(s, b, h, row):
    """Index of row `row` of unit (b, h) in a pool, and in its scales."""
    c = s["case"]
    page, slot = s["table"][b, row // c["page"]].long(), row % c["page"]
    return ((page, h, slot) if c["layout"] == "phsd" else (page, slot, h)), (page, h, slot)


def _put(s, layer, kv, at, x):
    """Rows x [..., d] quantised into a layer's pool."""
    codes, e = _quantised(x, s["case"]["cache"])
    s["codes"][layer][kv][at[0]] = codes.view(torch.uint8)
    s["scales"][layer][kv][at[1]] = (e + 127).to(torch.uint8)


def _got(s, layer, kv, at):
    """Rows of a layer's pool as what they stand for, in 32 bits."""
    codes = s["codes"][layer][kv][at[0]].view(torch.float8_e4m3fn if s["case"]["cache"] == "e4m3" else torch.int8)
    return _times_power(codes.float(), s["scales"][layer][kv][at[1]].int().unsqueeze(-1) - 127)


def _store(s):
    c = s["case"]
    B, hk, new = c["batch"], c["kv_heads"], c["new"]
    news = torch.tensor(s["news"], device="cuda")
    angle = _angles(s).unsqueeze(1)
    q = _turned(s["q"], s["q_weight"], angle, c).to(_dtype(c))
    k, v = _turned(s["k"], s["k_weight"], angle, c), s["v"].float()
    if c["ragged"]:
        b = torch.repeat_interleave(torch.arange(B, device="cuda"), news).view(-1, 1)
        nth = (torch.arange(b.shape[0], device="cuda") - (news.cumsum(0) - news)[b.view(-1)]).view(-1, 1)
        h = torch.arange(hk, device="cuda").view(1, -1)
    else:
        b, h, nth = (torch.arange(x, device="cuda") for x in (B, hk, new))
        b, h, nth = b.view(-1, 1, 1), h.view(1, -1, 1), nth.view(1, 1, -1)
    at = _places(s, b, h, s["lengths"].long()[b, h] + nth)
    out = {"q": q, "lengths": s["lengths"] + news.view(-1, 1).to(torch.int32)}
    b, h, nth = torch.broadcast_tensors(b, h, nth)
    for kv, (name, x) in enumerate((("k_rows", k), ("v_rows", v))):
        _put(s, 0, kv, at, x)
        rows = torch.zeros((B, hk, new, c["d"]), dtype=torch.bfloat16, device="cuda")
        rows[b, h, nth] = _got(s, 0, kv, at).to(torch.bfloat16)
        out[name] = rows
    return out


def _fill(s):
    c = s["case"]
    B, hk, omega, alpha = c["batch"], c["kv_heads"], c["omega"], c["alpha"]
    lens = torch.tensor(s["lens"], device="cuda").view(B, 1, 1)
    kept = s["kept"].long().unsqueeze(-1)
    r = torch.arange(s["most"], device="cuda").view(1, 1, -1)
    there = r < kept
    review = kept - lens.clamp(max=alpha)                                  # rows of the windows
    nth = (r // omega).clamp(max=s["k_max"] - 1)
    of_window = s["window_idx"].long().gather(-1, nth.expand(B, hk, -1)) * omega + r % omega
    source = torch.where(r < review, of_window, lens - kept + r)
    b, h, to = there.nonzero(as_tuple=True)
    source = source[b, h, to]
    if c["ragged"]:
        source = source + torch.tensor(s["cu"][:-1], device="cuda")[b]
    at = _places(s, b, h, to)
    got = []
    for layer in range(c["layers"]):
        for kv, x in enumerate((s["k"][layer], s["v"][layer])):
            _put(s, layer, kv, at, x[source, h] if c["ragged"] else x[b, h, source])
            rows = torch.zeros((B, hk, s["most"], c["d"]), dtype=torch.bfloat16, device="cuda")
            rows[b, h, to] = _got(s, layer, kv, at).to(torch.bfloat16)
            got.append(rows)
    return {"rows": got}


def _cached(s, kv):
    """The first n rows of every unit in order, [B, hk, n, d] in 32 bits."""
    c = s["case"]
    if c["cache"] == "plain":
        x = s["v_pool" if kv else "k_pool"][s["table"].long()].float()                # [B, pages, ., ., d]
    else:
        codes = s["codes"][0][kv][s["table"].long()].view(torch.float8_e4m3fn if c["cache"] == "e4m3" else torch.int8)
        e = s["scales"][0][kv][s["table"].long()].int() - 127                         # [B, pages, hk, page]
        x = _times_power(codes.float(), (e if c["layout"] == "phsd" else e.transpose(2, 3)).unsqueeze(-1))
    x = x.transpose(1, 2) if c["layout"] == "phsd" else x.permute(0, 3, 1, 2, 4)
    return x.flatten(2, 3)[:, :, : c["n"]]


def _attend(s):
    c = s["case"]
    B, hk, G, new, n = c["batch"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["new"], c["n"]
    q = _padded(s["q"], s["cu"], new) if c["ragged"] else s["q"]
    q = q.float().unflatten(1, (hk, G))
    k, v = _cached(s, 0), _cached(s, 1)
    news = torch.tensor(s["news"], device="cuda").view(B, 1, 1)
    nth = torch.arange(new, device="cuda").view(1, 1, -1)
    row = torch.arange(n, device="cuda")
    before = s["lengths"].long().unsqueeze(-1) - news                                 # [B, hk, 1]: rows in front of the new ones
    if c["op"] == "tree":
        # row j of a unit is new token j - before of its sequence
        place = row - before
        among = s["sees"].unsqueeze(1).expand(B, hk, new, new).gather(-1, place.clamp(0, new - 1).unsqueeze(2).expand(B, hk, new, n))
        sees = (place < 0).unsqueeze(2) | (among & (place < news).unsqueeze(2))
    else:
        sees = row < (before + nth + 1).unsqueeze(-1)
    sees = sees & (nth < news).unsqueeze(-1)
    x = torch.matmul(q.flatten(2, 3), k.transpose(-1, -2)).unflatten(2, (G, new)) / math.sqrt(c["d"])
    x.masked_fill_(~sees.unsqueeze(2), float("-inf"))
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    p = x.sub_(top).exp_()
    z = p.sum(-1, keepdim=True)
    z = torch.where(z == 0, torch.ones_like(z), z)
    out = (torch.matmul(p.flatten(2, 3), v).unflatten(2, (G, new)) / z).flatten(1, 2).to(_dtype(c))
    lse = torch.where(nth < news, (z.log() + top).squeeze(-1).flatten(1, 2), torch.zeros((), device="cuda"))
    weights = None
    if c.get("weights"):
        # a sum of few positive terms beside a term of a thousand cached rows' size: 64 bits for the column sums
        mine = p.div_(z).sum((2, 3), dtype=torch.float64)
        there = row < s["lengths"].unsqueeze(-1)
        weights = torch.zeros_like(s["weights"])
        weights[:, :, :n] = torch.where(there, s["weights"][:, :, :n] + mine, torch.zeros_like(mine)).float()
    return {"out": _packed(out, s["news"]) if c["ragged"] else out, "lse": lse, "weights": weights}


# ---- the definition in 64 bits ------------------------------------------------------------------
def _exact_turned(x, weight, positions, c, freq):
    """Rows x [rows, d] at positions [axes, rows]."""
    y = x.double()
    if c["norm"]:
        y = y / torch.sqrt((y ** 2).sum(1, keepdim=True) / c["d"] + _EPS) * weight.double()
    z = y.clone()
    for i, axis in enumerate(_axis_of_pair(c)):
        j, k = (i, i + c["rot"] // 2) if c["order"] == "half" else (2 * i, 2 * i + 1)
        a = positions[axis].double() * float(freq[i])
        z[:, j] = y[:, j] * torch.cos(a) - y[:, k] * torch.sin(a)
        z[:, k] = y[:, j] * torch.sin(a) + y[:, k] * torch.cos(a)
    return z


def _two_to(e):
    """2^e for whole numbers e, from the language's own powers (-200 <= e <= 200)."""
    return torch.tensor([2.0 ** k for k in range(-200, 201)], dtype=torch.float64, device="cuda")[(e + 200).long()]


def _exact_held(x, kind):
    """What the cache holds of rows x [rows, d]: the nearest multiple of the code's step, ties to even."""
    y = x.double()
    most = 448.0 if kind == "e4m3" else 127.0
    big = y.abs().amax(1)
    e = torch.ceil(torch.log2(big / most)).clamp(min=-100)
    e = torch.where(big > most * _two_to(e), e + 1, e)                    # (the logarithm's own rounding)
    e = torch.where((e > -100) & (big <= most * _two_to(e - 1)), e - 1, e)
    y = y / _two_to(e)[:, None]
    step = torch.ones_like(y)
    if kind == "e4m3":                                                    # three bits behind the first, which is 2^-6 at least
        step = _two_to(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * _two_to(e)[:, None]


def exact(case, seed):
    global own
    c, was = case, own
    own = False
    s = prepare(case, seed)
    own = was
    B, hq, hk, d = c["batch"], c["q_heads"], c["kv_heads"], c["d"]
    G = hq // hk
    f64 = torch.float64

    def turned(name, heads):
        x = s[name]
        z = torch.empty(x.shape, dtype=f64, device="cuda")
        for h in range(heads):
            if c["ragged"]:
                z[:, h] = _exact_turned(x[:, h], s[name + "_weight"], s["positions"], c, s["freq"])
            else:
                for b in range(B):
                    z[b, h] = _exact_turned(x[b, h], s[name + "_weight"], s["positions"][:, b], c, s["freq"])
        return z

    if c["op"] == "turn":
        return {"q": turned("q", hq), "k": turned("k", hk)}
    if c["op"] == "store":
        # Values are quantised as they stand.  Of the keys, one that lies as near to a border of two codes as 32 bits can tell takes either
        # code: they have no such value.
        rows = torch.zeros((B, hk, c["new"], d), dtype=f64, device="cuda")
        for b, m in enumerate(s["news"]):
            for h in range(hk):
                rows[b, h, :m] = _exact_held(s["v"][s["cu"][b]:s["cu"][b] + m, h] if c["ragged"] else s["v"][b, h], c["cache"])
        return {"q": turned("q", hq), "k_rows": None, "v_rows": rows, "lengths": None}
    if c["op"] == "fill":
        got = []
        for layer in range(c["layers"]):
            for x in (s["k"][layer], s["v"][layer]):
                rows = torch.zeros((B, hk, s["most"], d), dtype=f64, device="cuda")
                for b, n in enumerate(s["lens"]):
                    for h in range(hk):
                        from_ = []
                        for w in s["window_idx"][b, h].tolist():
                            if w >= 0:
                                from_ += range(w * c["omega"], min((w + 1) * c["omega"], n - c["alpha"]))
                        from_ += range(max(0, n - c["alpha"]), n)
                        mine = x[s["cu"][b]:s["cu"][b] + n, h] if c["ragged"] else x[b, h]
                        rows[b, h, : len(from_)] = _exact_held(mine[torch.tensor(from_, device="cuda")], c["cache"])
                got.append(rows)
        return {"rows": got}

    def rows_of(kv, b, h, count):
        at = torch.arange(count, device="cuda")
        page, slot = s["table"][b][at // c["page"]].long(), at % c["page"]
        pool = s["v_pool" if kv else "k_pool"] if c["cache"] == "plain" else s["codes"][0][kv].view(
            torch.float8_e4m3fn if c["cache"] == "e4m3" else torch.int8).float()
        x = (pool[page, h, slot] if c["layout"] == "phsd" else pool[page, slot, h]).double()
        if c["cache"] != "plain":
            x = x * _two_to(s["scales"][0][kv][page, h, slot].int() - 127)[:, None]
        return x

    out = torch.zeros(s["q"].shape, dtype=f64, device="cuda")
    lse = torch.zeros((B, hq, c["new"]), dtype=f64, device="cuda")
    weights = torch.zeros(s["weights"].shape, dtype=f64, device="cuda") if c.get("weights") else None
    for b, m in enumerate(s["news"]):
        for h in range(hk):
            n = int(s["lengths"][b, h])
            keys, values = rows_of(0, b, h, n), rows_of(1, b, h, n)
            sees = torch.ones((m, n), dtype=torch.bool, device="cuda")
            sees[:, n - m:] = s["sees"][b, :m, :m] if c["op"] == "tree" else torch.tril(sees[:, :m])
            if weights is not None:
                weights[b, h, :n] = s["weights"][b, h, :n].double()
            for head in range(h * G, h * G + G):
                part = (slice(s["cu"][b], s["cu"][b] + m), head) if c["ragged"] else (b, head)
                x = s["q"][part].double() @ keys.T * d ** -0.5
                x[~sees] = float("-inf")
                l = torch.logsumexp(x, 1)
                p = torch.exp(x - l[:, None])
                out[part], lse[b, head, :m] = p @ values, l
                if weights is not None:
                    weights[b, h, :n] += p.sum(0)
    return {"out": out, "lse": lse, "weights": weights}
